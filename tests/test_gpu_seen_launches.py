"""GPU: batches of few rows that take more than one launch: more records than the workspace holds (fewer entries a launch, and one entry
too long for them at all in tiles), and more metadata than one upload. Against the oracle, in the first launch and in later ones."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import seen as so
from tests.helpers import f64
from tests.seen_helpers import assert_within, tree

pytestmark = pytest.mark.gpu

# Records have room for 512 tiles of 256 rows (and their sums): a kv head's 64 rows of one item are a quarter and a little more of such a tile,
# so 64 kv heads at head dim 64 leave room for 32 items of four blocks of rows. Items are 8192 keys at the longest.
HQ, HKV, D, ROOM = 512, 64, 64, 32


def _randn(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _pool(fmt, hq, hkv, d, lens):
    from paper_2606_01839_amd import KVPool
    pages = [(n + 15) // 16 for n in lens]
    pool = KVPool(1, hq, hkv, d, n_pages=sum(pages) + 2, max_convs=len(lens), max_pages_per_conv=max(pages), placement_seed=3, device="cuda",
                  kv_format=fmt)
    convs = [pool.conv_create() for _ in lens]
    for i, (c, n) in enumerate(zip(convs, lens)):
        for a in range(0, n, 32768):
            m = min(n - a, 32768)
            pool.kv_append(c, _randn((1, m, hkv, d), 1000 * i + a // 32768), _randn((1, m, hkv, d), 500000 + 1000 * i + a // 32768))
    return pool, convs


def _launches(pool, call):
    pool.profile_start()
    out = call()
    return out, pool.profile_stop()["attn_fwd"][1]


def _check_heads(pool, conv, length, q, out, see, fmt, heads, rows, what):
    """Some rows and query heads of an entry."""
    k, v = pool.kv_read([conv], [0], [length])
    group = pool.n_q_heads // pool.n_kv_heads
    rows = torch.tensor(rows)
    for h in heads:
        kf, vf = (f64(x[0, :, h // group:h // group + 1].cpu()) for x in (k, v))
        qf, o = f64(q[rows][:, h:h + 1].cpu()), out[rows][:, h:h + 1].cpu()
        s = np.ones((len(rows), length), dtype=bool) if see is None else see[rows.numpy()]
        assert_within(o, qf, kf, vf, s, so.attend(qf, kf, vf, s), f"{what} head {h}", fmt == "fp4")


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_more_records_than_room(fmt):
    """Trees whose items do not fit the records at any size: the batch is halved, and its second half is a launch of its own."""
    lens = [8300 + 61 * i for i in range(20)]      # two items each: 40 of 32
    ns = [8 - i % 3 for i in range(20)]            # 64, 56 and 48 rows a kv head
    pool, convs = _pool(fmt, HQ, HKV, D, lens)
    parents = [tree(n, i) for i, n in enumerate(ns)]
    q = 4 * _randn((sum(ns), HQ, D), 7)   # scores that few keys win: a wrong key or row is far off
    whole = torch.full((sum(ns) + 8, HQ, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:sum(ns)]
    _, launches = _launches(pool, lambda: pool.attn_tree(convs, ns, parents, 0, q, out))
    assert launches >= 4 and (whole[sum(ns):] == 7).all()
    for i in (0, 1, 4, 5, 9, 10, 11, 14, 15, 19):
        r0 = sum(ns[:i])
        _check_heads(pool, convs[i], lens[i], q[r0:r0 + ns[i]], out[r0:r0 + ns[i]], so.tree_sees(parents[i], lens[i]), fmt, (0, 77, 511),
                     [0, ns[i] - 1], f"conversation {i}")
    assert torch.equal(pool.attn_tree(convs, ns, parents, 0, q), out)
    for i in (0, 19):   # a batch of its own: other items, the same up to their rounding
        r0 = sum(ns[:i])
        alone = pool.attn_tree([convs[i]], [ns[i]], [parents[i]], 0, q[r0:r0 + ns[i]].contiguous()).float()
        assert (alone - out[r0:r0 + ns[i]].float()).norm() < 2 * 2.0 ** -8 * alone.norm()   # bf16 weights at other maxima, bf16 outputs
    pool.close()


def test_one_entry_of_more_records_than_room():
    """Beside short ones, of which one is long enough for records too: the long one goes to the tiles."""
    lens = [400, (ROOM + 1) * 8192 + 777, 9000, 30]
    ns = [3, 8, 8, 2]
    pool, convs = _pool("fp4", HQ, HKV, D, lens)
    for call, see in ((lambda q: pool.attn_tree(convs, ns, [tree(n, i) for i, n in enumerate(ns)], 0, q), True),
                      (lambda q: pool.attn_cross(convs, ns, 0, q), False)):
        q = 4 * _randn((sum(ns), HQ, D), 9)
        out, launches = _launches(pool, lambda: call(q))
        assert launches >= 4   # rows, the long one's tiles and their merge, rows and their merge
        for i in range(4):
            r0 = sum(ns[:i])
            long = i == 1
            _check_heads(pool, convs[i], lens[i], q[r0:r0 + ns[i]], out[r0:r0 + ns[i]], so.tree_sees(tree(ns[i], i), lens[i]) if see else None,
                         "fp4", (511,) if long else (0, 200), [ns[i] - 1] if long else [0, ns[i] - 1], f"conversation {i} {see}")
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_more_metadata_than_an_upload(fmt):
    """120,000 entries of one to three rows on a few conversations, one of them long enough for records."""
    hq, hkv, d = 4, 2, 64
    lens = [40, 9000, 1, 100, 16]
    pool, convs = _pool(fmt, hq, hkv, d, lens)
    n = 120000
    pick = [(0, 2, 3, 4)[i % 4] if i % 1000 else 1 for i in range(n)]
    ns = [1 + i % 3 for i in range(n)]
    rows = np.concatenate([[0], np.cumsum(ns)])
    q = _randn((int(rows[-1]), hq, d), 10)
    whole = torch.full((int(rows[-1]) + 8, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    _, launches = _launches(pool, lambda: pool.attn_cross([convs[i] for i in pick], ns, 0, q, whole[:-8]))
    assert launches > 4 and (whole[-8:] == 7).all()
    kv = pool.kv_read(convs, [0] * 5, lens)
    kv = list(zip(*(x[0].split(lens) for x in kv)))
    # every row by float64 products on the GPU, entries of one conversation together
    pick_t = torch.repeat_interleave(torch.tensor(pick, device="cuda"), torch.tensor(ns, device="cuda"))
    for c in range(5):
        at = torch.nonzero(pick_t == c).flatten()
        if len(at) == 0:
            continue
        k, v = (x.double().repeat_interleave(hq // hkv, 1) for x in kv[c])
        for part in at.split(40000):
            for h in range(hq):
                x = q[part, h].double()
                w = torch.softmax(x @ k[:, h].t().contiguous() / d ** 0.5, 1)
                ref = w @ v[:, h].contiguous()
                # the bound of seen_helpers, |V - O| taken as |V| + |O|; 2^-20 for the fp32 exponents, scores being below 2^4
                delta = 2.0 ** -8 + 2.0 ** -20
                if fmt == "fp4":
                    off = 2.0 ** -16 * x.abs().amax(1, keepdim=True) * k[:, h].abs().sum(1).max() / d ** 0.5
                    delta = delta + torch.expm1(2 * off)
                mean = w @ v[:, h].abs().contiguous()
                got = whole[part, h].double()
                tol = delta / (1 - delta) * (mean + ref.abs()) + 2.0 ** -12 * mean + 2.0 ** -8 * got.abs()
                assert ((got - ref).abs() <= tol).all(), (c, h)
    for i in (0, 1, 39999, 40000, n - 1):   # and by the oracle's bound
        a, b = int(rows[i]), int(rows[i + 1])
        kf, vf, qf = f64(kv[pick[i]][0].cpu()), f64(kv[pick[i]][1].cpu()), f64(q[a:b].cpu())
        see = np.ones((b - a, lens[pick[i]]), dtype=bool)
        assert_within(whole[a:b].cpu(), qf, kf, vf, see, so.attend(qf, kf, vf, see), f"entry {i}", fmt == "fp4")
    pool.close()
