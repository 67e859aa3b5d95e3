"""GPU: attention of drafted token trees, their append at tree positions, keeping the accepted tokens, and cross
attention, against the oracle in 64 bits; tolerances are the derived bounds of tests/seen_helpers.py, and bit equality
where bytes only move."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import rope as orope
from oracle import seen as so
from tests.helpers import f64, half_ulp_bf16, kv_tokens, q_tokens
from tests.seen_helpers import assert_within, tree

pytestmark = pytest.mark.gpu

SEED = 77
SHAPES = [(32, 8, 128), (4, 2, 64), (8, 8, 128), (16, 8, 64), (8, 1, 128), (6, 3, 64), (64, 8, 128)]


def _pool(hq, hkv, d, fmt="bf16", nl=1, n_pages=1024, max_convs=16, max_pages=1024, seed=3):
    from paper_2606_01839_amd import KVPool
    return KVPool(nl, hq, hkv, d, n_pages=n_pages, max_convs=max_convs, max_pages_per_conv=max_pages, placement_seed=seed,
                  device="cuda", kv_format=fmt)


def _held(k, v, fmt):
    return o4.held(f64(k), f64(v)) if fmt == "fp4" and k.numel() else (f64(k), f64(v))   # (the oracle takes no empty cache)


def _fill(pool, lens, hkv, d, nl=1):
    kv = [kv_tokens(SEED, i, nl, 0, n, hkv, d) for i, n in enumerate(lens)]
    convs = [pool.conv_create() for _ in lens]
    pool.kv_append_batch(convs, lens, *(torch.cat([x[j] for x in kv], 1).contiguous().cuda() for j in (0, 1)))
    return convs, kv


def _queries(ns, hq, d):
    return torch.cat([q_tokens(SEED, 50 + i, 0, 0, n, hq, d) for i, n in enumerate(ns)])


def _check(out, q, ns, kv, sees, fmt, what):
    r0 = 0
    for i, n in enumerate(ns):
        k, v = _held(kv[i][0][0], kv[i][1][0], fmt)
        qi = f64(q[r0:r0 + n])
        see = np.ones((n, k.shape[0]), dtype=bool) if sees[i] is None else sees[i]
        if n and k.shape[0]:
            assert_within(out[r0:r0 + n].cpu(), qi, k, v, see, so.attend(qi, k, v, see), f"{what} conversation {i}", fmt == "fp4")
        r0 += n


# (prefix, tree) of each conversation of a batch: page, word and tile borders, no prefix at all, chains and stars
BATCHES = {
    "one token": [(0, 1), (1, 1), (15, 1), (16, 1), (333, 1)],
    "small": [(100, 3), (0, 7), (31, 5), (64, 2), (17, 0), (2000, 6)],
    "borders": [(31, 16), (32, 17), (33, 15), (47, 16), (63, 16), (64, 16), (65, 9)],
    "wide": [(0, 64), (50, 65), (1000, 100), (127, 63)],
    "very wide": [(300, 250), (10, 33), (70, 300)],
    "long": [(5000, 8), (9000, 13), (1200, 4)],
    "one long": [(16000, 16)],
}
LONG_SHAPES = [(32, 8, 128), (4, 2, 64), (8, 8, 128), (16, 8, 64)]   # those of the two largest batches
TREES = [(b, *s) for b in BATCHES for s in SHAPES if b not in ("very wide", "one long") or s in LONG_SHAPES]


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("batch,hq,hkv,d", TREES)
def test_tree(batch, hq, hkv, d, fmt):
    sizes = BATCHES[batch]
    lens, ns = [p + n for p, n in sizes], [n for _, n in sizes]
    pool = _pool(hq, hkv, d, fmt, n_pages=sum((x + 15) // 16 for x in lens) + 4)
    convs, kv = _fill(pool, lens, hkv, d)
    parents = [tree(n, i, ("mixed", "chain", "star", "mixed")[i % 4]) for i, n in enumerate(ns)]
    q = _queries(ns, hq, d)
    out = pool.attn_tree(convs, ns, parents, 0, q.cuda())
    again = pool.attn_tree(convs, ns, parents, 0, q.cuda())
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    _check(out, q, ns, kv, [so.tree_sees(p, L) if p else None for p, L in zip(parents, lens)], fmt, f"tree {batch}")
    pool.close()


def test_largest_tree_and_layers():
    """CS_MAX_DRAFT tokens behind a prefix, in the second layer of a pool."""
    hq, hkv, d, n, prefix = 4, 2, 64, 1024, 77
    pool = _pool(hq, hkv, d, nl=2, n_pages=80)
    convs, kv = _fill(pool, [prefix + n], hkv, d, nl=2)
    parents = [tree(n, 5)]
    q = _queries([n], hq, d)
    out = pool.attn_tree(convs, [n], parents, 1, q.cuda())
    torch.cuda.synchronize()
    k, v, qf = f64(kv[0][0][1]), f64(kv[0][1][1]), f64(q)
    see = so.tree_sees(parents[0], prefix + n)
    assert_within(out.cpu(), qf, k, v, see, so.attend(qf, k, v, see), "largest tree")
    pool.close()


def test_many_trees_in_several_uploads():
    """More words than one metadata upload holds (2 MiB): the batch is cut."""
    hq, hkv, d, n = 2, 2, 64, 1000
    convs_n = 24
    pool = _pool(hq, hkv, d, n_pages=convs_n * 66, max_convs=convs_n)
    lens = [n + 3 * i for i in range(convs_n)]
    convs, kv = _fill(pool, lens, hkv, d)
    parents = [tree(n, i) for i in range(convs_n)]
    ns = [n] * convs_n
    q = _queries(ns, hq, d)
    out = pool.attn_tree(convs, ns, parents, 0, q.cuda())
    torch.cuda.synchronize()
    pick = [0, 1, convs_n // 2, convs_n - 1]
    for i in pick:
        k, v, qf = f64(kv[i][0][0]), f64(kv[i][1][0]), f64(q[i * n:(i + 1) * n])
        see = so.tree_sees(parents[i], lens[i])
        assert_within(out[i * n:(i + 1) * n].cpu(), qf, k, v, see, so.attend(qf, k, v, see), f"conversation {i}")
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 8), (4, 2, 64, 20), (8, 8, 128, 70), (32, 8, 128, 100), (8, 2, 64, 120)])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_branches_do_not_meet(hq, hkv, d, n, fmt, bad):
    """A token of one branch holds NaN or infinities in K and V: the rows that do not see it have the oracle's values, those that do
    are not finite."""
    prefix, x = 45, float(bad)
    k, v = kv_tokens(SEED, 0, 1, 0, prefix + n, hkv, d)
    sick = prefix + n // 2
    k[0, sick, :, 3] = x
    v[0, sick, :, 5] = x
    pool = _pool(hq, hkv, d, fmt)
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    parents = tree(n, 9)
    q = _queries([n], hq, d)
    out = pool.attn_tree([c], [n], [parents], 0, q.cuda())
    torch.cuda.synchronize()
    see = so.tree_sees(parents, prefix + n)
    hit = see[:, sick]
    assert hit.any() and not hit.all()
    well_k, well_v = k.clone(), v.clone()
    well_k[0, sick], well_v[0, sick] = 0, 0
    kf, vf = _held(well_k[0], well_v[0], fmt)
    qf = f64(q)
    ok = ~hit
    assert_within(out[torch.tensor(ok)].cpu(), qf[ok], kf, vf, see[ok], so.attend(qf[ok], kf, vf, see[ok]), "unseen", fmt == "fp4")
    if bad == "nan":
        assert not np.isfinite(f64(out[torch.tensor(hit)].cpu())).any()
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 8), (4, 2, 64, 20), (8, 8, 128, 100), (16, 8, 64, 130)])
@pytest.mark.parametrize("prefix,back", [(30, None), (45, 1), (100, 3), (127, 40), (640, 30)])
def test_value_of_a_branch_not_finite(hq, hkv, d, n, prefix, back):
    """Only V is infinite, in one dim: that dim is infinite for the rows that see it (all of them, where it is a cached token's,
    `back` tokens before the tree), everything else is the oracle's."""
    k, v = kv_tokens(SEED, 0, 1, 0, prefix + n, hkv, d)
    sick = prefix + n // 3 if back is None else prefix - back
    well = v.clone()
    v[0, sick, :, 7] = float("inf")
    pool = _pool(hq, hkv, d)
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    parents = tree(n, 4)
    q = _queries([n], hq, d)
    out = pool.attn_tree([c], [n], [parents], 0, q.cuda()).cpu()
    see = so.tree_sees(parents, prefix + n)
    kf, vf, qf = f64(k[0]), f64(well[0]), f64(q)
    hit = torch.tensor(see[:, sick])
    assert (out[hit][:, :, 7] == float("inf")).all()
    ref = so.attend(qf, kf, vf, see)
    out[hit, :, 7] = torch.from_numpy(ref[see[:, sick]][:, :, 7]).to(torch.bfloat16)
    assert_within(out, qf, kf, vf, see, ref, "other dims")
    pool.close()


CROSS = {
    "single rows": [(1, 1), (16, 1), (50, 1), (1500, 1), (0, 1)],
    "hypotheses": [(700, 5), (64, 3), (65, 4), (1, 9), (0, 2), (333, 0)],
    "more rows than states": [(5, 40), (33, 100), (64, 64), (0, 70)],
    "texts": [(900, 300), (130, 500), (1, 129), (64, 65)],
    "long": [(9000, 3), (5000, 16)],
}


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("batch", list(CROSS))
def test_cross(batch, hq, hkv, d, fmt):
    sizes = CROSS[batch]
    lens, ns = [p for p, _ in sizes], [n for _, n in sizes]
    pool = _pool(hq, hkv, d, fmt)
    convs, kv = _fill(pool, lens, hkv, d)
    q = _queries(ns, hq, d)
    out = torch.full((sum(ns), hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pool.attn_cross(convs, ns, 0, q.cuda(), out)
    torch.cuda.synchronize()
    _check(out, q, ns, kv, [None] * len(ns), fmt, f"cross {batch}")
    r0 = 0
    for L, n in sizes:
        if L == 0:
            assert (out[r0:r0 + n] == 0).all(), "rows without states are zeros"
        r0 += n
    pool.close()


def test_cross_same_states_twice():
    """A conversation in several entries of a batch: every entry's rows, as alone."""
    hq, hkv, d = 16, 8, 128
    pool = _pool(hq, hkv, d)
    convs, kv = _fill(pool, [400, 90], hkv, d)
    ns = [2, 3, 1, 2]
    q = _queries(ns, hq, d)
    out = pool.attn_cross([convs[0], convs[1], convs[0], convs[0]], ns, 0, q.cuda())
    _check(out, q, ns, [kv[0], kv[1], kv[0], kv[0]], [None] * 4, "bf16", "same states")
    pool.close()


def test_chain_is_extend():
    """A chain sees what causal rows see."""
    hq, hkv, d = 32, 8, 128
    lens, ns = [500, 64, 2000], [7, 64, 130]
    pool = _pool(hq, hkv, d)
    convs, kv = _fill(pool, lens, hkv, d)
    q = _queries(ns, hq, d)
    a = pool.attn_tree(convs, ns, [tree(n, 0, "chain") for n in ns], 0, q.cuda())
    b = pool.attn_extend(convs, ns, 0, q.cuda())
    err = (a.float() - b.float()).norm() / b.float().norm()
    assert err < 2 * 2.0 ** -8, err   # both round weights to bf16, at other maxima
    pool.close()


# ---- append at tree positions --------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d,nl,ns", [(16, 8, 128, 4, [26]), (4, 2, 64, 1, [1, 0, 5, 17]), (32, 8, 128, 32, [64, 40, 33, 64]),
                                             (6, 3, 64, 2, [100, 300])])
@pytest.mark.parametrize("interleaved,rotary", [(False, 64), (True, 32)])
def test_append_at_tree_positions(hq, hkv, d, nl, ns, interleaved, rotary):
    from paper_2606_01839_amd import Rope
    before = [13 + 100 * i for i in range(len(ns))]
    pool = _pool(hq, hkv, d, nl=nl)
    convs, _ = _fill(pool, before, hkv, d, nl=nl)
    kv = [kv_tokens(SEED + 1, i, nl, 0, n, hkv, d) for i, n in enumerate(ns)]
    k, v = (torch.cat([x[j] for x in kv], 1).contiguous() for j in (0, 1))
    q = torch.stack([torch.cat([q_tokens(SEED, 9 * layer + i, layer, 0, n, hq, d) for i, n in enumerate(ns)]) for layer in range(nl)])
    parents = [tree(n, i) for i, n in enumerate(ns)]
    rope = Rope(rotary, base=10000.0, interleaved=interleaved)
    qin = q.cuda()
    qo = pool.kv_append_tree(convs, ns, parents, k.cuda(), v.cuda(), rope, q=qin)
    gk, gv = pool.kv_read(convs, before, ns)
    torch.cuda.synchronize()
    assert torch.equal(gv.cpu(), v) and torch.equal(qin.cpu(), q)
    pos = np.concatenate([b + so.depths(p) if p else np.zeros(0, dtype=np.int64) for b, p in zip(before, parents)])
    f, amp = orope.frequencies(rotary, 10000.0)
    for name, got, x in (("k", gk, k), ("q", qo, q)):
        ref = orope.rotate(f64(x), pos, f, amp, interleaved)
        tol = 2.0 ** -21 * 2 * np.abs(f64(x)).max() + half_ulp_bf16(ref)   # the header's bound and one rounding
        assert (np.abs(f64(got.cpu()) - ref) <= tol).all(), name
    assert [pool.conv_len(c) for c in convs] == [b + n for b, n in zip(before, ns)]
    pool.close()


@pytest.mark.parametrize("convs_n", [400, 600])
def test_append_of_many_trees(convs_n):
    """More page chunks than one upload holds (some 21,800); 600 trees of 1024 tokens have more rows than an upload has positions for, so
    their queries turn in the append's own launches."""
    from paper_2606_01839_amd import Rope
    n, d = 1024, 64
    pool = _pool(1, 1, d, n_pages=convs_n * 65, max_convs=convs_n, max_pages=66)
    convs = [pool.conv_create() for _ in range(convs_n)]
    one = torch.randn((1, convs_n, 1, d), device="cuda").to(torch.bfloat16)
    pool.kv_append_batch(convs, [1] * convs_n, one, one)   # trees begin in the middle of a page
    g = torch.Generator(device="cuda").manual_seed(5)
    k, q = (torch.randn((1, convs_n * n, 1, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    parents = [tree(n, i % 7) for i in range(convs_n)]
    depths = [so.depths(tree(n, i)) for i in range(7)]
    qo = pool.kv_append_tree(convs, [n] * convs_n, parents, k, k, Rope(d), q=q)
    f, amp = orope.frequencies(d, 10000.0)
    for i in (0, 1, convs_n // 2, 335, 336, convs_n - 1):
        rows = slice(i * n, (i + 1) * n)
        gk, gv = pool.kv_read([convs[i]], [1], [n])
        assert torch.equal(gv, k[:, rows])
        for got, x in ((gk, k[:, rows]), (qo[:, rows], q[:, rows])):
            xf = f64(x.cpu())
            ref = orope.rotate(xf, 1 + depths[i % 7], f, amp)
            tol = 2.0 ** -21 * 2 * np.abs(xf).max() + half_ulp_bf16(ref)
            assert (np.abs(f64(got.cpu()) - ref) <= tol).all(), i
    pool.close()


def test_chain_append_is_append_rope():
    """A chain's positions are its slots: the same bits as kv_append_rope, in place for the queries."""
    from paper_2606_01839_amd import Rope
    hq, hkv, d, nl, n = 16, 8, 128, 2, 37
    rope = Rope(128)
    k, v = kv_tokens(SEED, 0, nl, 0, n, hkv, d)
    q = torch.stack([q_tokens(SEED, 1, layer, 0, n, hq, d) for layer in range(nl)]).cuda()
    outs = []
    for fmt in ("bf16", "fp4"):
        pool = _pool(hq, hkv, d, fmt, nl=nl)
        a, b = pool.conv_create(), pool.conv_create()
        qa, qb = q.clone(), q.clone()
        pool.kv_append_tree([a], [n], [tree(n, 0, "chain")], k.cuda(), v.cuda(), rope, q=qa, q_out=qa)
        pool.kv_append_rope([b], [n], k.cuda(), v.cuda(), rope, q=qb, q_out=qb)
        ra, rb = pool.kv_read([a], [0], [n]), pool.kv_read([b], [0], [n])
        assert torch.equal(ra[0], rb[0]) and torch.equal(ra[1], rb[1]) and torch.equal(qa, qb)
        outs.append(qa)
        pool.close()
    assert torch.equal(*outs)


# ---- keep ----------------------------------------------------------------------------------------
KEEPS = [  # (tokens before, last, kept)
    (40, 8, [0, 2, 5]), (16, 16, [15]), (0, 5, [0, 1, 2, 3, 4]), (31, 40, []), (7, 3, [0, 1]), (100, 64, list(range(1, 64))),
    (48, 16, []), (20, 30, [3, 9, 10, 11, 12, 13, 14, 15, 16, 17, 18, 19, 20, 21, 28]), (5, 0, []), (12, 4, [2]),
]


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,nl", [(16, 8, 128, 2), (4, 2, 64, 3), (6, 3, 64, 1), (8, 1, 128, 1)])
def test_keep(hq, hkv, d, nl, fmt):
    """Bytes move as they are; slots behind the end are zeros; pages return; what is appended next is right."""
    pool = _pool(hq, hkv, d, fmt, nl=nl)
    lens = [b + n for b, n, _ in KEEPS]
    convs, kv = _fill(pool, lens, hkv, d, nl=nl)
    all_k, all_v = pool.kv_read(convs, [0] * len(lens), lens)
    pool.kv_keep(convs, [n for _, n, _ in KEEPS], [x for _, _, x in KEEPS])
    new = [b + len(x) for b, _, x in KEEPS]
    assert [pool.conv_len(c) for c in convs] == new
    pages = [len(pool.conv_pages(c)) for c in convs]
    assert pages == [(x + 15) // 16 for x in new] and pool.occupancy()[0] == sum(pages)
    k, v = pool.kv_read(convs, [0] * len(new), new)
    at, to = 0, 0
    for (before, n, kept), L, N in zip(KEEPS, lens, new):
        rows = torch.tensor(list(range(before)) + [before + i for i in kept], dtype=torch.int64, device="cuda") + at
        assert torch.equal(k[:, to:to + N], all_k[:, rows]) and torch.equal(v[:, to:to + N], all_v[:, rows]), (before, n, kept)
        at, to = at + L, to + N
    view = pool.kv_view()
    wire = [pool.kv_pack_fp4(c) if fmt == "fp4" else pool.kv_pack(c) for c in convs]
    for c, N, w in zip(convs, new, wire):   # pack zeroes what is behind the end: the pool has to hold the same
        ids = torch.tensor(pool.conv_pages(c), dtype=torch.int64, device="cuda")
        assert torch.equal(view[:, ids].contiguous().view(torch.uint8).reshape(-1), w.reshape(-1)), N
    more = [(3 * i) % 20 for i in range(len(new))]
    add = [kv_tokens(SEED + 5, i, nl, 0, n, hkv, d) for i, n in enumerate(more)]
    pool.kv_append_batch(convs, more, *(torch.cat([x[j] for x in add], 1).contiguous().cuda() for j in (0, 1)))
    k2, v2 = pool.kv_read(convs, [0] * len(new), new)
    assert torch.equal(k2, k) and torch.equal(v2, v)
    k3, _ = pool.kv_read(convs, new, more)
    want = torch.cat([x[0] for x in add], 1)
    if fmt == "bf16":
        assert torch.equal(k3.cpu(), want)
    pool.close()


def test_keep_many_and_nothing():
    """A whole batch cut to a page border needs no launch; thousands of moved tokens in one conversation."""
    hq, hkv, d = 4, 2, 64
    pool = _pool(hq, hkv, d, n_pages=600, max_pages=600)
    convs, _ = _fill(pool, [8000], hkv, d)
    k0, v0 = pool.kv_read(convs, [0], [8000])
    kept = list(range(1, 7000, 2))
    pool.kv_keep(convs, [7900], [kept])
    k, v = pool.kv_read(convs, [0], [100 + len(kept)])
    rows = torch.tensor(list(range(100)) + [100 + i for i in kept], device="cuda")
    assert torch.equal(k, k0[:, rows]) and torch.equal(v, v0[:, rows])
    n = pool.conv_len(convs[0])
    pool.kv_keep(convs, [n], [[]])
    assert pool.conv_len(convs[0]) == 0 and pool.occupancy()[0] == 0
    pool.kv_keep([], [], [])
    pool.close()


def test_failed_keep_changes_no_length():
    from paper_2606_01839_amd import ConserveError, CS_EHIP
    pool = _pool(4, 2, 64)
    convs, _ = _fill(pool, [50], 2, 64)
    used = pool.occupancy()
    pool.debug_fail_launches(0)
    with pytest.raises(ConserveError) as e:
        pool.kv_keep(convs, [20], [[3, 4]])
    pool.debug_fail_launches(-1)
    assert e.value.code == CS_EHIP and pool.conv_len(convs[0]) == 50 and pool.occupancy() == used
    pool.close()


# ---- a whole step --------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_draft_verify_keep(fmt):
    """Three rounds of a program: rotated drafts are appended, verified, an accepted path kept; then the cache holds what
    plain appends of the accepted tokens at their positions would have put there, bit for bit, and decode agrees."""
    from paper_2606_01839_amd import Rope
    hq, hkv, d, nl = 16, 8, 128, 2
    rope = Rope(128)
    pool, plain = (_pool(hq, hkv, d, fmt, nl=nl, seed=s) for s in (1, 2))
    lens = [37, 260]
    a, b = ([p.conv_create() for _ in lens] for p in (pool, plain))
    base = [kv_tokens(SEED, i, nl, 0, n, hkv, d) for i, n in enumerate(lens)]
    k, v = (torch.cat([x[j] for x in base], 1).contiguous().cuda() for j in (0, 1))
    pool.kv_append_rope(a, lens, k, v, rope)
    plain.kv_append_rope(b, lens, k, v, rope)
    for step in range(3):
        ns = [9 + step, 20]
        parents = [tree(n, 10 * step + i) for i, n in enumerate(ns)]
        draft = [kv_tokens(SEED + 2 + step, i, nl, 0, n, hkv, d) for i, n in enumerate(ns)]
        q = torch.stack([_queries(ns, hq, d)] * nl).cuda()
        k, v = (torch.cat([x[j] for x in draft], 1).contiguous().cuda() for j in (0, 1))
        qr = pool.kv_append_tree(a, ns, parents, k, v, rope, q=q)
        total = [pool.conv_len(c) for c in a]
        ck, cv = pool.kv_read(a, [0, 0], total)
        for layer in range(nl):
            out = pool.attn_tree(a, ns, parents, layer, qr[layer])
            r0 = t0 = 0
            for n, t, p in zip(ns, total, parents):
                kf, vf, qf = f64(ck[layer, t0:t0 + t].cpu()), f64(cv[layer, t0:t0 + t].cpu()), f64(qr[layer, r0:r0 + n].cpu())
                see = so.tree_sees(p, t)
                assert_within(out[r0:r0 + n].cpu(), qf, kf, vf, see, so.attend(qf, kf, vf, see), f"step {step} layer {layer}", fmt == "fp4")
                r0, t0 = r0 + n, t0 + t
        paths = []
        for p in parents:   # the deepest token's path
            j = int(np.argmax(so.depths(p)))
            path = []
            while j >= 0:
                path.append(j)
                j = p[j]
            paths.append(path[::-1])
        pool.kv_keep(a, ns, paths)
        rows = torch.tensor(paths[0] + [ns[0] + i for i in paths[1]], device="cuda")
        plain.kv_append_rope(b, [len(x) for x in paths], k[:, rows].contiguous(), v[:, rows].contiguous(), rope)
        got = pool.kv_read(a, [0, 0], [pool.conv_len(c) for c in a])
        want = plain.kv_read(b, [0, 0], [plain.conv_len(c) for c in b])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q1 = _queries([1, 1], hq, d).cuda()
    assert torch.equal(pool.attn_decode_batch(a, 0, q1), plain.attn_decode_batch(b, 0, q1))
    pool.close()
    plain.close()
