"""GPU: trees, cross attention and keeping under the calls that the documentation allows: captured and replayed, on several streams,
in batches whose entries take different kernels, in pools larger than 4 GiB, scores of any magnitude, more rows than a launch takes."""
import random

import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import seen as so
from tests.helpers import GAMMA_ACC, f64, half_ulp_bf16, kv_tokens, q_tokens
from tests.seen_helpers import assert_within, bound, tree

pytestmark = pytest.mark.gpu

SEED = 4711


def _pool(hq, hkv, d, fmt="bf16", nl=1, n_pages=2048, max_convs=64, max_pages=2048, seed=3):
    from paper_2606_01839_amd import KVPool
    return KVPool(nl, hq, hkv, d, n_pages=n_pages, max_convs=max_convs, max_pages_per_conv=max_pages, placement_seed=seed,
                  device="cuda", kv_format=fmt)


def _randn(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _fill(pool, lens, seed=SEED):
    convs = [pool.conv_create() for _ in lens]
    shape = (pool.n_layers, sum(lens), pool.n_kv_heads, pool.head_dim)
    pool.kv_append_batch(convs, lens, _randn(shape, seed), _randn(shape, seed + 1))
    return convs


def _compare(out, q, k, v, fmt, see, what):
    kf, vf, qf = f64(k.cpu()), f64(v.cpu()), f64(q.cpu())
    see = np.ones((q.shape[0], k.shape[0]), dtype=bool) if see is None else see
    assert_within(out.cpu(), qf, kf, vf, see, so.attend(qf, kf, vf, see), what, fmt == "fp4")


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_captured_and_replayed(fmt):
    """Two graphs of one pool (a tree whose words are too many for the launch's arguments, cross attention of few and of many rows), replayed
    in turn between eager calls of other batches, with new queries each time."""
    hq, hkv, d = 16, 8, 128
    pool = _pool(hq, hkv, d, fmt)
    lens = [700, 90, 3000, 260]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        convs = _fill(pool, lens)
    ns, rows = [70, 90, 20, 200], [1, 300, 3, 0]
    parents = [tree(n, i) for i, n in enumerate(ns)]
    calls = [(sum(ns), lambda q, o: pool.attn_tree(convs, ns, parents, 0, q, o)), (sum(rows), lambda q, o: pool.attn_cross(convs, rows, 0, q, o))]
    graphs = []
    for n, call in calls:
        q = torch.zeros(n, hq, d, dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            call(q, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call(q, out)
        graphs.append((graph, call, q, out))
    for turn in range(4):
        with torch.cuda.stream(s):
            for i in range(150):   # the upload ring goes round
                pool.attn_tree(convs[::-1], ns[::-1], parents[::-1], 0, _randn((sum(ns), hq, d), i))
        torch.cuda.synchronize()
        for graph, call, q, out in graphs[::1 if turn % 2 else -1]:
            x = _randn(q.shape, 100 + turn)
            q.copy_(x)
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                want = call(x, torch.empty_like(x))
            torch.cuda.synchronize()
            assert torch.equal(out, want), turn
    pool.close()


def test_keep_is_not_captured():
    from paper_2606_01839_amd import ConserveError, CS_ESTATE
    pool = _pool(4, 2, 64)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        convs = _fill(pool, [40])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    x = torch.zeros(4, device="cuda")
    codes = []
    with torch.cuda.graph(graph, stream=s):
        x.add_(1)
        for last, kept in ((8, [2, 3]), (8, [])):
            try:
                pool.kv_keep(convs, [last], [kept])
            except ConserveError as e:
                codes.append(e.code)
    assert codes == [CS_ESTATE] * 2 and pool.conv_len(convs[0]) == 40
    graph.replay()
    torch.cuda.synchronize()
    pool.kv_keep(convs, [8], [[2, 3]])
    assert pool.conv_len(convs[0]) == 34
    pool.close()


def test_streams():
    """A step whose calls are on different streams: the pool orders them."""
    from paper_2606_01839_amd import Rope
    hq, hkv, d = 16, 8, 128
    a, b = _pool(hq, hkv, d, seed=1), _pool(hq, hkv, d, seed=1)
    streams = [torch.cuda.Stream() for _ in range(3)]
    rope = Rope(d)
    outs = []
    for pool in (a, b):
        use = (lambda i: torch.cuda.stream(streams[i % 3])) if pool is a else (lambda i: torch.cuda.stream(torch.cuda.current_stream()))
        with use(0):
            convs = _fill(pool, [300, 31])
        got = []
        for step in range(6):
            ns = [12, 40]
            parents = [tree(n, step + i) for i, n in enumerate(ns)]
            k, v = (_randn((1, sum(ns), hkv, d), 10 * step + i) for i in (1, 2))
            q = _randn((1, sum(ns), hq, d), 10 * step + 3)
            torch.cuda.synchronize()
            with use(step):
                pool.kv_append_tree(convs, ns, parents, k, v, rope, q=q, q_out=q)
            with use(step + 1):
                if pool is a:
                    torch.cuda.current_stream().wait_stream(streams[step % 3])   # q is the caller's
                out = pool.attn_tree(convs, ns, parents, 0, q[0])
            with use(step + 2):
                pool.kv_keep(convs, ns, [[1, 3], [0, 5, 39]])
            torch.cuda.synchronize()
            got.append(out)
        with use(1):
            got += pool.kv_read(convs, [0, 0], [pool.conv_len(c) for c in convs])
        torch.cuda.synchronize()
        outs.append(got)
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    a.close()
    b.close()


@pytest.mark.parametrize("seed", range(8))
def test_random_batches(seed):
    """Batches whose entries take different kernels, with empty ones, one item and many, against the oracle."""
    r = random.Random(seed)
    hq, hkv, d = r.choice([(32, 8, 128), (4, 2, 64), (8, 8, 128), (16, 2, 64), (12, 3, 128), (2, 2, 64)])
    fmt = r.choice(["bf16", "fp4"])
    lens = [r.choice([0, 1, 17, 64, 300, 900, 2500]) + r.randrange(40) for _ in range(r.randint(1, 7))]
    pool = _pool(hq, hkv, d, fmt, seed=seed)
    convs = _fill(pool, lens, seed)
    k, v = pool.kv_read(convs, [0] * len(lens), lens)
    ks, vs = k[0].split(lens), v[0].split(lens)
    ns = [min(n, r.choice([0, 1, 3, 8, 30, 80, 150])) for n in lens]
    parents = [tree(n, r.randrange(1000), r.choice(["mixed", "mixed", "chain", "star"])) for n in ns]
    q = _randn((sum(ns), hq, d), seed + 50)
    out = pool.attn_tree(convs, ns, parents, 0, q)
    for i, (o, x) in enumerate(zip(out.split(ns), q.split(ns))):
        if ns[i]:
            _compare(o, x, ks[i], vs[i], fmt, so.tree_sees(parents[i], lens[i]), f"tree {i}: {lens} {ns}")
    pick = [r.randrange(len(lens)) for _ in range(r.randint(1, 9))]
    rows = [r.choice([0, 1, 2, 7, 40, 200]) for _ in pick]
    q = _randn((sum(rows), hq, d), seed + 51)
    out = pool.attn_cross([convs[i] for i in pick], rows, 0, q)
    for i, n, o, x in zip(pick, rows, out.split(rows), q.split(rows)):
        if n and lens[i]:
            _compare(o, x, ks[i], vs[i], fmt, None, f"cross {i}: {lens} {pick} {rows}")
        elif n:
            assert (o == 0).all()
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_pool_over_4_gib(fmt):
    """Page offsets past 2^32 bytes: three layers of a pool of several GiB with scattered pages, the last layer attended."""
    hq, hkv, d, nl = 16, 8, 128, 3
    n_pages = 40000 if fmt == "bf16" else 120000
    pool = _pool(hq, hkv, d, fmt, nl=nl, n_pages=n_pages)
    assert pool.kv.numel() > 1.4 * 2 ** 32
    lens, ns = [900, 130], [9, 80]
    convs = _fill(pool, lens)
    parents = [tree(n, i) for i, n in enumerate(ns)]
    q = _randn((sum(ns), hq, d), 5)
    out = pool.attn_tree(convs, ns, parents, nl - 1, q)
    k, v = pool.kv_read(convs, [0, 0], lens)
    for i in (0, 1):
        _compare(out.split(ns)[i], q.split(ns)[i], k[nl - 1].split(lens)[i], v[nl - 1].split(lens)[i], fmt, so.tree_sees(parents[i], lens[i]), f"{i}")
    pool.kv_keep(convs, ns, [[1, 8], [3, 7, 70]])
    k2, v2 = pool.kv_read(convs, [0, 0], [893, 53])
    rows = torch.tensor(list(range(891)) + [892, 899] + [900 + i for i in list(range(50)) + [53, 57, 120]], device="cuda")
    assert torch.equal(k2, k[:, rows]) and torch.equal(v2, v[:, rows])
    pool.close()


def test_more_rows_than_an_entry_of_a_launch():
    """70,000 rows on one set of states and some rows on others, against the same rows in small calls."""
    hq, hkv, d = 2, 2, 64
    pool = _pool(hq, hkv, d)
    convs = _fill(pool, [130, 40])
    rows = [3, 70000, 5]
    q = _randn((sum(rows), hq, d), 1)
    pick = [convs[1], convs[0], convs[1]]
    out = pool.attn_cross(pick, rows, 0, q)
    k, v = pool.kv_read(convs, [0, 0], [130, 40])
    ks, vs = k[0].split([130, 40]), v[0].split([130, 40])
    for r0, n, i in ((0, 3, 1), (3, 100, 0), (3 + 32700, 200, 0), (3 + 65500, 100, 0), (70003 - 50, 50, 0), (70003, 5, 1)):
        _compare(out[r0:r0 + n], q[r0:r0 + n], ks[i], vs[i], "bf16", None, f"rows {r0}")
    pool.close()


POWERS = [0, 12, 20, 23, 24, 27, 31, 33, 60, 100]


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,n,L", [(4, 2, 64, 10, 700), (8, 8, 128, 10, 3000), (8, 2, 128, 40, 500), (16, 2, 64, 10, 1500)])
def test_far_scores(fmt, hq, hkv, d, n, L):
    """Keys +-1, queries +-2^p: scores are exact in fp32, and from 2^12 on the softmax is the mean over the keys of the largest
    score, up to the output's rounding and the fp32 sums (as in test_gpu_far_scores)."""
    r = np.random.default_rng(7)
    k, v = r.choice([-1.0, 1.0], (L, hkv, d)), r.standard_normal((L, hkv, d))
    power = np.array([POWERS[i % len(POWERS)] for i in range(n)])
    q = r.choice([-1.0, 1.0], (n, hq, d)) * 2.0 ** power[:, None, None]
    k, v, q = (torch.from_numpy(x).to(torch.bfloat16) for x in (k, v, q))
    pool = _pool(hq, hkv, d, fmt)
    c = pool.conv_create()
    pool.kv_append(c, k[None].cuda(), v[None].cuda())
    hk, hv = o4.held(f64(k), f64(v)) if fmt == "fp4" else (f64(k), f64(v))
    parents = tree(n, 3)
    for what, see, out in (("tree", so.tree_sees(parents, L), pool.attn_tree([c], [n], [parents], 0, q.cuda())),
                           ("cross", np.ones((n, L), dtype=bool), pool.attn_cross([c], [n], 0, q.cuda()))):
        ref, g = so.attend(f64(q), hk, hv, see), f64(out.cpu())
        tol = half_ulp_bf16(np.maximum(np.abs(ref), np.abs(g))) + GAMMA_ACC * np.abs(hv).max()
        near = power == 0
        tol[near] += bound(f64(q)[near], hk, hv, see[near], ref[near])
        assert np.isfinite(g).all() and (np.abs(g - ref) <= tol).all(), (what, np.argwhere(~(np.abs(g - ref) <= tol))[:5], power)
    pool.close()


def test_outputs_of_other_rows_stay():
    """Rows of the output behind the batch's last are not written."""
    hq, hkv, d = 32, 8, 128
    pool = _pool(hq, hkv, d)
    convs = _fill(pool, [200, 700])
    for ns in ([3, 5], [40, 70]):
        n = sum(ns)
        whole = torch.full((n + 64, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        q = _randn((n, hq, d), 1)
        pool.attn_tree(convs, ns, [tree(x, 1) for x in ns], 0, q, whole[:n])
        pool.attn_cross(convs, ns, 0, q, whole[:n])
        assert (whole[n:] == 7).all() and torch.isfinite(whole).all()
    pool.close()


def test_failed_launches_report():
    """A launch that fails, of either kernel and of the merges, is CS_EHIP; the next call is right."""
    from paper_2606_01839_amd import ConserveError, CS_EHIP
    hq, hkv, d = 32, 8, 128
    pool = _pool(hq, hkv, d)
    convs = _fill(pool, [5000])
    for n, launches in ((4, 2), (40, 2)):
        q, parents = _randn((n, hq, d), n), [tree(n, 2)]
        want = pool.attn_tree(convs, [n], parents, 0, q)
        for after in range(launches):
            pool.debug_fail_launches(after)
            with pytest.raises(ConserveError) as e:
                pool.attn_tree(convs, [n], parents, 0, q)
            assert e.value.code == CS_EHIP
            pool.debug_fail_launches(-1)
        assert torch.equal(pool.attn_tree(convs, [n], parents, 0, q), want)
    used = pool.occupancy()
    from paper_2606_01839_amd import Rope
    pool.debug_fail_launches(0)
    with pytest.raises(ConserveError) as e:
        k = _randn((1, 30, hkv, d), 1)
        pool.kv_append_tree(convs, [30], [tree(30, 1)], k, k, Rope(d))
    pool.debug_fail_launches(-1)
    assert e.value.code == CS_EHIP and pool.conv_len(convs[0]) == 5000 and pool.occupancy() == used
    pool.close()
