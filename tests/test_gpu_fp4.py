"""GPU: the 4-bit KV cache. What it holds is exact (bit for bit the oracle's codes, powers and wire);
attention over it is compared with the oracle's attention of the held values, with the tolerances of the
bf16 cache: the kernels' arithmetic behind the conversion is the same (helpers.arith_bound)."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle.attention import attend_last, attend_rows, weights
from tests.helpers import arith_bound, assert_close, assert_within_arith_bound, f64, half_ulp_bf16, kv_tokens, q_tokens

pytestmark = pytest.mark.gpu

SEED = 606
SHAPES = [(4, 2, 64), (8, 8, 64), (16, 2, 64), (6, 3, 128), (32, 8, 128), (8, 8, 128), (8, 1, 128)]


def _pool(nl, hq, hkv, d, n_pages, seed=1, fmt="fp4", max_convs=8, max_pages=512):
    from paper_2606_01839_amd import KVPool
    return KVPool(nl, hq, hkv, d, n_pages=n_pages, max_convs=max_convs, max_pages_per_conv=max_pages, placement_seed=seed,
                  device="cuda", kv_format=fmt)


def _held(k, v):
    return o4.held(f64(k), f64(v))


def _read(pool, conv, start, n):
    k, v = pool.kv_read([conv], [start], [n])
    torch.cuda.synchronize()
    return f64(k), f64(v)


def _fill(pool, nl, lens, hkv, d, scale=None):
    """One conversation per length, appended in one batch; ([handle], [(K, V) bf16 on the CPU])."""
    kv = [kv_tokens(SEED, i, nl, 0, n, hkv, d, scale, scale) for i, n in enumerate(lens)]
    convs = [pool.conv_create() for _ in lens]
    pool.kv_append_batch(convs, lens, *(torch.cat([x[j] for x in kv], 1).contiguous().cuda() for j in (0, 1)))
    return convs, kv


# ---- what the cache holds ------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128), (6, 3, 128)])
@pytest.mark.parametrize("dirty", [False, True])
def test_appends_hold_the_oracles_values(hq, hkv, d, dirty):
    """Ragged appends across page boundaries, also into memory that held NaN scales and codes before."""
    nl = 2
    pool = _pool(nl, hq, hkv, d, 64)
    if dirty:
        pool.kv.fill_(0xFF)
    c = pool.conv_create()
    ks, vs, pos = [], [], 0
    for n in [1, 1, 13, 1, 16, 17, 2, 1, 0, 31, 64, 3, 100]:
        k, v = kv_tokens(SEED, 0, nl, pos, n, hkv, d)
        pool.kv_append(c, k.cuda(), v.cuda())
        ks.append(k)
        vs.append(v)
        pos += n
    k, v = torch.cat(ks, 1), torch.cat(vs, 1)
    wk, wv = _held(k, v)
    gk, gv = _read(pool, c, 0, pos)
    assert np.array_equal(gk, wk) and np.array_equal(gv, wv)
    for start, n in [(0, 1), (15, 2), (16, 16), (17, 100), (pos - 1, 1), (pos, 0), (33, 0)]:
        gk, gv = _read(pool, c, start, n)
        assert np.array_equal(gk, wk[:, start:start + n]) and np.array_equal(gv, wv[:, start:start + n])
    wire = pool.kv_pack(c)
    torch.cuda.synchronize()
    assert np.array_equal(wire.cpu().numpy(), o4.serialize(f64(k), f64(v)))
    assert torch.equal(wire, pool.kv_pack_fp4(c))
    pool.close()


@pytest.mark.parametrize("d", [64, 128])
def test_hard_values(d):
    """Ties, saturation, powers of two on both sides of a step, zero groups, the least and largest
    magnitudes; a value of a group of its own size beside far larger ones."""
    n, hkv = 40, 2
    r = np.random.default_rng(3)
    x = r.standard_normal((2, 1, n, hkv, d))
    x[:, :, 0] = 0
    x[:, :, 1] = r.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7.96875, -0.25, -2.5, -5, 0], (2, 1, hkv, d)) * 2.0 ** -9
    x[:, :, 2] = 1.0
    x[:, :, 3] = 1.9921875
    x[:, :, 4] *= 1e30
    x[:, :, 5] *= 1e-30
    x[:, :, 6] *= 2.0 ** -127
    x[:, :, 7] = 0
    x[:, :, 7, :, ::7] = 2.0 ** -133
    x[:, :, 8, :, 5] = 3e38
    x[:, :, 9, :, ::3] = -0.0
    x[:, :, 10, :, :32] *= 1000
    k, v = (torch.from_numpy(t).to(torch.bfloat16) for t in x)
    wk, wv = _held(k, v)
    pools = [_pool(1, 4, hkv, d, 8, fmt=f) for f in ("fp4", "bf16")]
    convs = [p.conv_create() for p in pools]
    for p, c in zip(pools, convs):
        p.kv_append(c, k.cuda(), v.cuda())
    gk, gv = _read(pools[0], convs[0], 0, n)
    # below bf16's least normal the read-back is as bf16 holds it
    tiny = 2.0 ** -126
    for g, w in ((gk, wk), (gv, wv)):
        big = np.abs(w) >= tiny
        assert np.array_equal(g[big | (w == 0)], w[big | (w == 0)])
        assert (np.abs(g - w)[~big] <= tiny * 2.0 ** -8).all()
    wire = o4.serialize(f64(k), f64(v))
    for p, c in zip(pools, convs):   # packed from either kind of pool
        got = p.kv_pack_fp4(c).cpu().numpy()
        torch.cuda.synchronize()
        same = got == wire
        # the sign of a zero is free
        lo, hi = (got & 7) == 0, (got & 0x70) == 0
        assert (same | (lo & ((got & 0xF0) == (wire & 0xF0))) | (hi & ((got & 0xF) == (wire & 0xF))) | (lo & hi)).all()
        p.close()


@pytest.mark.parametrize("d", [64, 128])
def test_a_group_with_an_infinity_or_nan_reads_back_as_nan(d):
    pool = _pool(1, 4, 2, d, 8)
    k, v = kv_tokens(SEED, 0, 1, 0, 20, 2, d)
    k[0, 3, 1, 40] = float("inf")
    v[0, 18, 0, 5] = float("nan")
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    gk, gv = _read(pool, c, 0, 20)
    bad_k, bad_v = np.zeros(gk.shape, bool), np.zeros(gv.shape, bool)
    bad_k[0, 3, 1, 32:64] = True
    bad_v[0, 18, 0] = True
    assert np.array_equal(np.isnan(gk), bad_k) and np.array_equal(np.isnan(gv), bad_v)
    # head 0 of K and tokens 0 .. 17 are as without it: queries of them see none of it
    q = q_tokens(SEED, 0, 0, 17, 1, 4, d)
    short = _pool(1, 4, 2, d, 8)
    s = short.conv_create()
    short.kv_append(s, k[:, :18].contiguous().cuda(), v[:, :18].contiguous().cuda())
    out = short.attn_decode_batch([s], 0, q.cuda())
    torch.cuda.synchronize()
    assert torch.isfinite(out[0, :2]).all() and not torch.isfinite(out[0, 2:]).any()
    pool.close()
    short.close()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (6, 3, 128), (32, 8, 128)])
def test_transfer_round_trips(hq, hkv, d):
    """bf16 prefiller -> 4-bit wire -> 4-bit decoder, and between 4-bit pools; then it continues."""
    nl = 2
    pre, a, b = _pool(nl, hq, hkv, d, 64, 3, "bf16"), _pool(nl, hq, hkv, d, 64, 5), _pool(nl, hq, hkv, d, 64, 7)
    for n in [1, 15, 16, 17, 250]:
        k, v = kv_tokens(SEED, n, nl, 0, n + 5, hkv, d)
        c = pre.conv_create()
        pre.kv_append(c, k[:, :n].contiguous().cuda(), v[:, :n].contiguous().cuda())
        wire = pre.kv_pack_fp4(c)
        assert wire.numel() == nl * ((n + 15) // 16) * hkv * 17 * d == pre.kv_pack_fp4_size(c)
        ca = a.kv_unpack(wire, n)
        cb = b.kv_unpack(a.kv_pack(ca), n)
        wk, wv = _held(k, v)
        want = o4.serialize(f64(k[:, :n]), f64(v[:, :n]))
        torch.cuda.synchronize()
        assert np.array_equal(wire.cpu().numpy(), want) and np.array_equal(b.kv_pack(cb).cpu().numpy(), want)
        b.kv_append(cb, k[:, n:].contiguous().cuda(), v[:, n:].contiguous().cuda())
        gk, gv = _read(b, cb, 0, n + 5)
        assert np.array_equal(gk, wk) and np.array_equal(gv, wv)
        rk, rv = pre.kv_read([c], [0], [n])
        torch.cuda.synchronize()
        assert torch.equal(rk.cpu(), k[:, :n]) and torch.equal(rv.cpu(), v[:, :n])   # a bf16 pool: the bits
        for p, x in ((pre, c), (a, ca), (b, cb)):
            p.conv_destroy(x)
    for p in (pre, a, b):
        assert p.occupancy() == (0, 64)
        p.close()


def test_unpack_zeroes_slots_past_the_end():
    """A wire whose tail slots hold rubbish: the pool's are zeros, and the next tokens go over them."""
    nl, hkv, d, n = 1, 2, 128, 21
    pool = _pool(nl, 4, hkv, d, 8)
    k, v = kv_tokens(SEED, 0, nl, 0, n, hkv, d)
    want = o4.serialize(f64(k), f64(v))
    wire = want.reshape(nl, 2, hkv, 17 * d).copy()
    full = o4.serialize(f64(torch.cat([k, k], 1)[:, :32]), f64(torch.cat([v, v], 1)[:, :32])).reshape(nl, 2, hkv, 17 * d)
    wire[:, 1] = full[:, 1]
    wire[:, 1, :, 16 * d + d // 2 + 16:] = 0xAB
    c = pool.kv_unpack(torch.from_numpy(wire.reshape(-1)).cuda(), n)
    got = pool.kv_view().cpu().numpy()[:, pool.conv_pages(c)].reshape(-1)
    torch.cuda.synchronize()
    assert np.array_equal(got, want)
    pool.close()


def test_batched_reads_and_large_ones():
    """Several conversations in one read; more chunks than one upload of the ring holds."""
    nl, hq, hkv, d = 1, 2, 1, 64
    for fmt in ("fp4", "bf16"):
        n = 16 * 70000
        pool = _pool(nl, hq, hkv, d, 70100, fmt=fmt, max_pages=70050)
        lens = [37, n, 5]
        convs = [pool.conv_create() for _ in lens]
        g = torch.Generator(device="cuda").manual_seed(1)
        k, v = (torch.randn((1, sum(lens), 1, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        pool.kv_append_batch(convs, lens, k, v)
        gk, gv = pool.kv_read(convs, [30, 0, 1], [7, n, 4])
        rows = torch.cat([torch.arange(30, 37), torch.arange(37, 37 + n), torch.arange(38 + n, 42 + n)]).cuda()
        if fmt == "bf16":
            assert torch.equal(gk, k[:, rows]) and torch.equal(gv, v[:, rows])
        else:
            at = torch.cat([torch.arange(50), torch.arange(n - 50, n + 11)])
            wk, wv = _held(k[:, rows][:, at].cpu(), v[:, rows][:, at].cpu())
            assert np.array_equal(f64(gk[:, at].cpu()), wk) and np.array_equal(f64(gv[:, at].cpu()), wv)
        torch.cuda.synchronize()
        pool.close()


# ---- attention over it -----------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_decode(hq, hkv, d):
    """Lengths around pages, page pairs and splits, alone and together; one-item and merged batches."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 255, 256, 257, 700, 1024, 1025, 3000]
    pool = _pool(1, hq, hkv, d, 600, max_convs=16)
    convs, kv = _fill(pool, 1, lens, hkv, d)
    q = torch.cat([q_tokens(SEED, i, 0, n - 1, 1, hq, d) for i, n in enumerate(lens)])
    refs = [attend_last(f64(q[i:i + 1]), *[x[0] for x in _held(*kv[i])]) for i in range(len(lens))]
    for idx in (list(range(len(lens))), [14], [0], [5, 3, 13], [2, 1]):
        sel, qq = [convs[i] for i in idx], q[idx].contiguous().cuda()
        out = pool.attn_decode_batch(sel, 0, qq)
        again = pool.attn_decode_batch_noalloc(sel, 0, qq, torch.full_like(out, float("nan")))
        torch.cuda.synchronize()
        assert torch.equal(out, again)
        for r, i in enumerate(idx):
            assert_close(out[r:r + 1], refs[i], f"decode of {lens[i]} in {idx}")
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,lens", [
    (32, 8, 128, [40003]),                                                  # longer items in one round of the CUs
    (32, 8, 64, [1000 + 37 * i * i for i in range(15)]),                    # ragged ones
    (32, 8, 128, [300 + 27 * i for i in range(64)]),                        # two rounds, a single item each
    (64, 8, 128, [9000 - 7 * i for i in range(9)]),
])
def test_decode_in_whole_rounds(hq, hkv, d, lens):
    """Batches whose items the plan of 4-bit pools makes longer: alone on the workspace and on the static records,
    and a part of the batch, whose plan is another."""
    pool = _pool(1, hq, hkv, d, sum(lens) // 16 + 80, max_convs=len(lens), max_pages=max(lens) // 16 + 2)
    convs, kv = _fill(pool, 1, lens, hkv, d)
    q = torch.cat([q_tokens(SEED, i, 0, n - 1, 1, hq, d) for i, n in enumerate(lens)])
    out = pool.attn_decode_batch(convs, 0, q.cuda())
    again = pool.attn_decode_batch_noalloc(convs, 0, q.cuda(), torch.full_like(out, float("nan")))
    part = sorted({0, 1, len(lens) // 2, len(lens) - 1} & set(range(len(lens))))
    alone = pool.attn_decode_batch([convs[i] for i in part], 0, q[part].contiguous().cuda())
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    for r, i in enumerate(part):
        ref = attend_last(f64(q[i:i + 1]), *[x[0] for x in _held(*kv[i])])
        assert_close(out[i:i + 1], ref, f"decode of {lens[i]} in the batch")
        assert_close(alone[r:r + 1], ref, f"decode of {lens[i]}")
    pool.close()


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_extend_and_prefill(hq, hkv, d):
    """Chunks of 0 .. all tokens in one launch, whole tiles and pieces, padding rows of a query tile."""
    lens, new = [1, 40, 130, 700, 64, 65, 2500, 9], [1, 40, 1, 129, 64, 3, 33, 0]
    pool = _pool(1, hq, hkv, d, 600)
    convs, kv = _fill(pool, 1, lens, hkv, d)
    q = [q_tokens(SEED, i, 0, n - m, m, hq, d) for i, (n, m) in enumerate(zip(lens, new))]
    refs = [attend_last(f64(q[i]), *[x[0] for x in _held(*kv[i])]) for i in range(len(lens))]
    for idx in (list(range(8)), [6], [3, 0], [1]):
        out = pool.attn_extend([convs[i] for i in idx], [new[i] for i in idx], 0, torch.cat([q[i] for i in idx]).cuda())
        torch.cuda.synchronize()
        row = 0
        for i in idx:
            if new[i]:
                assert_close(out[row:row + new[i]], refs[i], f"extend of {new[i]} on {lens[i]} in {idx}")
            row += new[i]
    idx = [1, 0, 4]
    out = pool.attn_prefill_turn1([convs[i] for i in idx], [lens[i] for i in idx], 0, torch.cat([q[i] for i in idx]).cuda())
    torch.cuda.synchronize()
    assert_close(out[:40], refs[1], "prefill")
    pool.close()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128)])
def test_long_prefill_and_many_tiles(hq, hkv, d):
    """A launch of more than two rounds of tiles at both head dims (at 64: two workgroups a CU)."""
    n = 6500 if d == 64 else 2600
    lens = [n, 333, n - 100]
    pool = _pool(1, hq, hkv, d, 1400)
    convs, kv = _fill(pool, 1, lens, hkv, d)
    q = [q_tokens(SEED, i, 0, 0, m, hq, d) for i, m in enumerate(lens)]
    out = pool.attn_prefill_turn1(convs, lens, 0, torch.cat(q).cuda())
    torch.cuda.synchronize()
    row = 0
    for i, m in enumerate(lens):
        rows = np.unique(np.r_[0:70, m // 2:m // 2 + 40, m - 70:m])
        hk, hv = (x[0] for x in _held(*kv[i]))
        assert_close(out[row + torch.from_numpy(rows)], attend_rows(f64(q[i][rows]), rows, hk, hv), f"prefill {m}")
        row += m
    pool.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("profile", ["peaked", "big_v", "mixed_scales", "zero_q"])
def test_hard_attention_within_the_arithmetic_bound(d, profile):
    """Peaked weights, outputs far over 1, V powers that differ by 2^60 between tokens, even weights."""
    hq, hkv, L, n = 8, 2, 300, 40
    r = np.random.default_rng(5)
    k, v, q = r.standard_normal((L, hkv, d)), r.standard_normal((L, hkv, d)), r.standard_normal((n, hq, d))
    if profile == "peaked":
        q *= 12
    if profile == "big_v":
        v *= 64
    if profile == "mixed_scales":
        v *= 2.0 ** r.integers(-50, 10, (L, 1, 1))
    if profile == "zero_q":
        q[:] = 0
    k, v, q = (torch.from_numpy(x).to(torch.bfloat16) for x in (k, v, q))
    pool = _pool(1, hq, hkv, d, 32)
    c = pool.conv_create()
    pool.kv_append(c, k[None].cuda(), v[None].cuda())
    hk, hv = o4.held(f64(k), f64(v))
    ext = pool.attn_extend([c], [n], 0, q.cuda())
    dec = pool.attn_decode_batch([c], 0, q[-1:].contiguous().cuda())
    torch.cuda.synchronize()
    ref = attend_last(f64(q), hk, hv)
    assert_within_arith_bound(ext, f64(q), np.arange(L - n, L), hk, hv, ref, f"extend {profile}")
    assert_within_arith_bound(dec, f64(q[-1:]), [L - 1], hk, hv, ref[-1:], f"decode {profile}")
    pool.close()


@pytest.mark.parametrize("d", [64, 128])
def test_queries_with_outliers(d):
    """One dim of a query far larger than the other 31 of its block, which the score product then holds to
    2^-16 of it (down to 2^-8 of it exactly): the arithmetic bound, and what that does to the weights."""
    hq, hkv, L, n = 4, 2, 200, 8
    r = np.random.default_rng(8)
    k, v, q = r.standard_normal((L, hkv, d)), r.standard_normal((L, hkv, d)), r.standard_normal((n, hq, d))
    k[:, :, 3] *= 2.0 ** -9
    q[:, :, 3] = 700.0 * np.sign(q[:, :, 3])
    k, v, q = (torch.from_numpy(x).to(torch.bfloat16) for x in (k, v, q))
    pool = _pool(1, hq, hkv, d, 32)
    c = pool.conv_create()
    pool.kv_append(c, k[None].cuda(), v[None].cuda())
    hk, hv = o4.held(f64(k), f64(v))
    ext = pool.attn_extend([c], [n], 0, q.cuda())
    dec = pool.attn_decode_batch([c], 0, q[-1:].contiguous().cuda())
    torch.cuda.synchronize()
    qf = f64(q)
    ref = attend_last(qf, hk, hv)
    pos = np.arange(L - n, L)
    tol = arith_bound(qf, pos, hk, hv, ref) + half_ulp_bf16(ref)
    for h in range(hq):
        g = h // (hq // hkv)
        top = np.abs(qf[:, h].reshape(n, d // 32, 32)).max(-1)
        moved = 2.0 ** -16 / np.sqrt(d) * np.einsum("rb,jb->rj", top, np.abs(hk[:, g].reshape(L, d // 32, 32)).sum(-1)).max(-1)
        w = weights(qf[:, h], pos, hk[:, g])
        mad = np.einsum("rj,rjd->rd", w, np.abs(hv[None, :w.shape[1], g] - ref[:, h][:, None]))
        tol[:, h] += np.expm1(2 * moved)[:, None] * mad
    assert (np.abs(f64(ext) - ref) <= tol).all()
    assert (np.abs(f64(dec) - ref[-1:]) <= tol[-1:]).all()
    pool.close()


@pytest.mark.parametrize("d", [64, 128])
def test_a_query_that_is_not_finite_spoils_its_own_rows_only(d):
    hq, hkv, lens, new = 8, 2, [70, 300, 33], [5, 40, 1]
    pool = _pool(1, hq, hkv, d, 64)
    convs, kv = _fill(pool, 1, lens, hkv, d)
    q = [q_tokens(SEED, i, 0, n - m, m, hq, d) for i, (n, m) in enumerate(zip(lens, new))]
    ref = np.concatenate([attend_last(f64(x), *[y[0] for y in _held(*kv[i])]) for i, x in enumerate(q)])
    q = torch.cat(q)
    q[2, 3, 40], q[20, 7, 0] = float("nan"), float("inf")
    ext = pool.attn_extend(convs, new, 0, q.cuda())
    last = [4, 44, 45]     # the conversations' last rows
    qd = q[last].clone()
    qd[1, 4, 10] = float("-inf")
    dec = pool.attn_decode_batch(convs, 0, qd.contiguous().cuda())
    torch.cuda.synchronize()
    # (The other rows of a wave keep their tolerance, not their bits: a row that is not finite has the wave refresh its
    # running maxima in every tile, so their weights are rounded against other maxima.)
    for got, want, where in ((ext, ref, [(2, 3), (20, 7)]), (dec, ref[last], [(1, 4)])):
        spoilt = np.zeros(want.shape[:2], dtype=bool)
        for i in where:
            spoilt[i] = True
        assert np.isnan(f64(got.cpu())[spoilt]).all()
        assert_close(got.cpu()[torch.from_numpy(~spoilt)], want[~spoilt])
    pool.close()


def test_nothing_past_the_end_leaks():
    """The whole pool holds NaN scales before the appends: slots past a conversation's end, and pages
    that belong to nobody, reach no output."""
    for d in (64, 128):
        lens = [1, 17, 33, 300, 1100]
        pool = _pool(1, 8, 2, d, 200)
        pool.kv.fill_(0xFF)
        convs, kv = _fill(pool, 1, lens, 2, d)
        q = torch.cat([q_tokens(SEED, i, 0, n - 1, 1, 8, d) for i, n in enumerate(lens)])
        outs = [pool.attn_decode_batch(convs, 0, q.cuda()), pool.attn_extend(convs, [1] * 5, 0, q.cuda())]
        torch.cuda.synchronize()
        for i, n in enumerate(lens):
            ref = attend_last(f64(q[i:i + 1]), *[x[0] for x in _held(*kv[i])])
            for out in outs:
                assert_close(out[i:i + 1], ref, f"{n}")
        pool.close()


def test_results_do_not_depend_on_placement_or_order():
    lens = [500, 33, 2100]
    outs = []
    for seed, order in ((1, [0, 1, 2]), (9, [0, 1, 2]), (4, [2, 0, 1])):
        pool = _pool(1, 32, 8, 128, 256, seed)
        convs, _ = _fill(pool, 1, lens, 8, 128)
        q = torch.cat([q_tokens(SEED, i, 0, n - 1, 1, 32, 128) for i, n in enumerate(lens)])[order].contiguous().cuda()
        o = pool.attn_decode_batch([convs[i] for i in order], 0, q)
        torch.cuda.synchronize()
        outs.append({i: o[r].clone() for r, i in enumerate(order)})
        pool.close()
    for other in outs[1:]:
        assert all(torch.equal(outs[0][i], other[i]) for i in range(3))


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128), (8, 1, 128)])
@pytest.mark.parametrize("ordered", [False, True])
def test_mixed_step_equals_separate_calls(hq, hkv, d, ordered):
    """Steps of extend chunks and decodes, all layers; bit for bit the separate calls' outputs where neither
    cuts its keys another way, and the oracle's."""
    nl = 3
    lens, new = [300, 1, 1500, 64, 900], [40, 1, 1, 130, 1]
    ext, dec = [0, 3], [1, 2, 4]
    pool = _pool(nl, hq, hkv, d, 400)
    kv = [kv_tokens(SEED, i, nl, 0, n + m, hkv, d) for i, (n, m) in enumerate(zip(lens, new))]
    convs = [pool.conv_create() for _ in lens]
    pool.kv_append_batch(convs, lens, *(torch.cat([x[j][:, :n] for x, n in zip(kv, lens)], 1).contiguous().cuda() for j in (0, 1)))
    k, v = (torch.cat([kv[i][j][:, lens[i]:] for i in ext + dec], 1).contiguous().cuda() for j in (0, 1))
    q = {i: torch.stack([q_tokens(SEED, i, l, lens[i], new[i], hq, d) for l in range(nl)]) for i in range(5)}
    qe, qd = (torch.cat([q[i] for i in g], 1).contiguous().cuda() for g in (ext, dec))
    oe, od = pool.mixed_step([convs[i] for i in ext], [new[i] for i in ext], [convs[i] for i in dec], k, v, qe, qd,
                             layer_ordered=ordered)
    torch.cuda.synchronize()
    for l in range(nl):
        sd = pool.attn_decode_batch([convs[i] for i in dec], l, qd[l].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(sd, od[l])
        row = 0
        for i in ext:
            hk, hv = (x[l] for x in _held(*kv[i]))
            assert_close(oe[l, row:row + new[i]], attend_last(f64(q[i][l]), hk, hv), f"layer {l} conv {i}")
            row += new[i]
        for r, i in enumerate(dec):
            hk, hv = (x[l] for x in _held(*kv[i]))
            assert_close(od[l, r:r + 1], attend_last(f64(q[i][l]), hk, hv), f"layer {l} conv {i}")
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,nl,P,n,dec,ordered", [
    (32, 8, 128, 2, 1200, 300, [30000] * 12, True), (16, 8, 128, 2, 1200, 300, [30000] * 12, True),
    (32, 8, 64, 2, 1200, 300, [30000] * 12, True), (32, 8, 128, 24, 1500, 500, [2100, 700], False),
    (32, 8, 64, 24, 1200, 300, [2100, 700], False), (32, 8, 64, 24, 1500, 500, [2100, 700], False)])
def test_chained_tiles(hq, hkv, d, nl, P, n, dec, ordered):
    """Sizes at which a mixed step has one workgroup take a cut tile's pieces in turn, as in a layer's launch beside
    a large decode or in one launch of all layers: the same bits as the separate calls, which give each piece a workgroup."""
    lens, new, m = [P] + dec, [n] + [1] * len(dec), len(dec)
    pool = _pool(nl, hq, hkv, d, sum((a + b + 15) // 16 for a, b in zip(lens, new)) + 16, max_pages=2048, max_convs=16)
    g = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    convs = [pool.conv_create() for _ in lens]
    pool.kv_append_batch(convs, lens, rand(nl, sum(lens), hkv, d), rand(nl, sum(lens), hkv, d))
    qe, qd = rand(nl, n, hq, d), rand(nl, m, hq, d)
    oe, od = pool.mixed_step(convs[:1], [n], convs[1:], rand(nl, n + m, hkv, d), rand(nl, n + m, hkv, d), qe, qd, layer_ordered=ordered)
    for l in range(nl):
        assert torch.equal(pool.attn_extend(convs[:1], [n], l, qe[l]), oe[l]), l
        assert torch.equal(pool.attn_decode_batch(convs[1:], l, qd[l]), od[l]), l
    k, v = pool.kv_read(convs[:1], [0], [P + n])
    torch.cuda.synchronize()
    rows = [0, n // 2, n - 1]
    assert_close(oe[-1, rows].cpu(), attend_rows(f64(qe[-1, rows].cpu()), [P + r for r in rows], f64(k[-1].cpu()), f64(v[-1].cpu())))
    pool.close()


# ---- streams, graphs, failures ---------------------------------------------------------------------
def test_streams_and_two_pools():
    """A pool used from stream after stream; two pools at once on streams of their own."""
    lens = [600, 40]
    streams = [torch.cuda.Stream() for _ in range(2)]
    pools = [_pool(1, 32, 8, 128, 128, s) for s in (1, 2)]
    q = torch.cat([q_tokens(SEED, i, 0, n - 1, 1, 32, 128) for i, n in enumerate(lens)])
    filled = [_fill(p, 1, lens, 8, 128) for p in pools]
    qc = q.cuda()
    torch.cuda.synchronize()
    outs = []
    for turn in range(3):
        for p, (convs, _), s in zip(pools, filled, streams if turn % 2 else streams[::-1]):
            with torch.cuda.stream(s):
                outs.append(p.attn_decode_batch(convs, 0, qc))
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    for i in range(2):
        assert_close(outs[0][i:i + 1], attend_last(f64(q[i:i + 1]), *[x[0] for x in _held(*filled[0][1][i])]))
    for p in pools:
        p.close()


def test_captured_decode_replays():
    """cs_attn_decode_batch_noalloc in a captured graph: every replay gives the eager result for the
    queries of that replay, with eager work on the pool between replays."""
    lens = [700, 33, 4000]
    pool = _pool(1, 32, 8, 128, 400)
    convs, _ = _fill(pool, 1, lens, 8, 128)
    q = torch.zeros(3, 32, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        pool.attn_decode_batch_noalloc(convs, 0, q, out)   # the pool's work moves to this stream before the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pool.attn_decode_batch_noalloc(convs, 0, q, out)
    for turn in range(4):
        x = torch.cat([q_tokens(SEED + turn, i, 0, n - 1, 1, 32, 128) for i, n in enumerate(lens)]).cuda()
        q.copy_(x)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            want = pool.attn_decode_batch(convs, 0, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want), turn
    pool.close()


def test_failed_appends_change_nothing():
    from paper_2606_01839_amd import CS_EHIP, ConserveError
    pool = _pool(1, 8, 2, 64, 32)
    k, v = kv_tokens(SEED, 0, 1, 0, 60, 2, 64)
    c = pool.conv_create()
    pool.kv_append(c, k[:, :20].contiguous().cuda(), v[:, :20].contiguous().cuda())
    before = pool.conv_len(c), pool.conv_pages(c).tolist(), pool.occupancy()
    pool.debug_fail_launches(0)
    q = q_tokens(SEED, 0, 0, 19, 1, 8, 64).cuda()
    for call in (lambda: pool.kv_append(c, k[:, 20:].contiguous().cuda(), v[:, 20:].contiguous().cuda()),
                 lambda: pool.kv_read([c], [0], [20]), lambda: pool.kv_pack_fp4(c), lambda: pool.attn_decode_batch([c], 0, q)):
        with pytest.raises(ConserveError) as e:
            call()
        assert e.value.code == CS_EHIP
        assert before == (pool.conv_len(c), pool.conv_pages(c).tolist(), pool.occupancy())
    pool.debug_fail_launches(-1)
    pool.kv_append(c, k[:, 20:].contiguous().cuda(), v[:, 20:].contiguous().cuda())
    gk, gv = _read(pool, c, 0, 60)
    wk, wv = _held(k, v)
    assert np.array_equal(gk, wk) and np.array_equal(gv, wv)
    pool.close()


def test_offsets_past_32_bits():
    """Blocks more than 2^32 bytes into the pool (every layer's offset, and every page's, is 64-bit)."""
    nl, hq, hkv, d = 40, 8, 8, 128
    n_pages = 8000                     # 139 MB a layer, 5.6 GB in all
    pool = _pool(nl, hq, hkv, d, n_pages, seed=2)
    c = pool.conv_create()
    n = 333
    k, v = kv_tokens(SEED, 0, 1, 0, n, hkv, d)
    pool.kv_append(c, k.expand(nl, -1, -1, -1).contiguous().cuda(), v.expand(nl, -1, -1, -1).contiguous().cuda())
    q = q_tokens(SEED, 0, 0, n - 5, 5, hq, d)
    hk, hv = (x[0] for x in _held(k, v))
    ref = attend_last(f64(q), hk, hv)
    for layer in (0, 31, 39):
        out = pool.attn_extend([c], [5], layer, q.cuda())
        dec = pool.attn_decode_batch([c], layer, q[-1:].contiguous().cuda())
        torch.cuda.synchronize()
        assert_close(out, ref)
        assert_close(dec, ref[-1:])
    gk, _ = _read(pool, c, 0, n)
    assert np.array_equal(gk[39], hk)
    pool.close()
