"""GPU: scores of any magnitude that fp32 holds. Keys and queries are +-1 times powers of two, so every score is an
integer times a power of two, exact in fp32 and in both kinds of pages; from 2^12 on the softmax is the mean over the
keys of the largest score (the next is 2^12 2 / sqrt(d) and more below), which the kernels give up to the output's
rounding and their fp32 sums (helpers.GAMMA_ACC): the weights of equal scores are equal."""
import numpy as np
import pytest
import torch

from oracle.attention import attend_rows
from oracle import fp4 as o4
from tests.helpers import GAMMA_ACC, arith_bound, f64, half_ulp_bf16

pytestmark = pytest.mark.gpu

POWERS = [0, 12, 20, 22, 23, 24, 27, 30, 31, 33, 40, 60, 100]


def _inputs(L, n, hq, hkv, d, seed):
    """K with powers 0, Q with the powers of a score in turn. Query head 0 points away from every key: all its scores
    are negative, and a key's rises with the dims in which it differs."""
    r = np.random.default_rng(seed)
    sign = lambda *s: r.choice([-1.0, 1.0], s)
    k, v, q = sign(L, hkv, d), r.standard_normal((L, hkv, d)), sign(n, hq, d)
    u = sign(d)
    k[:, 0] = u * np.where(r.random((L, d)) < 0.1, -1, 1)
    q[:, 0] = -u
    power = np.array([POWERS[i % len(POWERS)] for i in range(n)])
    q *= 2.0 ** power[:, None, None]
    return *(torch.from_numpy(x).to(torch.bfloat16) for x in (k, v, q)), power


def _check(got, q, pos, power, hk, hv, what):
    ref = attend_rows(f64(q), pos, hk, hv)
    g = f64(got)
    assert np.isfinite(g).all(), f"{what}: {(~np.isfinite(g)).any((1, 2)).nonzero()[0][:20]} of powers {power}"
    tol = half_ulp_bf16(np.maximum(np.abs(ref), np.abs(g))) + GAMMA_ACC * np.abs(hv).max()
    near = power == 0
    if near.any():
        tol[near] += arith_bound(f64(q)[near], np.asarray(pos)[near], hk, hv, ref[near])
    bad = np.argwhere(np.abs(g - ref) > tol)
    assert bad.size == 0, f"{what}: {bad[:5]} powers {power[bad[:5, 0]]}"


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (16, 2, 64), (8, 2, 128), (8, 8, 128)])
def test_prefill_extend_and_decode(fmt, hq, hkv, d):
    from paper_2606_01839_amd import KVPool
    L = 1500
    k, v, q, power = _inputs(L, L, hq, hkv, d, 5)
    pool = KVPool(1, hq, hkv, d, n_pages=400, max_convs=len(POWERS) + 1, max_pages_per_conv=100, device="cuda", kv_format=fmt)
    hk, hv = o4.held(f64(k), f64(v)) if fmt == "fp4" else (f64(k), f64(v))
    assert np.array_equal(hk, f64(k))
    c = pool.conv_create()
    pool.kv_append(c, k[None].cuda(), v[None].cuda())
    pre = pool.attn_prefill_turn1([c], [L], 0, q.cuda())
    n = 45   # few rows: their keys are cut into pieces
    ext = pool.attn_extend([c], [n], 0, q[-n:].contiguous().cuda())
    dec = torch.cat([pool.attn_decode_batch([c], 0, (q[-1:].double() * 2.0 ** (p - power[-1])).to(torch.bfloat16).contiguous().cuda())
                     for p in POWERS])
    torch.cuda.synchronize()
    rows = np.r_[0:90, 600:640, L - 70:L]
    _check(pre.cpu()[rows], q[rows], rows, power[rows], hk, hv, "prefill")
    _check(ext.cpu(), q[-n:], np.arange(L - n, L), power[-n:], hk, hv, "extend")
    ps = np.array(POWERS)
    qd = torch.cat([(q[-1:].double() * 2.0 ** (p - power[-1])).to(torch.bfloat16) for p in POWERS])
    _check(dec.cpu(), qd, [L - 1] * len(POWERS), ps, hk, hv, "decode")
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("ordered", [False, True])
def test_mixed_step(fmt, hq, hkv, d, ordered):
    """The same bits as the separate calls, and the oracle's."""
    from paper_2606_01839_amd import KVPool
    L, n = 700, 60
    k, v, q, power = _inputs(L + n, n, hq, hkv, d, 6)
    k2, v2, q2, _ = _inputs(L + 1, len(POWERS), hq, hkv, d, 7)
    hold = (lambda *x: o4.held(*map(f64, x))) if fmt == "fp4" else (lambda *x: tuple(map(f64, x)))
    m = len(POWERS)
    pool = KVPool(1, hq, hkv, d, n_pages=50 * (m + 2), max_convs=m + 1, max_pages_per_conv=60, device="cuda", kv_format=fmt)
    c, convs = pool.conv_create(), [pool.conv_create() for _ in range(m)]
    pool.kv_append(c, k[None, :L].contiguous().cuda(), v[None, :L].contiguous().cuda())
    for x in convs:
        pool.kv_append(x, k2[None, :L].contiguous().cuda(), v2[None, :L].contiguous().cuda())
    cat = lambda a, b: torch.cat([a[L:]] + [b[L:]] * m)[None].contiguous().cuda()
    oe, od = pool.mixed_step([c], [n], convs, cat(k, k2), cat(v, v2), q[None].cuda(), q2[None].cuda(), layer_ordered=ordered)
    se, sd = pool.attn_extend([c], [n], 0, q.cuda()), pool.attn_decode_batch(convs, 0, q2.cuda())
    torch.cuda.synchronize()
    assert torch.equal(od[0], sd)
    _check(oe[0].cpu(), q, np.arange(L, L + n), power, *hold(k, v), "mixed extend")
    _check(se.cpu(), q, np.arange(L, L + n), power, *hold(k, v), "extend")
    _check(od[0].cpu(), q2, [L] * m, np.array(POWERS), *hold(k2, v2), "mixed decode")
    pool.close()
