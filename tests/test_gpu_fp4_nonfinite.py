"""GPU: infinities and NaN that enter a 4-bit cache against its rule (K and V must be finite): a group with one is NaN to
every call that reads it, and nothing else is touched."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle.attention import attend_last
from tests.helpers import assert_close, f64, kv_tokens, q_tokens

pytestmark = pytest.mark.gpu

SEED = 611
HQ, HKV = 8, 2


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L", [20, 300, 3000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("via", ["append", "transfer"])
def test_a_value_that_is_not_finite_is_nan_to_every_reader(d, L, bad, via):
    """One value of kv head 0's V, at the first token, in the middle and at the last, beside values of every magnitude: the
    queries of that head get NaN in all dims, however small the token's weight; head 1 keeps its outputs. The transfer
    from a bf16 pool holds the bytes of an append."""
    from paper_2606_01839_amd import KVPool

    def pool(fmt):
        return KVPool(1, HQ, HKV, d, n_pages=L // 16 + 4, max_convs=2, max_pages_per_conv=L // 16 + 2, device="cuda", kv_format=fmt)

    k, v = kv_tokens(SEED, 0, 1, 0, L, HKV, d)
    q = q_tokens(SEED, 0, 0, L - 1, 1, HQ, d)
    hk, hv = o4.held(f64(k), f64(v))
    ref = attend_last(f64(q), hk[0], hv[0])
    for at in (0, L // 2, L - 1):
        for shift in (0, 80):
            kk, vv, qq = k.clone(), v.clone(), q.clone()
            vv[0, at, 0, 5], vv[0, at, 0, 9], vv[0, at, 0, 17] = bad, 3e38, -1e-30
            if shift:   # the bad token's key far against every query of its head: its weight is 0 in fp32
                kk[0, at, 0], qq[0, :4] = -shift, 1.0
            p, src = pool("fp4"), pool("bf16")
            cs = src.conv_create()
            src.kv_append(cs, kk.cuda(), vv.cuda())
            wire = src.kv_pack_fp4(cs)
            if via == "append":
                c = p.conv_create()
                p.kv_append(c, kk.cuda(), vv.cuda())
            else:
                c = p.kv_unpack(wire, L)
            dec, ext = p.attn_decode_batch([c], 0, qq.cuda()), p.attn_extend([c], [1], 0, qq.cuda())
            _, gv = p.kv_read([c], [0], [L])
            torch.cuda.synchronize()
            assert torch.equal(p.kv_pack(c), wire)
            spoilt = np.zeros((L, HKV), bool)
            spoilt[at, 0] = True
            assert np.isnan(f64(gv.cpu())[0, spoilt]).all() and np.array_equal(f64(gv.cpu())[0, ~spoilt], hv[0, ~spoilt])
            for out in (dec, ext):
                assert torch.isnan(out[0, :4]).all(), (at, shift)
                assert_close(out[:, 4:], ref[:, 4:])
            p.close()
            src.close()
