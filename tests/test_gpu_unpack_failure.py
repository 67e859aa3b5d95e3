"""GPU: an unpack whose launch fails changes nothing: no conversation is left behind, no page is taken, and the next
unpack gets the pages that the failed one had."""
import pytest
import torch

from tests.helpers import kv_tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_a_failed_unpack_leaves_nothing(fmt):
    from paper_2606_01839_amd import CS_EHIP, ConserveError, KVPool
    n = 100

    def pool(max_convs=2):
        return KVPool(1, 4, 2, 64, n_pages=16, max_convs=max_convs, max_pages_per_conv=16, placement_seed=4, device="cuda",
                      kv_format=fmt)

    src, dst, other = pool(), pool(), pool()
    k, v = kv_tokens(1, 0, 1, 0, n, 2, 64)
    c = src.conv_create()
    src.kv_append(c, k.cuda(), v.cuda())
    wire = src.kv_pack(c)
    for _ in range(4):   # more often than the pool has slots or pages for
        dst.debug_fail_launches(0)
        with pytest.raises(ConserveError) as e:
            dst.kv_unpack(wire, n)
        assert e.value.code == CS_EHIP and dst.occupancy() == (0, 16)
        dst.debug_fail_launches(-1)
    a, b = dst.kv_unpack(wire, n), other.kv_unpack(wire, n)
    assert dst.conv_pages(a).tolist() == other.conv_pages(b).tolist()
    assert torch.equal(dst.kv_pack(a), wire)
    dst.conv_create()   # the other slot is free
    torch.cuda.synchronize()
    for p in (src, dst, other):
        p.close()
