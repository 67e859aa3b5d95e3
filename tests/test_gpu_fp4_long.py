"""GPU: the 4-bit transfer of conversations of more pages than one launch of it takes (2^24 pages of 256 threads are
2^32, more than a grid holds). 270 million tokens at one layer, one kv head of 64: 18 GB of 4-bit pages."""
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGES = (1 << 24) + 3
D = 64


def _pool(fmt, pages, seed):
    from paper_2606_01839_amd import KVPool
    return KVPool(1, 1, 1, D, n_pages=pages, max_convs=1, max_pages_per_conv=pages, placement_seed=seed, device="cuda",
                  kv_format=fmt)


def test_pack_of_a_4_bit_pool():
    """A wire unpacked and packed again is the wire, from the first byte to the last."""
    wire = torch.empty(PAGES * 17 * D, dtype=torch.uint8, device="cuda")
    wire.view(torch.int32).random_(generator=torch.Generator(device="cuda").manual_seed(1))
    pool = _pool("fp4", PAGES, 3)
    c = pool.kv_unpack(wire, 16 * PAGES)
    assert pool.kv_pack_size(c) == wire.numel()
    assert torch.equal(pool.kv_pack(c), wire)
    torch.cuda.synchronize()
    pool.close()


def test_pack_from_a_bf16_pool():
    """The same million pages sixteen times over, and three more: their wire sixteen times, and its start."""
    part = 1 << 20
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.empty((1, 16 * part, 1, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    pool = _pool("bf16", PAGES, 5)
    c = pool.conv_create()
    pool.kv_append(c, k, v)
    first = pool.kv_pack_fp4(c)
    for _ in range(15):
        pool.kv_append(c, k, v)
    pool.kv_append(c, k[:, :16 * (PAGES - 16 * part)].contiguous(), v[:, :16 * (PAGES - 16 * part)].contiguous())
    wire = pool.kv_pack_fp4(c)
    torch.cuda.synchronize()
    for i in range(17):
        got = wire[i * first.numel():(i + 1) * first.numel()]
        assert torch.equal(got, first[:got.numel()]), i
    pool.close()
