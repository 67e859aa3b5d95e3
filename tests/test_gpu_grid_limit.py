"""GPU: batches of more workgroups than a grid holds (2^32 threads; such a launch runs some of them and reports no error)
are refused, and the largest that fit are computed. A conversation of one token gives its value exactly."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_decode_and_extend_of_66000_conversations_at_128_heads():
    from paper_2606_01839_amd import CS_EHIP, ConserveError, KVPool
    n, heads, d = 66000, 128, 64          # 8.4 million workgroups of 512 threads; 65500 fit
    pool = KVPool(1, heads, heads, d, n_pages=n, max_convs=n, max_pages_per_conv=1, placement_seed=3, device="cuda", kv_format="fp4")
    convs = [pool.conv_create() for _ in range(n)]
    g = torch.Generator(device="cuda").manual_seed(1)
    k, q = (torch.empty((n, heads, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    v = torch.randint(-1, 2, (n, heads, d), generator=g, device="cuda").to(torch.bfloat16)   # -1, 0, 1: as 4 bits hold them
    pool.kv_append_batch(convs, [1] * n, k[None], v[None])
    out = torch.empty_like(q)
    for call in (lambda: pool.attn_decode_batch(convs, 0, q, out), lambda: pool.attn_decode_batch_noalloc(convs, 0, q, out)):
        with pytest.raises(ConserveError) as e:
            call()
        assert e.value.code == CS_EHIP
    m = 65500
    out[:m].fill_(float("nan"))
    pool.attn_decode_batch(convs[:m], 0, q[:m], out[:m])
    assert torch.equal(out[:m], v[:m])
    out.fill_(float("nan"))
    pool.attn_extend(convs, [1] * n, 0, q, out)   # two launches
    assert torch.equal(out, v)
    torch.cuda.synchronize()
    pool.close()
