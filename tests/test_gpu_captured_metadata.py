"""GPU: calls captured into a graph whose metadata is too large for their launches' own arguments (3 KiB): it
is part of the graph, so a replay reads it whatever the pool's upload ring (8 MiB) has held since."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SEED = 909
HQ, HKV, D = 4, 2, 64


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_replays_after_the_ring_has_gone_round(fmt):
    """Queries of 500 conversations (one of them merged from several items) rotated and decoded in one graph, 420 of
    them in another order in a second; between replays eager decodes of other batches fill the ring 1.5 times."""
    from paper_2606_01839_amd import KVPool, Rope
    n = 500
    lens = [1 + (37 * i) % 53 for i in range(n)]
    lens[7] = 5000
    pool = KVPool(1, HQ, HKV, D, n_pages=sum((x + 15) // 16 for x in lens) + 8, max_convs=n, max_pages_per_conv=400,
                  placement_seed=5, device="cuda", kv_format=fmt)
    convs = [pool.conv_create() for _ in range(n)]
    rope = Rope(D)
    s = torch.cuda.Stream()
    g = torch.Generator(device="cuda").manual_seed(SEED)
    k, v = (torch.randn((1, sum(lens), HKV, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):   # the pool's work moves to this stream before the capture
        pool.kv_append_rope(convs, lens, k, v, rope)
    torch.cuda.synchronize()
    batches = [convs, convs[::-1][:420]]
    graphs = []
    for sel in batches:
        q = torch.zeros(len(sel), HQ, D, dtype=torch.bfloat16, device="cuda")
        turned, out = torch.empty_like(q), torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            pool.attn_decode_batch_noalloc(sel, 0, q, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            pool.rope_q(sel, [1] * len(sel), q, rope, turned)
            pool.attn_decode_batch_noalloc(sel, 0, turned, out)
        graphs.append((graph, sel, q, turned, out))
    other = convs[3:400][::-1]
    qo = torch.randn((len(other), HQ, D), generator=g, device="cuda").to(torch.bfloat16)
    oo = torch.empty_like(qo)
    torch.cuda.synchronize()
    for turn in range(4):
        with torch.cuda.stream(s):
            for _ in range(1500):   # 8 KiB of descriptors each
                pool.attn_decode_batch(other, 0, qo, oo)
        torch.cuda.synchronize()
        for graph, sel, q, turned, out in graphs[::1 if turn % 2 else -1]:
            x = torch.randn(q.shape, generator=g, device="cuda").to(torch.bfloat16)
            q.copy_(x)
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                want_q = pool.rope_q(sel, [1] * len(sel), x, rope)
                want = pool.attn_decode_batch(sel, 0, want_q)
            torch.cuda.synchronize()
            assert torch.equal(turned, want_q) and torch.equal(out, want), turn
    pool.close()
