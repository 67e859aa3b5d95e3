"""GPU: cross attention over states that hold infinities, and over a cache whose slots behind the last state hold what a failed
append left there. Every row sees every state: an infinite value makes its dim infinite (of both signs: NaN) whatever the number of
rows, and what is no state reaches no row."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import seen as so
from tests.helpers import f64, kv_tokens, q_tokens
from tests.seen_helpers import assert_within

pytestmark = pytest.mark.gpu

SEED = 2718
TILES = [(4, 2, 64, 70), (8, 8, 128, 100), (16, 8, 64, 40), (32, 8, 128, 17), (8, 1, 128, 300)]   # more than 64 rows a kv head
ROWS = [(4, 2, 64, 1), (32, 8, 128, 3), (8, 8, 128, 40), (16, 8, 64, 32), (32, 8, 128, 16), (32, 8, 64, 12)]   # 2 to 64
LENS = [5, 16, 30, 64, 81, 100, 128, 333, 1000]   # 1 to 63 pages, of every remainder to four; whole last pages and others


def _pool(hq, hkv, d, fmt="bf16", nl=1, n_pages=128, max_convs=4):
    from paper_2606_01839_amd import KVPool
    return KVPool(nl, hq, hkv, d, n_pages=n_pages, max_convs=max_convs, max_pages_per_conv=n_pages, placement_seed=3, device="cuda",
                  kv_format=fmt)


def _infinity(hq, hkv, d, n, length):
    """Dim 7 holds an infinity in the last state, dim 9 a negative one in the first of the last page, dim 11 both."""
    pool = _pool(hq, hkv, d)
    k, v = kv_tokens(SEED, length, 1, 0, length, hkv, d)
    well, last = v.clone(), (length - 1) // 16 * 16
    v[0, length - 1, :, 7] = float("inf")
    v[0, last, :, 9] = -float("inf")
    v[0, length - 1, :, 11], v[0, length // 2, :, 11] = float("inf"), -float("inf")
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    q = q_tokens(SEED, 1, 0, 0, n, hq, d)
    out = pool.attn_cross([c], [n], 0, q.cuda()).cpu()
    assert (out[:, :, 7] == float("inf")).all() and (out[:, :, 9] == -float("inf")).all()
    assert torch.isnan(out[:, :, 11]).all()
    kf, vf, qf = f64(k[0]), f64(well[0]), f64(q)
    see = np.ones((n, length), dtype=bool)
    ref = so.attend(qf, kf, vf, see)
    dims = [7, 9, 11]
    out[:, :, dims] = torch.from_numpy(ref[:, :, dims]).to(torch.bfloat16)
    assert_within(out, qf, kf, vf, see, ref, "other dims")
    pool.close()


@pytest.mark.parametrize("length", LENS)
@pytest.mark.parametrize("hq,hkv,d,n", TILES)
def test_infinite_value_many_rows(hq, hkv, d, n, length):
    _infinity(hq, hkv, d, n, length)


@pytest.mark.parametrize("length", LENS)
@pytest.mark.parametrize("hq,hkv,d,n", ROWS)
def test_infinite_value_few_rows(hq, hkv, d, n, length):
    _infinity(hq, hkv, d, n, length)


@pytest.mark.parametrize("length", [5, 81, 128, 1000])
@pytest.mark.parametrize("hq,hkv,d,n", [x for x in TILES + ROWS if x[1] > 1])
def test_value_over_4_bit_pages(hq, hkv, d, n, length):
    """The last state's group of a kv head is NaN, and all dims of the heads that read it."""
    pool = _pool(hq, hkv, d, "fp4")
    k, v = kv_tokens(SEED, length, 1, 0, length, hkv, d)
    well = v.clone()
    v[0, length - 1, 1, 5] = float("inf")
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    q = q_tokens(SEED, 1, 0, 0, n, hq, d)
    out = pool.attn_cross([c], [n], 0, q.cuda()).cpu()
    mine = slice(hq // hkv, 2 * (hq // hkv))
    assert torch.isnan(out[:, mine]).all()
    (kf, vf), qf = o4.held(f64(k[0]), f64(well[0])), f64(q)
    see = np.ones((n, length), dtype=bool)
    ref = so.attend(qf, kf, vf, see)
    out[:, mine] = torch.from_numpy(ref).to(torch.bfloat16)[:, mine]
    assert_within(out, qf, kf, vf, see, ref, "other heads", True)
    pool.close()


def _failed_append(hq, hkv, d, n, fmt, length, bad):
    """An append whose K and V are stored and whose queries' launch then fails: no conversation is longer, and attention is bit for
    bit what it was before."""
    from paper_2606_01839_amd import CS_EHIP, ConserveError, Rope
    pool = _pool(hq, hkv, d, fmt, n_pages=1300, max_convs=2)
    c, other = pool.conv_create(), pool.conv_create()
    k, v = kv_tokens(SEED, 3, 1, 0, length, hkv, d)
    pool.kv_append(c, k.cuda(), v.cuda())
    q = q_tokens(SEED, 4, 0, 0, n, hq, d).cuda()
    want = pool.attn_cross([c], [n], 0, q)
    assert torch.isfinite(want).all()
    news = [40, 20000]   # so many queries turn in a launch of their own, behind the append's
    x = torch.full((1, sum(news), hkv, d), float(bad), dtype=torch.bfloat16, device="cuda")
    turned = torch.zeros((1, sum(news), hq, d), dtype=torch.bfloat16, device="cuda")
    pool.debug_fail_launches(1)
    with pytest.raises(ConserveError) as e:
        pool.kv_append_rope([c, other], news, x, x, Rope(d), q=turned, q_out=turned)
    pool.debug_fail_launches(-1)
    assert e.value.code == CS_EHIP and pool.conv_len(c) == length and pool.conv_len(other) == 0
    if length % 16:
        page = pool.kv_view()[0, pool.conv_pages(c)[-1]]
        assert not torch.isfinite(page.view(torch.bfloat16)).all() if fmt == "bf16" else (page == 255).any()   # it was stored
    assert torch.equal(pool.attn_cross([c], [n], 0, q), want)
    pool.close()


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("length", [5, 30, 333])
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,n", TILES)
def test_failed_append_many_rows(hq, hkv, d, n, fmt, length, bad):
    _failed_append(hq, hkv, d, n, fmt, length, bad)


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("length", [5, 30, 333])
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,n", ROWS)
def test_failed_append_few_rows(hq, hkv, d, n, fmt, length, bad):
    _failed_append(hq, hkv, d, n, fmt, length, bad)
