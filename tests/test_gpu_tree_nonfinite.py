"""GPU: rows of a tree that see a token which is not finite. What the formula gives them: a score of NaN or +infinity makes the row NaN, one
of -infinity takes the key out; an infinite value makes its dim that infinity, values of both signs NaN; a value over 4-bit pages whose
scale is NaN makes all dims of the kv head NaN. Rows that do not see the token have the oracle's values."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import seen as so
from tests.helpers import f64, kv_tokens, q_tokens
from tests.seen_helpers import assert_within, tree

pytestmark = pytest.mark.gpu

SEED = 1618
SHAPES = [(32, 8, 128, 8), (4, 2, 64, 20), (8, 8, 128, 40), (8, 8, 128, 100), (16, 8, 64, 130)]   # few rows a kv head, and tiles
PREFIXES = [0, 45, 2047]


def _run(k, v, hq, hkv, d, n, length, fmt):
    from paper_2606_01839_amd import KVPool
    pool = KVPool(1, hq, hkv, d, n_pages=256, max_convs=2, max_pages_per_conv=256, placement_seed=3, device="cuda", kv_format=fmt)
    c = pool.conv_create()
    pool.kv_append(c, k.cuda(), v.cuda())
    parents = tree(n, 9)
    q = q_tokens(SEED, 1, 0, 0, n, hq, d)
    out = pool.attn_tree([c], [n], [parents], 0, q.cuda()).cpu()
    pool.close()
    return out, q, so.tree_sees(parents, length)


def _path(n):
    """A token that some rows do not see, and a descendant of it that fewer see."""
    see = so.ancestors(tree(n, 9))
    a = max(range(n // 4, n - 1), key=lambda j: (see[:, j].sum() < n, see[:, j].sum()))
    b = int(np.argwhere(see[a + 1:, a])[0, 0]) + a + 1
    assert see[:, a].sum() > see[:, b].sum() and not see[:, a].all()
    return a, b


def _held(k, v, fmt):
    return o4.held(f64(k), f64(v)) if fmt == "fp4" else (f64(k), f64(v))


@pytest.mark.parametrize("prefix", PREFIXES)
@pytest.mark.parametrize("hq,hkv,d,n", SHAPES)
def test_values_of_both_signs(hq, hkv, d, n, prefix):
    """+infinity in dim 7 of a token, -infinity in it of a descendant, -infinity alone in dim 9 and NaN in dim 11 of the descendant."""
    a, b = _path(n)
    k, v = kv_tokens(SEED, n, 1, 0, prefix + n, hkv, d)
    well = v.clone()
    v[0, prefix + a, :, 7] = float("inf")
    v[0, prefix + b, :, 7] = -float("inf")
    v[0, prefix + b, :, 9] = -float("inf")
    v[0, prefix + b, :, 11] = float("nan")
    out, q, see = _run(k, v, hq, hkv, d, n, prefix + n, "bf16")
    kf, vf, qf = f64(k[0]), f64(well[0]), f64(q)
    ref = so.attend(qf, kf, vf, see)
    sa, sb = see[:, prefix + a], see[:, prefix + b]
    assert (out[sa & ~sb][:, :, 7] == float("inf")).all()
    assert torch.isnan(out[sa & sb][:, :, 7]).all() and not (sb & ~sa).any()
    assert (out[sb][:, :, 9] == -float("inf")).all() and torch.isnan(out[sb][:, :, 11]).all()
    fill = torch.from_numpy(ref).to(torch.bfloat16)
    out[sa, :, 7] = fill[sa][:, :, 7]
    out[sb, :, 9], out[sb, :, 11] = fill[sb][:, :, 9], fill[sb][:, :, 11]
    assert_within(out, qf, kf, vf, see, ref, "the rest")


@pytest.mark.parametrize("prefix", PREFIXES)
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("hq,hkv,d,n", SHAPES)
def test_value_over_4_bit_pages(hq, hkv, d, n, bad, prefix):
    """The group of a token and kv head is NaN: all dims of the rows that see it, in the heads of that kv head."""
    a, _ = _path(n)
    k, v = kv_tokens(SEED, n, 1, 0, prefix + n, hkv, d)
    well = v.clone()
    v[0, prefix + a, 1, 5] = float(bad)
    out, q, see = _run(k, v, hq, hkv, d, n, prefix + n, "fp4")
    kf, vf = _held(k[0], well[0], "fp4")
    ref = so.attend(f64(q), kf, vf, see)
    hit = torch.tensor(see[:, prefix + a])
    group = hq // hkv
    mine = slice(group, 2 * group)
    assert torch.isnan(out[hit][:, mine]).all()
    out[hit, mine] = torch.from_numpy(ref).to(torch.bfloat16)[hit][:, mine]
    assert_within(out, f64(q), kf, vf, see, ref, "the rest", True)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("prefix", PREFIXES)
@pytest.mark.parametrize("hq,hkv,d,n", SHAPES)
def test_infinite_key(hq, hkv, d, n, prefix, fmt):
    """A key of +infinity in one dim: where the row's query is positive there the row is NaN, where it is negative the weight is 0 and the row
    is as if the key were not there. Over 4-bit pages the key's group is NaN, and so is every row that sees it."""
    a, _ = _path(n)
    k, v = kv_tokens(SEED, n, 1, 0, prefix + n, hkv, d)
    well = k.clone()
    k[0, prefix + a, :, 3] = float("inf")
    out, q, see = _run(k, v, hq, hkv, d, n, prefix + n, fmt)
    kf, vf = _held(well[0], v[0], fmt)
    qf = f64(q)
    hit = see[:, prefix + a]
    without = see.copy()
    without[:, prefix + a] = False
    some = without.any(axis=1)
    without[~some] = see[~some]
    ref = so.attend(qf, kf, vf, without)
    nan = hit[:, None] & ((qf[:, :, 3] >= 0) | ~some[:, None]) if fmt == "bf16" else np.repeat(hit[:, None], hq, axis=1)
    assert nan.any() and (fmt == "fp4" or (hit[:, None] & ~nan).any())
    assert torch.isnan(out[torch.tensor(nan)]).all()
    out[torch.tensor(nan)] = torch.from_numpy(ref[nan]).to(torch.bfloat16)
    assert_within(out, qf, kf, vf, without, ref, "the rest", fmt == "fp4")
