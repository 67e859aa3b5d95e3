"""GPU: what include/conserve_attn.h says of a rotated value before its rounding: within 2^-21 amplitude (|a| + |b|) at
any position. Seen where a pair's two terms cancel, so that the rounding to bf16 is far below that. The bound: the angle is
rounded to fp32 in turns (2^-26 turns, 9.4e-8 radians, near half a turn), its cos and sin are within 1.9e-7
(v_cos_f32, v_sin_f32), and three roundings of 2^-24 follow: 4.7e-7 of |a| + |b| in all."""
import os
import re

import numpy as np
import pytest
import torch

from tests.helpers import f64

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_header_states_the_bounds():
    """CPU: the angle as the kernels make it (64-bit fraction of a turn, its upper 32 bits, fp32) against exact
    arithmetic: the bound that the header names (2^-26 of the rounding to fp32 and 2^-32 of the bits dropped)."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    rng, worst = np.random.default_rng(4), 0.0
    for _ in range(20000):
        f, p = float(np.exp(rng.uniform(np.log(1e-7), np.log(3.0)))), int(rng.integers(0, 1 << 30))
        turns = Decimal(f) / (2 * pi)
        frac = int(turns % 1 * 2 ** 64 + Decimal("0.5")) % 2 ** 64
        top = (frac * p % 2 ** 64) >> 32
        used = float(np.float32(top - 2 ** 32 if top >= 2 ** 31 else top)) / 2 ** 32
        err = (Decimal(used) - turns * p) % 1
        worst = max(worst, float(min(err, 1 - err)))
    src = open(os.path.join(ROOT, "include", "conserve_attn.h")).read()
    m = re.search(r"angle[^.]*within 2\^-(\d+) turns", src)
    assert m, "the header names no bound of the angle"
    stated = int(m[1])
    assert 2.0 ** -(stated + 2) < worst <= 2.0 ** -stated, (worst, stated)
    assert re.search(r"2\^-21 amplitude \(\|a\| \+ \|b\|\)", src)


@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("start", [0, 900_000])
def test_cancelling_pairs(inter, start):
    from paper_2606_01839_amd import KVPool, Rope
    n, d, hq = 3000, 128, 2
    total = start + n
    pool = KVPool(1, hq, 1, d, n_pages=total // 16 + 2, max_convs=1, max_pages_per_conv=total // 16 + 1, device="cuda", kv_format="fp4")
    c = pool.conv_create()
    z = torch.zeros(1, total, 1, d, dtype=torch.bfloat16, device="cuda")
    pool.kv_append(c, z, z)
    rope = Rope(d, base=50000.0, interleaved=inter)
    # (the double product's own error at position 10^6: 1e-10 radians)
    angle = np.arange(start, total)[:, None] * rope.inv_freq
    cos, sin = np.cos(angle), np.sin(angle)
    mant = (128 + np.arange(128)) / 128.0
    head = []
    for first in (True, False):   # a cos - b sin, then a sin + b cos
        p, q = (cos, -sin) if first else (sin, cos)
        big = np.abs(p) >= np.abs(q)           # the term of the larger factor takes the value that is searched for
        ratio = np.where(big, -q / p, -p / q)
        x = mant[None, None] * ratio[..., None]
        xb = f64(torch.from_numpy(x).float().to(torch.bfloat16))
        best = np.abs(xb - x).argmin(-1)
        y, x = mant[best], np.take_along_axis(xb, best[..., None], -1)[..., 0]
        head.append((np.where(big, x, y), np.where(big, y, x)))
    rows = np.zeros((n, hq, d))
    at = (slice(0, d, 2), slice(1, d, 2)) if inter else (slice(0, d // 2), slice(d // 2, d))
    for h, (a, b) in enumerate(head):
        rows[:, h, at[0]], rows[:, h, at[1]] = a, b
    out = f64(pool.rope_q([c], [n], torch.from_numpy(rows).to(torch.bfloat16).cuda(), rope).cpu())
    torch.cuda.synchronize()
    worst, seen = 0.0, 0
    for h, (a, b) in enumerate(head):
        want = a * cos - b * sin if h == 0 else a * sin + b * cos
        size, got = np.abs(a) + np.abs(b), out[:, h, at[h]]
        err = np.abs(got - want)
        assert (err <= 2.0 ** -21 * size + 2.0 ** -8 * np.maximum(np.abs(want), np.abs(got)) + 1e-9).all()   # 2^-8: half a bf16 step
        small = np.abs(want) <= 2.0 ** -15 * size     # the rounding is at most 2^-23 of size there
        seen += small.sum()
        worst = max(worst, (err / size)[small].max())
    print(f"{seen} pairs that cancel to 2^-15, worst error {worst:.3g} of |a| + |b|")
    assert seen > 20000
    pool.close()
