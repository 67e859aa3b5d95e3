"""Shared by the tests of trees and cross attention: trees, and the bound of a kernel's rounding for rows that see any
set of keys (derived in tests/helpers.py for causal rows: only the weights differ)."""
from __future__ import annotations

import math
import random

import numpy as np

from oracle import seen as so
from tests.helpers import DELTA_BF16, GAMMA_ACC, f64, half_ulp_bf16


def tree(n: int, seed: int, kind: str = "mixed"):
    """Parents of n tokens: a chain, siblings only, or both with several roots."""
    r = random.Random(seed)
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1] * n
    return [-1 if i == 0 or r.random() < 0.1 else i - 1 if r.random() < 0.4 else r.randrange(i) for i in range(n)]


def bound(q, k, v, see, ref, query_bits=False):
    """Per element, without the output's rounding: |O' - O| <= delta / (1 - delta) sum_j w_j |V_j - O| + 2^-12 sum_j w_j
    |V_j|, with delta the relative error of a weight (helpers.arith_bound). `query_bits`: scores over 4-bit pages take a
    query's dims below 2^-8 of the largest of their 32 (head dim 64: 16) to within 2^-16 of that largest, which moves a score by at most
    2^-16 max|q| sum |k| / sqrt(d); a weight relative to the others moves by e to the power of twice that."""
    r, hq, d = q.shape
    out = np.zeros_like(ref)
    for h in range(hq):
        g = h // (hq // k.shape[1])
        w = so.weights(q[:, h], k[:, g], see)
        s = np.abs(q[:, h] @ k[:, g].T) / (math.log(2.0) * math.sqrt(d))
        x = np.where(w > 0, s, 0.0).max(axis=1)
        delta = DELTA_BF16 + math.log(2.0) * (d / 16 + 3) * 2.0 ** -24 * x + 2.0 ** -21
        if query_bits:
            off = 2.0 ** -16 * np.abs(q[:, h]).max(axis=1) * np.abs(k[:, g]).sum(axis=1).max() / math.sqrt(d)
            delta = delta + np.expm1(2 * off)
        dev = np.abs(v[None, :, g, :] - ref[:, h][:, None, :])
        out[:, h] = (delta / (1 - delta))[:, None] * np.einsum("rj,rjd->rd", w, dev) + GAMMA_ACC * (w @ np.abs(v[:, g]))
    return out


def assert_within(got, q, k, v, see, ref, what="", query_bits=False):
    g = f64(got)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    assert np.isfinite(g).all(), f"{what}: non-finite output"
    tol = bound(q, k, v, see, ref, query_bits) + half_ulp_bf16(np.maximum(np.abs(ref), np.abs(g)))
    err = np.abs(g - ref)
    worst = np.unravel_index(np.argmax(err / tol), err.shape)
    assert (err <= tol).all(), f"{what}: |err| {err[worst]:.3e} > bound {tol[worst]:.3e} at {worst} (ref {ref[worst]:.4e}, got {g[worst]:.4e})"
