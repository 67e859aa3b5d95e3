"""Oracle: what a 4-bit KV cache holds of K and V, and its wire format (float64, no library code).

A group of values (K: 32 consecutive dims of one token and kv head; V: all dims of one) is held as
e2m1 values times one power of two. Readings: the power is 2^(floor(log2 a) - 2) with a the group's
largest magnitude, at least 2^-126, so that the largest e2m1 value, 6, is reached; values round to the
nearest, ties to the even code, and saturate at 6.

Wire: [layer][logical page][kv head] blocks of 17 d bytes: two 4-bit codes a byte, the first in the low
bits, K as [d/32 groups][16 tokens][32 dims], V as [4][16 rows c][d/16 tiles t][4 tokens] (part i: dim
16 t + c of tokens 4 i ..); then the powers as bytes e (2^(e - 127)): K [16 tokens][d/32], V [16 tokens];
zeros up to 17 d. Token slots past the end are zeros.
"""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])   # of codes 0 .. 7; 8 .. 15 are their negatives
PAGE = 16


def encode(x: np.ndarray, group: int):
    """(codes 0 .. 15, exponents) of x [..., d] with one exponent per `group` values."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    top = np.abs(g).max(-1, keepdims=True)
    e = np.frexp(top)[1] - 1 - 2                                # floor(log2 top) - 2
    e = np.maximum(np.where(top > 0, e, -126), -126)
    y = np.abs(g) * 2.0 ** -e.astype(np.float64)
    dist = np.abs(y[..., None] - VALUES)
    near = dist.min(-1, keepdims=True)
    c = np.arange(8)
    # the nearest value; of two equally near the one of even code
    code = np.where(dist == near, c + 8 * (c % 2), 99).min(-1)
    code = np.where(code >= 8, code - 8, code)
    codes = code + 8 * np.signbit(g)
    return codes.reshape(x.shape).astype(np.uint8), e[..., 0]


def decode(codes: np.ndarray, e: np.ndarray) -> np.ndarray:
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes & 7]
    g = v.reshape(*v.shape[:-1], e.shape[-1], -1) * 2.0 ** e[..., None].astype(np.float64)
    return g.reshape(v.shape)


def held(k: np.ndarray, v: np.ndarray):
    """The values a 4-bit cache holds of k and v [..., d]."""
    d = k.shape[-1]
    return decode(*encode(k, 32)), decode(*encode(v, d))


def serialize(k: np.ndarray, v: np.ndarray) -> np.ndarray:
    """k, v: [layers][L][Hkv][d] float64 values -> wire bytes."""
    nl, L, hkv, d = k.shape
    n_pages = (L + PAGE - 1) // PAGE
    kc, ke = encode(k, 32)
    vc, ve = encode(v, d)
    out = np.zeros((nl, n_pages, hkv, 17 * d), dtype=np.uint8)

    def paged(a):   # [layers][pages][Hkv][16 tokens][...], zeros past the end
        p = np.zeros((nl, n_pages * PAGE) + a.shape[2:], dtype=np.int64)
        p[:, :L] = a
        p = p.reshape((nl, n_pages, PAGE) + a.shape[2:])
        return np.moveaxis(p, 2, 3)

    def nibbles(a):
        a = a.reshape(nl, n_pages, hkv, -1)
        return (a[..., 0::2] + 16 * a[..., 1::2]).astype(np.uint8)

    kp = paged(kc).reshape(nl, n_pages, hkv, PAGE, d // 32, 32)
    out[..., :8 * d] = nibbles(np.moveaxis(kp, 4, 3))
    vp = paged(vc).reshape(nl, n_pages, hkv, 4, 4, d // 16, 16)          # [i][token of i][t][c]
    out[..., 8 * d:16 * d] = nibbles(vp.transpose(0, 1, 2, 3, 6, 5, 4))   # [i][c][t][token]
    n_k = PAGE * d // 32
    out[..., 16 * d:16 * d + n_k] = paged(ke + 127).reshape(nl, n_pages, hkv, -1)
    out[..., 16 * d + n_k:16 * d + n_k + PAGE] = paged(ve + 127).reshape(nl, n_pages, hkv, PAGE)
    return out.reshape(-1)
