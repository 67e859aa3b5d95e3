"""Oracle: attention of rows that see any set of keys, and trees of drafted tokens (float64, no library code).

A tree of n tokens follows P cached ones: parent[j] is -1 (the last cached token) or an earlier token of the
tree. Token j sees the cached tokens, its ancestors and itself; its position is P plus its depth.
"""
from __future__ import annotations

import math

import numpy as np


def ancestors(parents) -> np.ndarray:
    """[n][n]: whether token j is token i or one of its ancestors, by climbing from i."""
    n = len(parents)
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            j = int(parents[j])
    return see


def depths(parents) -> np.ndarray:
    """Ancestors of each token, itself not counted."""
    return ancestors(parents).sum(axis=1) - 1


def tree_sees(parents, length: int) -> np.ndarray:
    """[n][length]: what the tree that ends a conversation of that length sees."""
    n = len(parents)
    return np.concatenate([np.ones((n, length - n), dtype=bool), ancestors(parents)], axis=1)


def weights(q: np.ndarray, k: np.ndarray, see: np.ndarray) -> np.ndarray:
    """Softmax weights [r][L] of one head's rows q [r][d] over keys k [L][d], exact zeros where a row does not
    see the key (whatever the key holds)."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = (q @ k.T) / math.sqrt(q.shape[-1])
    s = np.where(see, s, -np.inf)
    w = np.exp(s - s.max(axis=1, keepdims=True))
    return w / w.sum(axis=1, keepdims=True)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, see: np.ndarray | None = None) -> np.ndarray:
    """q [r][Hq][d], k, v [L][Hkv][d], see [r][L] (None: everything) -> [r][Hq][d]; zeros without keys."""
    r, hq, d = q.shape
    out = np.zeros((r, hq, d))
    if k.shape[0] == 0 or r == 0:
        return out
    if see is None:
        see = np.ones((r, k.shape[0]), dtype=bool)
    for h in range(hq):
        g = h // (hq // k.shape[1])
        w = weights(q[:, h], k[:, g], see)
        seen = see.any(axis=0)   # keys nobody sees take no part
        out[:, h] = np.where(see[:, seen], w[:, seen], 0.0) @ v[seen, g] if np.isfinite(v[seen, g]).all() else _rowwise(w, v[:, g], see)
    return out


def _rowwise(w, v, see):
    """The same row by row, so that values a row does not see (infinities, NaN) cannot reach it."""
    return np.stack([w[i, see[i]] @ v[see[i]] for i in range(w.shape[0])])


def keep(x: np.ndarray, n_last: int, kept) -> np.ndarray:
    """x [L][..] of a conversation after the last n_last tokens were cut down to those with the given indexes."""
    base = x.shape[0] - n_last
    return np.concatenate([x[:base], x[base:][np.asarray(kept, dtype=np.int64)]])
