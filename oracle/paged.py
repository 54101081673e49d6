"""CPU definitions of rotary positions, of rows written into the pages of a
cache and of the attention over pages and drafted rows, in numpy float64 — test
infrastructure only, like the rest of this package.  Pinned by
``tests/test_oracle_paged.py``.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from . import mx

# pi to 60 digits, as a fraction: angles of far positions are reduced with it before they are rounded.
PI = Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59)


def angle(freq: float, pos: int) -> float:
    """pos x freq, reduced to one turn in exact arithmetic."""
    return float(Fraction(float(freq)) * int(pos) % (2 * PI))


def rotate(x: np.ndarray, pos: np.ndarray, freq, axis, adjacent: bool = False) -> np.ndarray:
    """The rows x [H, rows, d] turned by pos [axes, rows]."""
    out = np.array(x, np.float64)
    pairs = len(freq)
    for i in range(pairs):
        a = np.array([angle(freq[i], p) for p in pos[axis[i]]])
        u, w = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
        out[..., u] = x[..., u] * np.cos(a) - x[..., w] * np.sin(a)
        out[..., w] = x[..., w] * np.cos(a) + x[..., u] * np.sin(a)
    return out


def places(pages: np.ndarray, ps: int, pool: int, start, m: int, count=None) -> list:
    """(sequence, new row, page, row of the page) of every row that goes in."""
    out = []
    for b in range(pages.shape[0]):
        for i in range(m if count is None else min(m, int(count[b]))):
            place = int(start[b]) + i
            if 0 <= place < pages.shape[1] * ps and 0 <= pages[b, place // ps] < pool:
                out.append((b, i, int(pages[b, place // ps]), place % ps))
    return out


def tree_attention(Q, K, V, pages, n: int, Kt=None, Vt=None, cache_len=None, tree_len=None, mask=None, scale=None,
                   absolute: bool = False) -> np.ndarray:
    """Attention of Q [B, Hq, q, d] over rows of the pool K, V [pages, H, ps, d]
    and drafted rows Kt, Vt [B, H, n_t, d] (or None).  mask [B, q, n_t] of truth
    values (None: all).  absolute: of |V|, the scale of the errors."""
    B, Hq, q, d = Q.shape
    H, ps = K.shape[1:3]
    out = np.zeros(Q.shape)
    scale = 1 / math.sqrt(d) if scale is None else scale
    for b in range(B):
        m = n if cache_len is None else min(n, max(0, int(cache_len[b])))
        j = np.arange(m)
        page = np.clip(pages[b, j // ps], 0, K.shape[0] - 1)
        t = 0 if Kt is None else Kt.shape[2] if tree_len is None else min(Kt.shape[2], max(0, int(tree_len[b])))
        for hq in range(Hq):
            h = hq // (Hq // H)
            Kc, Vc = K[page, h, j % ps], V[page, h, j % ps]
            for i in range(q):
                Ks, Vs = Kc, Vc
                if t:
                    seen = np.arange(t) if mask is None else np.flatnonzero(mask[b, i, :t])
                    Ks, Vs = np.concatenate([Ks, Kt[b, h, seen]]), np.concatenate([Vs, Vt[b, h, seen]])
                out[b, hq, i] = mx.attention(Q[b, hq, i:i + 1], Ks, np.abs(Vs) if absolute else Vs, scale)[0]
    return out
