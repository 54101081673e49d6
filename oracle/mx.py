"""CPU definitions of the quantised cache and of the attention over shared
prompts, in numpy float64 — test infrastructure only, like the rest of this
package.

Blocks of 32 channels share a power of two 2^e; codes are E4M3 ("mxfp8") or
E2M1 ("mxfp4").  The magnitudes of a format are listed in full, so that the
nearest one (ties to the even code) is found by search and not by the
arithmetic of a conversion.  Pinned by ``tests/test_oracle_mx.py``.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def magnitudes(fmt: str) -> np.ndarray:
    """Magnitudes by code, ascending (without the sign bit and NaN)."""
    if fmt == "mxfp4":
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    codes = np.arange(127)
    e, m = codes >> 3, codes & 7
    return np.where(e == 0, m * 2.0 ** -9, (8.0 + m) * 2.0 ** (e - 10.0))


def quantize(x: np.ndarray, fmt: str):
    """(codes, scale bytes) of the rows x ([..., d] float64): codes one a byte
    with the sign in its top bit (mxfp8) or bit 3 (mxfp4, not yet packed)."""
    levels = magnitudes(fmt)
    v = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    e = np.full(top.shape, -127)
    while (short := (levels[-1] * np.exp2(e.astype(float)) < top)).any():
        e = e + short
    y = np.abs(v) / np.exp2(e.astype(float))[..., None]
    hi = np.clip(np.searchsorted(levels, y), 1, len(levels) - 1)
    lo = hi - 1
    below, above = y - levels[lo], levels[hi] - y
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = code | np.where(np.signbit(v), 128 if fmt == "mxfp8" else 8, 0)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Codes as they are stored: two a byte for mxfp4, the even channel low."""
    return codes if fmt == "mxfp8" else codes[..., 0::2] | (codes[..., 1::2] << 4)


def values(stored: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """The float64 rows of stored codes and scale bytes."""
    if fmt == "mxfp4":
        c = np.stack([stored & 15, stored >> 4], -1).reshape(*stored.shape[:-1], 2 * stored.shape[-1])
        sign, c = c >> 3, c & 7
    else:
        sign, c = stored >> 7, stored & 127
    v = np.append(magnitudes(fmt), np.nan)[c] * np.where(sign, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(float) - 127))
    return v * np.repeat(s, BLOCK, -1)


def attention(Q, K, V, scale: float | None = None) -> np.ndarray:
    """softmax(scale Q K^T) V in float64, 0 for a row without keys or with logits
    -inf alone."""
    Q, K, V = (np.asarray(t, np.float64) for t in (Q, K, V))
    if not K.shape[0]:
        return np.zeros_like(Q)
    s = Q @ K.T * (1 / math.sqrt(Q.shape[1]) if scale is None else scale)
    top = np.maximum(s.max(1, keepdims=True), -np.finfo(float).max)
    p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    return np.where(total > 0, (p @ V) / np.where(total > 0, total, 1.0), 0.0)


def prefix_attention(Q, K, V, Kg, Vg, k: int, idx=None, prefix_len=None, gen_len=None, scale=None) -> np.ndarray:
    """The attention of Q [B, Hq, q, d] over prompts K, V [P, H, n, d] and own
    rows Kg, Vg [B, H, ng, d] (or None), sequence by sequence."""
    B, Hq = Q.shape[:2]
    P, H, n = K.shape[:3]
    out = np.zeros(Q.shape)
    for b in range(B):
        p = b // (B // P)
        np_ = k if prefix_len is None else min(k, max(0, int(prefix_len[p])))
        ng = 0 if Kg is None else Kg.shape[2] if gen_len is None else min(Kg.shape[2], max(0, int(gen_len[b])))
        for hq in range(Hq):
            h = hq // (Hq // H)
            rows = np.arange(np_) if idx is None else np.clip(np.asarray(idx)[p * H + h, :np_], 0, n - 1)
            Ks, Vs = K[p, h, rows], V[p, h, rows]
            if ng:
                Ks, Vs = np.concatenate([Ks, Kg[b, h, :ng]]), np.concatenate([Vs, Vg[b, h, :ng]])
            out[b, hq] = attention(Q[b, hq], Ks, Vs, scale)
    return out
