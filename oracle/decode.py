"""Oracle of the decoding operators (test infrastructure only): rotary positions, the cache's 8-bit rows and the attention of
new tokens over cached ones, in fp64 numpy from their definitions.
"""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                     original_len: float = 0.0, low_turns: float = 1.0, high_turns: float = 4.0) -> np.ndarray:
    """Angle a position of each rotated pair."""
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    w = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if scaling == "linear":
        w = w / factor
    if scaling == "banded":
        g = np.clip((original_len * w / (2 * math.pi) - low_turns) / (high_turns - low_turns), 0.0, 1.0)
        w = (1 - g) * w / factor + g * w
    return w


def rotate(x, pos, freq, interleaved: bool = False, amplitude: float = 1.0, inverse: bool = False) -> np.ndarray:
    """x [n x heads x d]: pair i of each row turned by pos * freq[i] (by the negated angle if inverse), times amplitude."""
    y = np.array(x, dtype=np.float64)
    for i, w in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(freq))
        angle = np.asarray(pos, dtype=np.float64)[:, None] * w * (-1.0 if inverse else 1.0)
        u, v = np.array(y[..., a]), np.array(y[..., b])
        y[..., a] = amplitude * (u * np.cos(angle) - v * np.sin(angle))
        y[..., b] = amplitude * (v * np.cos(angle) + u * np.sin(angle))
    return y


def attend(q, k, v, lengths, new_tokens: int, scale: float, starts=None, window: int = 0):
    """q [seqs * T x heads x d]; k and v: per sequence [tokens x kv_heads x d]. Returns out, lse, and for error bounds the
    sum of p |v| per output and the largest sum of |q k| * scale among a row's visible keys."""
    n, heads, d = q.shape
    out, mass = np.zeros((n, heads, d)), np.zeros((n, heads, d))
    lse, span = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for s, length in enumerate(lengths):
        kv_heads = k[s].shape[1]
        for t in range(new_tokens):
            p = length - new_tokens + t
            lo = max(0, 0 if starts is None else int(starts[s]), p - window + 1 if window else 0)
            if p < lo:
                continue
            r = s * new_tokens + t
            for h in range(heads):
                g = h // (heads // kv_heads)
                kk, vv = k[s][lo:p + 1, g], v[s][lo:p + 1, g]
                score = kk @ q[r, h] * scale
                w = np.exp(score - score.max())
                out[r, h] = w @ vv / w.sum()
                mass[r, h] = w @ np.abs(vv) / w.sum()
                lse[r, h] = score.max() + math.log(w.sum())
                span[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
    return out, lse, mass, span
