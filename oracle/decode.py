"""Oracle of the decoding operators (test infrastructure only): rotary positions, the attention of new tokens over cached ones,
the weights that cached tokens gather and eviction by them, in fp64 numpy from their definitions.
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


def weigh(q, k, lengths, new_tokens: int, scale: float, lse, past=None, decay: float = 1.0, starts=None, window: int = 0):
    """q [seqs * T x heads x d], lse [seqs * T x heads]; k and past: per sequence [tokens x kv_heads x d] and [kv_heads x tokens].
    Returns per sequence the weights [kv_heads x tokens], and the same sums with each query's share times
    its largest sum of |q k| * scale, and times |lse|, for error bounds."""
    got = []
    for s, length in enumerate(lengths):
        kv_heads, heads = k[s].shape[1], q.shape[1]
        w, by_span, by_lse = (np.zeros((kv_heads, length)) for _ in range(3))
        if past is not None:
            w[:, :max(0, length - new_tokens)] = decay * np.asarray(past[s], np.float64)[:, :max(0, length - new_tokens)]
        for t in range(new_tokens):
            p = length - new_tokens + t
            lo = max(0, 0 if starts is None else int(starts[s]), p - window + 1 if window else 0)
            if p < lo:
                continue
            r = s * new_tokens + t
            for h in range(heads):
                if lse[r, h] == -np.inf:
                    continue
                g = h // (heads // kv_heads)
                kk = k[s][lo:p + 1, g]
                share = np.exp(kk @ q[r, h] * scale - lse[r, h])
                w[g, lo:p + 1] += share
                by_span[g, lo:p + 1] += share * (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
                by_lse[g, lo:p + 1] += share * abs(lse[r, h])
        got.append((w, by_span, by_lse))
    return got


def evict(weights, lengths, keep: int, recent: int, starts=None):
    """weights: per sequence [kv_heads x tokens]. Per sequence and head the kept positions, ascending."""
    kept = []
    for s, length in enumerate(lengths):
        start = min(length, max(0, 0 if starts is None else int(starts[s])))
        rows = []
        for w in np.asarray(weights[s], np.float64):
            held = list(range(start, length))
            if len(held) <= keep:
                rows.append(held)
                continue
            last = held[len(held) - recent:]
            rest = sorted(held[:len(held) - recent], key=lambda j: (np.isnan(w[j]), 0.0 if np.isnan(w[j]) else -w[j], j))
            rows.append(sorted(rest[:keep - recent] + last))
        kept.append(rows)
    return kept
