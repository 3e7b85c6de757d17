"""Draft verification for reusing the lookahead prefix on a miss (test infrastructure only).

Section 3.3 ("Speculative Decoding"): when a query is not served from the cache, its k draft tokens f_k(x),
already decoded for the lookahead check, are verified by the target model f in one forward pass. From the
first token on, draft token t is accepted if P_f(t) >= P_g(t), where P_f and P_g are the probabilities the
target and the draft assign to it. The first rejected token ends the reuse, and f decodes from there. The
tokens reused for a query are its accepted prefix: the number of leading positions that pass. A served query
(HIT) decodes nothing, so none of its tokens are verified (-1).

verify_sample is the form for drafts that were drawn: acceptance and the next token by given random numbers, in exact
rational arithmetic on the fp32 values.
"""
from __future__ import annotations

from fractions import Fraction
from itertools import accumulate

import numpy as np

from .lookup import HIT


def accepted_prefix(p_target, p_draft, status=None) -> np.ndarray:
    """Per query: the number of leading draft tokens with P_f >= P_g; -1 for a HIT when status is given."""
    pf = np.asarray(p_target, dtype=np.float64)
    pg = np.asarray(p_draft, dtype=np.float64)
    B, k = pf.shape
    out = np.empty(B, dtype=np.int32)
    for b in range(B):
        n = 0
        while n < k and pf[b, n] >= pg[b, n]:
            n += 1
        out[b] = n
    if status is not None:
        out[np.asarray(status) == HIT] = -1
    return out


def _whole(x) -> list:
    """fp32 values as whole multiples of 2^-149; NaN and what is not positive as 0."""
    x = np.asarray(x, dtype=np.float32)
    m, e = np.frexp(np.where(x > 0, x, 0).astype(np.float64))
    return [int(a) << int(b) if b >= 0 else int(a) >> -int(b) for a, b in zip(m * 2.0 ** 24, e.astype(int) - 24 + 149)]


def draw(weights: list, u: float) -> int:
    """The first i whose cumulative weight exceeds u times the total; the last of any weight if none does; -1 without any."""
    upto = list(accumulate(weights))
    some = [i for i, w in enumerate(weights) if w > 0]
    if not some:
        return -1
    target = Fraction(float(u)) * upto[-1]
    return next((i for i in some if upto[i] > target), some[-1])


def verify_sample(p_target, p_draft, drafts, u, status=None):
    """p_target [B x k + 1 x V], p_draft [B x k x V] or None, drafts [B x k], u [B x k + 1]: (accepted, token) per query."""
    p_target = np.asarray(p_target, dtype=np.float32)
    B, rows, V = p_target.shape
    accepted, token = np.full(B, -1, np.int32), np.full(B, -1, np.int32)
    for b in range(B):
        if status is not None and status[b] == HIT:
            continue
        n, refused = 0, -1
        while n < rows - 1 and 0 <= drafts[b][n] < V:
            x = int(drafts[b][n])
            q, p = 1.0 if p_draft is None else float(p_draft[b][n][x]), float(p_target[b, n, x])
            if not (np.isfinite(q) and np.isfinite(p) and Fraction(float(u[b][n])) * Fraction(q) < Fraction(p)):
                refused = x
                break
            n += 1
        accepted[b] = n
        p = _whole(p_target[b, n])
        if refused >= 0:
            q = np.zeros(V, np.float32) if p_draft is None else np.asarray(p_draft[b][n], np.float32)
            if p_draft is None:
                q[refused] = 1.0
            seen = np.isfinite(q)
            less = [max(x - y, 0) if ok else 0 for x, y, ok in zip(p, _whole(q), seen)]
            p = less if any(less) else p
        token[b] = draw(p, u[b][rows - 1])
    return accepted, token
