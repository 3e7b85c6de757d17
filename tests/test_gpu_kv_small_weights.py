"""Rows whose weight lies on one key, whose value is 0 in some dimensions: there the output is made of the other keys' small weights.

f16 weights (f16 caches; 8-bit caches with few rows, where they are weight times V's scale) keep 11 bits down to 2^-14, and below that
2^-25. The kernels bring a row's largest to 2^7 or more, so a small one is off by 2^-32 of the largest at most, and an output by that
times the sum of its values: 2^-32 max_j(p_j a_j) sum_j |v_jd| / a_j, where a_j is 1 for f16 caches and the row's largest |v| for 8-bit
ones, whose values are a code of at most 1 (of the largest one) times it. With |v_jd| <= a_j that is at most
2^-32 max_j(p_j a_j) times the number of keys."""
import numpy as np
import pytest
import torch

from test_gpu_kv_shared import filled, ints, library  # noqa: F401 (the fixture)
from kv_cases import TORCH, bounds as tolerances
from oracle import decode

pytestmark = pytest.mark.gpu


def largest_share(q, k, v, lengths, scale, eight):
    """max_j p_j a_j a row, times the number of keys (8 bit), or max_j p_j times the sum of |v_jd|."""
    heads = q.shape[1]
    out = np.zeros(q.shape)
    for s, n in enumerate(lengths):
        for h in range(heads):
            g = h // (heads // k[s].shape[1])
            kk, vv = k[s][:n, g], np.abs(v[s][:n, g])
            w = kk @ q[s, h] * scale
            p = np.exp(w - w.max())
            p /= p.sum()
            out[s, h] = (p * vv.max(-1)).max() * n if eight else p.max() * vv.sum(0)
    return out


@pytest.mark.parametrize("fmt,dtype", [("f16", "f16"), ("int8", "bf16"), ("e4m3", "bf16"), ("int8", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("head_dim,group", [(64, 2), (128, 2), (256, 2), (256, 7), (128, 7)])
@pytest.mark.parametrize("strength", [1.0, 1.5, 2.0, 4.0])
def test_one_key_outweighs_all_others(fmt, dtype, head_dim, group, strength):
    H, common = 2, 700
    c = filled(fmt, [(common, [720 + 5 * i for i in range(6)])], H, head_dim, seed=51)
    B, f = len(c.lengths), head_dim ** -0.5
    # a common key's own direction as every query (some of them the sequences' own keys), its value 0 but in every fourth dimension
    gen = torch.Generator(device="cuda")
    gen.manual_seed(52)
    k = torch.randn(1, H, head_dim, generator=gen, device="cuda")
    v = torch.zeros(1, H, head_dim, device="cuda")
    v[..., ::4] = 50.0
    at = ints([333])
    c.kv.append(k.to(TORCH[dtype]), v.to(TORCH[dtype]), ints([0]), at, c.table)
    q = (k.repeat_interleave(group, 1).expand(B, H * group, head_dim) * strength * 8 / head_dim ** 0.5).to(TORCH[dtype]).contiguous()
    pool = c.kv.pool()                                       # values so large that the bound's least, 2^-24, is none
    pool["vs" if "vs" in pool else "v"].mul_(2.0 ** (6 if dtype == "f16" else 20))
    kk, vv = c.values()
    hq = q.double().cpu().numpy()
    want, want_lse, mass, span = decode.attend(hq, kk, vv, c.lengths, 1, f)
    tol, _ = tolerances(want, mass, span, want_lse, hq, kk, f, dtype)
    if fmt != "bf16":
        tol = tol + 2.0 ** -32 * largest_share(hq, kk, vv, c.lengths, f, fmt in ("int8", "e4m3"))
    shared = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common))
    plain = c.kv.attend(q, c.table, c.len_dev)
    c.kv.sync()
    for got in (shared, plain):
        off = np.abs(got.double().cpu().numpy() - want)
        assert np.all(off <= tol), float((off / tol).max())
