"""Rotary positions against the fp64 oracle."""
import ctypes

import numpy as np
import pytest
import torch

from kv_cases import TORCH
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu

# of the larger of a pair's magnitudes: the output's rounding, and fp32 angles, cosines and products
EPS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -10, "f32": 2.0 ** -21}


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def bound(x, freq, interleaved, amplitude, dtype):
    """Per element: its pair's magnitude times the eps (elements that are only copied: 0)."""
    size = np.zeros(x.shape)
    for i in range(len(freq)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(freq))
        size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b]) * abs(amplitude)
    return size * EPS[dtype] + (2.0 ** -24 if dtype == "f16" else 0.0) * (size > 0)


def check(n, heads, head_dim, rot, dtype, interleaved=False, inverse=False, first=0, amplitude=1.0, seed=0, **scaling):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(n, heads, head_dim, generator=gen, device="cuda").to(TORCH[dtype])
    pos = (torch.randint(0, 5000, (n,), generator=gen, device="cuda") + first).to(torch.int32)
    rope = L.Rope(rot, interleaved=interleaved, amplitude=amplitude, **scaling)
    y = rope.apply(x, pos, inverse=inverse)
    freq = decode.rope_frequencies(rot, **scaling)
    hx = x.double().cpu().numpy()
    want = decode.rotate(hx, pos.cpu().numpy(), freq, interleaved, amplitude, inverse)
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= bound(hx, freq, interleaved, amplitude, dtype))
    assert torch.equal(y[..., rot:], x[..., rot:])
    return x, pos, rope, y


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,heads,head_dim,rot", [(1, 1, 8, 2), (1, 32, 128, 128), (5, 3, 64, 32), (17, 5, 80, 80),
                                                  (3, 2, 96, 24), (2, 7, 256, 256), (9, 1, 40, 18), (300, 4, 64, 64),
                                                  (4, 9, 200, 144), (7, 71, 128, 62)])
def test_rotation_and_gradient(dtype, interleaved, inverse, n, heads, head_dim, rot):
    check(n, heads, head_dim, rot, dtype, interleaved, inverse, amplitude=1.125 if n % 2 else 1.0, seed=n)


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="banded", factor=8.0, original_len=8192),
                                     dict(scaling="banded", factor=16.0, original_len=4096, low_turns=1.0, high_turns=32.0),
                                     dict(base=500000.0), dict(scaling="linear", factor=0.125)])
def test_scalings(scaling):
    check(20, 4, 128, 128, "f32", seed=4, **scaling)
    check(20, 4, 96, 64, "f32", interleaved=True, seed=5, **scaling)


@pytest.mark.parametrize("first", [1 << 20, (1 << 31) - 5001, -(1 << 31), -4000])
def test_far_and_negative_positions(first):
    # the phase is exact at any int32 position; the oracle's own fp64 angle is off by 2^31 * 2^-52 at most
    check(40, 2, 64, 64, "f32", first=first, seed=6)


def test_strides_and_in_place():
    x, pos, rope, y = check(33, 6, 64, 48, "bf16", seed=7)
    fused = torch.randn(33, 10, 64, device="cuda").bfloat16()
    fused[:, 2:8] = x
    rest = fused.clone()
    out = rope.apply(fused[:, 2:8], pos, out=fused[:, 2:8])
    assert torch.equal(out, y) and torch.equal(fused[:, :2], rest[:, :2]) and torch.equal(fused[:, 8:], rest[:, 8:])
    heads_first = torch.empty(6, 33, 64, device="cuda", dtype=torch.bfloat16)
    rope.apply(x, pos, out=heads_first.transpose(0, 1))
    assert torch.equal(heads_first.transpose(0, 1), y)
    # in place in the layout whose halves cross chunks
    odd = L.Rope(36)
    want = odd.apply(x, pos)
    assert torch.equal(odd.apply(x, pos, out=x), want)


def test_gradient_through_autograd():
    # <g, R x> differentiated by x equals the inverse applied to g, in fp32
    rope = L.Rope(32, interleaved=True, amplitude=1.5)
    pos = torch.arange(100, 105, dtype=torch.int32, device="cuda")
    x, g = torch.randn(5, 2, 40, device="cuda"), torch.randn(5, 2, 40, device="cuda")
    grad = rope.apply(g, pos, inverse=True)
    for _ in range(5):
        d = torch.randn_like(x)
        f = [(g.double() * rope.apply(x + e * 0.5 * d, pos).double()).sum() for e in (1, -1)]
        assert abs(float(f[0] - f[1]) - float((grad.double() * d.double()).sum())) < 1e-4
    back = rope.apply(rope.apply(x, pos), pos, inverse=True)
    assert torch.allclose(back[..., :32], x[..., :32] * 2.25, atol=1e-5) and torch.equal(back[..., 32:], x[..., 32:])


def test_no_tokens_and_a_side_stream():
    rope = L.Rope(16)
    empty = torch.empty(0, 3, 16, device="cuda")
    assert rope.apply(empty, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 3, 16)
    x, pos = torch.randn(9, 3, 16, device="cuda"), torch.arange(9, dtype=torch.int32, device="cuda")
    want = rope.apply(x, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = rope.apply(x, pos)
    side.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    lib = L.load()
    x, pos = torch.randn(4, 2, 64, device="cuda").bfloat16(), torch.arange(4, dtype=torch.int32, device="cuda")
    rope = L.Rope(64).plan

    def status(n=4, heads=2, head_dim=64, dtype=L.LACACHE_BF16, data=x.data_ptr(), stride=128, p=pos.data_ptr(), plan=rope):
        rows = L.lacache_rows(data, stride, 64)
        return lib.lacache_rope_apply(ctypes.addressof(plan) if plan else None, n, heads, head_dim, dtype, ctypes.addressof(rows),
                                      p, 0, ctypes.addressof(rows), None)

    bad, no = L.LACACHE_ERR_INVALID_ARG, L.LACACHE_ERR_UNSUPPORTED
    for kw, want in [(dict(n=-1), bad), (dict(heads=0), bad), (dict(dtype=3), bad), (dict(data=None), bad),
                     (dict(data=x.data_ptr() + 8), bad), (dict(stride=100), bad), (dict(p=None), bad), (dict(plan=None), bad),
                     (dict(head_dim=56), bad), (dict(head_dim=68), no), (dict(head_dim=264), no), (dict(n=0, data=None), 0)]:
        assert status(**kw) == want, kw
    wrong = [dict(x=x[:, :, ::2]), dict(x=x.double()), dict(pos=pos.long()), dict(pos=pos[:3]), dict(x=x[0]),
             dict(out=torch.empty(4, 2, 64, device="cuda")), dict(pos=pos.cpu())]
    for kw in wrong:
        args = dict(x=x, pos=pos)
        args.update(kw)
        with pytest.raises((ValueError, L.LacacheError)):
            L.Rope(32).apply(**args)
