"""iquantize_weights_s4's numbers are w / scale to nearest, ties to even, of the scale that it returns: half of a group's largest number is 3.5 steps of max / 7, and with a
float32 scale the rounding of max / 7 moves it to one side or the other by less than a float32 quotient shows."""
import numpy as np
import pytest
import torch

from ff_util import DTYPES, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu


def nearest(w, s):
    """The definition, exactly: of float64 numbers that hold float32 ones, (2 t + 1) s has four more bits than s"""
    a = np.abs(w)
    t = np.minimum(np.floor(a / s), 7)
    t = np.where(t * s > a, t - 1, t)
    t = np.where((t + 1) * s <= a, t + 1, t)
    d = 2 * a - (2 * t + 1) * s
    t = np.where(d > 0, t + 1, np.where(d < 0, t, t + t % 2))
    return (np.minimum(t, 7) * np.sign(w)).astype(int)


def quantized(w, group, scales):
    n, k = w.shape
    p, s = torch.empty(B.iweights_s4_bytes(n, k), dtype=torch.uint8, device="cuda:0"), torch.empty((n, -(-k // group)), dtype=DTYPES[scales][0], device="cuda:0")
    code = next(c for t, c in DTYPES.values() if t is w.dtype)
    B.iquantize_weights_s4(B.quantize_s4_desc(n=n, k=k, group=group, dtype=code, scale_dtype=DTYPES[scales][1]), w.to("cuda:0"), p, s)
    torch.cuda.synchronize()
    half = to_numpy(p).reshape(n, -1, 16)
    q = np.concatenate([half & 15, half >> 4], 2).reshape(n, -1)[:, :k].astype(int)
    return np.where(q > 7, q - 16, q), to_numpy(s)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scales", list(DTYPES))
@pytest.mark.parametrize("group", [32, 128, 256])
def test_every_number_is_the_nearest(dtype, scales, group):
    g = torch.Generator().manual_seed(group)
    w = (torch.randn((300, 1024), generator=g) * (torch.rand((300, 1), generator=g) + 0.5)).to(DTYPES[dtype][0])
    top = w.view(300, -1, group).abs().amax(2).float() / 2
    w.view(300, -1, group)[:, :, 3] = top.to(w.dtype)
    w.view(300, -1, group)[:, :, group - 2] = -top.to(w.dtype)
    q, s = quantized(w, group, scales)
    wide = np.repeat(s, group, 1)
    halves = np.abs(to_numpy(w)) * 2 == np.repeat(2 * top.to(w.dtype).double().numpy(), group, 1)
    assert halves.sum() >= 2 * top.numel()
    want = nearest(to_numpy(w), wide)
    assert (q == want).all(), (int((q != want).sum()), int((q != want)[halves].sum()))


@pytest.mark.parametrize("size", [1.0, 2.0 ** -20, 2.0 ** -128, 2.0 ** 120])
def test_numbers_next_to_a_tie(size):
    """float32 weights on both sides of (t + 1/2) scale, as near as there are, also where scales are subnormal"""
    g = np.random.default_rng(4)
    most = (7 * g.uniform(1, 2, size=(4000, 1)) * size).astype(np.float32)
    s = most / np.float32(7)
    at = ((np.arange(7) + 0.5) * s.astype(np.float64)).astype(np.float32)
    w = np.concatenate([most, at, np.nextafter(at, np.float32(0)), np.nextafter(at, np.float32(np.inf)), -at, np.zeros((4000, 3), np.float32)], 1)
    w = np.clip(w, -most, most)
    q, got = quantized(torch.from_numpy(w), 32, "f32")
    assert (got == s).all()
    want = nearest(w.astype(np.float64), s.astype(np.float64))
    assert (q == want).all(), int((q != want).sum())
