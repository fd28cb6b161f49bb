"""GELU in its erf form with float32 results, as near its definition as its formula in float32 is: one product of 1 * 1, a row's scale as the activation's argument."""
import numpy as np
import pytest
import torch

from ff_util import act64
from paper_2006_11735_amd import binding as B
from scipy.special import ndtr

pytestmark = pytest.mark.gpu


def gelu(v, kernel, gated, k=64, n=8):
    """v: the arguments, one a row; by kernel (of "ff_kernel").  The first output of each row"""
    rows = len(v)
    x, w = torch.zeros((rows, k), dtype=torch.int8, device="cuda:0"), torch.zeros((n, k), dtype=torch.int8, device="cuda:0")
    x[:, 0] = 1
    w[:, 0] = 1
    xs, one = torch.from_numpy(v).to("cuda:0"), torch.ones(n, device="cuda:0")
    y = torch.empty((rows, n), device="cuda:0")
    d = B.linear_desc(rows=rows, k=k, n=n, act=B.ICNN_ACT_GELU, dtype=B.ICNN_F32)
    try:
        B.icnn_set_tuning("ff_kernel", kernel)
        if gated:                                      # (the second product is zero, its bias 1)
            B.igated_linear_s8(d, x, xs, w, one, None, torch.zeros_like(w), one, one, y)
        else:
            B.ilinear_s8(d, x, xs, w, one, None, None, y)
    finally:
        B.icnn_set_tuning("reset")
    torch.cuda.synchronize()
    assert torch.allclose(y, y[:, :1].expand_as(y), rtol=0, atol=0, equal_nan=True)
    return y[:, 0].cpu().numpy().astype(np.float64)


def check(v, got):
    """In units of 2^-24.  Up to 1.25, of F = 1/2 + v P: half a unit of 1/2 from the sum, of v P (at most 0.395) 2 from P's last step, its coefficients and u, 0.2 from the
    fit, together 1.4 of 1; and 1 of the result from the last product.  Beyond, of F(-|v|): 2 from the reciprocal, 1 from its argument, 3 from R's last steps, 0.8 from the
    fit, 2 from the exponential, 2 from the products, 1.25 v^2 from the exponential's argument; one more than that where it is 1 less it."""
    wide = v.astype(np.float64)
    want, a = wide * ndtr(wide), np.abs(wide)
    below = (11 + 1.25 * a * a) * ndtr(-a)
    unit = np.where(a <= 1.25, 1.4, np.where(wide < 0, below, below + 1))
    tol = 2.0 ** -24 * (a * unit + np.abs(want)) + 2.0 ** -126
    assert (np.abs(got - want) <= tol).all(), (v[np.argmax(np.abs(got - want) - tol)], (np.abs(got - want) / tol).max())
    return np.sqrt(((got - want) ** 2).sum() / (want ** 2).sum())


@pytest.mark.parametrize("gated", [0, 1])
def test_over_its_whole_range(gated):
    for lo, hi in ((-13, 13), (-1.3, 1.3)):
        v = np.linspace(lo, hi, 400001).astype(np.float32)
        check(v, gelu(v, 0, gated))


def test_where_most_arguments_are():
    """Beside the formula in float32 (act64's, taken step by step in float32), which has 3.7e-8 here and 5.6e-8 between -1 and 0"""
    for v, most in ((np.random.default_rng(0).normal(size=300000), 4.2e-8), (np.linspace(-1, 0, 300000), 6.0e-8)):
        v = v.astype(np.float32)
        got = gelu(v, 0, 0)
        check(v, got)
        want = act64(v.astype(np.float64), "gelu")
        assert np.sqrt(((got - want) ** 2).sum() / (want ** 2).sum()) <= most


@pytest.mark.parametrize("kernel,rows", [(1, 300), (2, 4), (3, 64), (4, 300), (9, 300)])
def test_by_every_kernel(kernel, rows):
    for at in (-9.0, -1.25, 0.0, 1.25):
        v = (at + np.linspace(-0.3, 0.3, rows)).astype(np.float32)
        check(v, gelu(v, kernel, 0))
        check(v, gelu(v, kernel, 1))


def test_special_numbers():
    v = np.array([0.0, -0.0, 1e-38, -1e-38, 3e38, -3e38, 40.0, -40.0, np.nan, np.inf], dtype=np.float32)
    got = gelu(v, 0, 0)
    assert (got[:2] == 0).all() and np.allclose(got[2:4], [0.5e-38, -0.5e-38], rtol=1e-3, atol=2e-45)
    assert got[4] == np.float32(3e38) and got[5] == 0 and got[6] == 40 and got[7] == 0 and np.isnan(got[8]) and got[9] == np.inf
