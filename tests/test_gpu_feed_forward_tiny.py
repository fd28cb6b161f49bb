"""irms_norm_s8 of rows whose squares leave float32's normal numbers, without an eps that would outweigh them: their norm is that of any other row."""
import numpy as np
import pytest
import torch

from ff_util import DTYPES, rows64, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu

SIZES = [1.0, 2.0 ** -49, 2.0 ** -52, 2.0 ** -62, 1e-21, 1e-23, 1e-30, 2.0 ** -110]     # of a row's numbers


def check(q, scale, s, gamma, eps):
    """tolerances of the other rows: a mean of c squares and five roundings; five of 2^-24 of at most 127"""
    u, want = rows64(s, gamma, eps)
    tol = (s.shape[1] / 64 + 16) * 2.0 ** -25 + 5 * 2.0 ** -24
    assert (np.abs(scale - want) <= tol * want).all(), (scale, want)
    assert (np.abs(q - u / want[:, None]) <= 0.5 + 127 * 5 * 2.0 ** -24).all() and (np.abs(q).max(1) == 127).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-35, 1e-30, 1e-12])
@pytest.mark.parametrize("c", [1, 64, 1000, 1500, 4096, 5001, 9000, 20000, 40000])
def test_tiny_rows(dtype, eps, c):
    torch_dtype, code = DTYPES[dtype]
    g = torch.Generator().manual_seed(c)
    size = torch.tensor(SIZES + SIZES[::-1], dtype=torch.float64)[:, None]
    x = ((torch.rand((len(size), c), generator=g, dtype=torch.float64) + 0.5) * size).to(torch_dtype)
    r = ((torch.rand((len(size), c), generator=g, dtype=torch.float64) - 0.5) * 0.5 * size).to(torch_dtype)
    gamma = torch.rand(c, generator=g) + 0.5
    total = (x.float() + r.float()).to(torch_dtype)
    X, R, G = x.to("cuda:0"), r.to("cuda:0"), gamma.to("cuda:0")
    d = B.norm_desc(rows=len(size), c=c, dtype=code, gamma_dtype=B.ICNN_F32, eps=eps)
    for residual, keep in ((False, None), (True, None), (True, "own"), (True, "x"), (True, "residual")):
        x2, r2 = X.clone(), R.clone()
        out = {None: None, "own": torch.zeros_like(X), "x": x2, "residual": r2}[keep]
        q, scale = torch.empty((len(size), c), dtype=torch.int8, device="cuda:0"), torch.empty(len(size), device="cuda:0")
        B.irms_norm_s8(d, x2, r2 if residual else None, G, out, q, scale)
        torch.cuda.synchronize()
        s = total if residual else x
        if out is not None:
            assert torch.equal(out.cpu(), s)
        check(to_numpy(q).astype(np.int64), to_numpy(scale), to_numpy(s), to_numpy(gamma), float(np.float32(eps)))


@pytest.mark.parametrize("c", [3, 700, 4096, 40000])
def test_tiny_rows_and_large_gammas(c):
    """products with gamma of the usual size: they are what decides that a row is none of zeros"""
    g = torch.Generator().manual_seed(c)
    x = ((torch.rand((2, c), generator=g) + 0.5) * torch.tensor([[2.0 ** -120], [2.0 ** -100]])).to("cuda:0")
    gamma = ((torch.rand(c, generator=g) + 0.5) * 2.0 ** 100).to("cuda:0")
    q, scale = torch.empty((2, c), dtype=torch.int8, device="cuda:0"), torch.empty(2, device="cuda:0")
    B.irms_norm_s8(B.norm_desc(rows=2, c=c, dtype=B.ICNN_F32, eps=0), x, None, gamma, None, q, scale)
    torch.cuda.synchronize()
    check(to_numpy(q).astype(np.int64), to_numpy(scale), to_numpy(x), to_numpy(gamma), 0)


def test_a_scale_beyond_float32_is_a_nan():
    """one number of 2^125 among zeros of a row with a gamma that takes the normalised value beyond float32"""
    x, gamma = torch.zeros((2, 4096), device="cuda:0"), torch.ones(4096, device="cuda:0")
    x[:, 7] = torch.tensor([2.0 ** -60, 2.0 ** -20], device="cuda:0")
    gamma[7] = 2.0 ** 127 + 2.0 ** 126
    d = B.norm_desc(rows=2, c=4096, dtype=B.ICNN_F32, eps=0)
    q, scale = torch.ones((2, 4096), dtype=torch.int8, device="cuda:0"), torch.zeros(2, device="cuda:0")
    B.irms_norm_s8(d, x, None, gamma, None, q, scale)
    torch.cuda.synchronize()
    want = 64 * 1.5 * 2.0 ** 127 / 127                # below the largest float32: the row is a row like any other
    assert torch.allclose(scale, torch.full_like(scale, want), rtol=1e-5) and (q[:, 7] == 127).all() and q.sum() == 254
    x = torch.zeros((1, 1 << 20), device="cuda:0")
    x[0, 9] = 1.0
    gamma = torch.full((1 << 20,), 2.0 ** 126, device="cuda:0")
    q, scale = torch.empty((1, 1 << 20), dtype=torch.int8, device="cuda:0"), torch.zeros(1, device="cuda:0")
    B.irms_norm_s8(B.norm_desc(rows=1, c=1 << 20, dtype=B.ICNN_F32, eps=0), x, None, gamma, None, q, scale)
    torch.cuda.synchronize()
    assert scale.isnan().all()
