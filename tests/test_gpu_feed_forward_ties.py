"""iquantize_rows_s8 on 16-bit streams gives the very numbers of its definition, u * 127 / max|u| to nearest, ties to even: a number of such a row is a multiple of
its spacing, so only an exact tie comes nearer to a border than float32 holds apart.  Half of a row's largest number, at 63.5, is one."""
import numpy as np
import pytest
import torch

from ff_util import DTYPES, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu


def nearest(x):
    """The definition on float64 numbers that hold a 16-bit stream's: every product below is exact"""
    a, m = np.abs(x), np.abs(x).max(1, keepdims=True)
    k = np.floor(a * 127 / m)
    k = np.where(k * m > 127 * a, k - 1, k)
    k = np.where((k + 1) * m <= 127 * a, k + 1, k)
    d = 254 * a - (2 * k + 1) * m
    return (np.where(d > 0, k + 1, np.where(d < 0, k, k + k % 2)) * np.sign(x)).astype(np.int64), int((d == 0).sum())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,c", [(64, 500), (300, 4096), (64, 16384), (9, 40000)])      # the kernels of a wave, of one and of more workgroups' rows, and of two passes
def test_every_number_is_the_nearest(dtype, rows, c):
    torch_dtype, code = DTYPES[dtype]
    g = torch.Generator().manual_seed(c)
    x = (torch.randn((rows, c), generator=g) * (torch.rand((rows, 1), generator=g) + 0.5)).to(torch_dtype)
    half = x.abs().amax(1, keepdim=True).float() / 2
    x[:, 3:5] = torch.cat([half, -half], 1).to(torch_dtype)
    want, ties = nearest(to_numpy(x))
    assert ties >= 2 * rows
    X, q, scale = x.to("cuda:0"), torch.empty((rows, c), dtype=torch.int8, device="cuda:0"), torch.empty(rows, device="cuda:0")
    B.iquantize_rows_s8(B.norm_desc(rows=rows, c=c, dtype=code), X, q, scale)
    torch.cuda.synchronize()
    wrong = (to_numpy(q).astype(np.int64) != want).sum()
    assert wrong == 0, (int(wrong), ties)


@pytest.mark.parametrize("exponent", [-14, 0, 15])
def test_every_largest_number_of_a_binade_has_its_tie_at_64(exponent):
    m = (1 + torch.arange(1024) / 1024) * 2.0 ** exponent
    x = torch.stack([m, m / 2, -m / 2, torch.zeros(1024)], 1).to(torch.float16).to("cuda:0")
    q, scale = torch.empty((1024, 4), dtype=torch.int8, device="cuda:0"), torch.empty(1024, device="cuda:0")
    B.iquantize_rows_s8(B.norm_desc(rows=1024, c=4, dtype=B.ICNN_F16), x, q, scale)
    torch.cuda.synchronize()
    exact = (x[:, 1] * 2 == x[:, 0]).cpu()             # (a subnormal half may be rounded)
    assert exact.sum() >= 512 and (q.cpu()[exact] == torch.tensor([127, 64, -64, 0], dtype=torch.int8)).all()
