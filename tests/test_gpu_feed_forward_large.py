"""Products whose outputs no single launch holds: what lies around the borders of their ranges, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from ff_util import gated64, linear64, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.get_device_properties(0).total_memory < 200 << 30, reason="tens of gigabytes")]


def bytes_of(rows, k, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    t = torch.empty((rows, k), dtype=torch.int8, device="cuda:0")
    for at in range(0, rows, max(1, (1 << 30) // k)):  # (a gigabyte at a time)
        t[at:at + max(1, (1 << 30) // k)].random_(-127, 128, generator=g)
    return t


def scales(n, seed):
    return torch.rand(n, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0").add_(0.5).mul_(0.01)


def around(total, borders):
    at = sorted({i for b in (0, total, *borders) for i in range(max(0, b - 40), min(total, b + 40))})
    return torch.tensor(at, device="cuda:0")


def check(x, xs, layers, y, rows, columns, act="none"):
    pick = lambda t, i: t[i].cpu().numpy()  # noqa: E731
    part = [(pick(w, columns), pick(s, columns)) for w, s in layers]
    if len(part) == 2:
        want, tol = gated64(pick(x, rows), pick(xs, rows), *part[0], None, *part[1], None, act, "f16")
    else:
        want, tol = linear64(pick(x, rows), pick(xs, rows), *part[0], None, act, None, "f16")
    got = to_numpy(y[rows][:, columns])
    assert (np.abs(got - want) <= tol).all()


def test_more_rows_than_tiles_of_a_launch():
    rows, k, n = (1 << 30) + 77, 16, 1
    x, xs, w, ws = bytes_of(rows, k, 1), scales(rows, 2), bytes_of(n, k, 3), scales(n, 4)
    y = torch.full((rows, n), float("nan"), dtype=torch.float16, device="cuda:0")
    B.ilinear_s8(B.linear_desc(rows=rows, k=k, n=n, dtype=B.ICNN_F16), x, xs, w, ws, None, None, y)
    torch.cuda.synchronize()
    assert not y.isnan().any()
    check(x, xs, [(w, ws)], y, around(rows, [i << 26 for i in range(1, 16)]), torch.arange(n, device="cuda:0"))


def test_single_tokens_on_more_outputs_than_a_launch():
    rows, k, n = 2, 8208, (1 << 23) + 5
    x, xs, w, ws = bytes_of(rows, k, 1), scales(rows, 2), bytes_of(n, k, 3), scales(n, 4)
    up = scales(n, 5)
    y = torch.full((rows, n), float("nan"), dtype=torch.float16, device="cuda:0")
    B.igated_linear_s8(B.linear_desc(rows=rows, k=k, n=n, dtype=B.ICNN_F16, act=B.ICNN_ACT_RELU), x, xs, w, ws, None, w, up, None, y)
    torch.cuda.synchronize()
    assert not y.isnan().any()
    check(x, xs, [(w, ws), (w, up)], y, torch.arange(rows, device="cuda:0"), around(n, [1 << 22, 1 << 23]), "relu")


def test_the_plain_kernel_on_more_outputs_than_a_launch():
    rows, k, n = (1 << 20) + 9, 8, (1 << 14) + 33
    x, xs, w, ws = bytes_of(rows, k, 1), scales(rows, 2), bytes_of(n, k, 3), scales(n, 4)
    y = torch.full((rows, n), float("nan"), dtype=torch.float16, device="cuda:0")
    B.ilinear_s8(B.linear_desc(rows=rows, k=k, n=n, dtype=B.ICNN_F16), x, xs, w, ws, None, None, y)
    torch.cuda.synchronize()
    assert not any(part.isnan().any() for part in y.split(1 << 16))
    check(x, xs, [(w, ws)], y, around(rows, [1 << 19, 522752, 522240]), around(n, [1 << 13]))
