"""Split k in a workspace of exactly the size that was asked for, with a guard behind it: operands at every kind of address, the library's own choice of kernel."""
import numpy as np
import pytest
import torch

from ff_util import Placed, linear64, gated64, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu

GUARD = 1 << 25                                        # bytes: several times the largest workspace there is here


def product(rows, k, n, gated, seed):
    g = np.random.default_rng(seed)
    ints = lambda *s: np.clip(np.rint(g.normal(size=s) * 40), -127, 127).astype(np.int8)  # noqa: E731
    scales = lambda c: g.uniform(0.5, 1.5, size=c).astype(np.float32) / (40 * k ** 0.5)  # noqa: E731
    return ints(rows, k), scales(rows), [(ints(n, k), scales(n)) for _ in range(1 + gated)], g.normal(size=n).astype(np.float32)


def call(d, gated, x, xs, w, bias, y, ws):
    if gated:
        B.igated_linear_s8(d, x, xs, w[0][0], w[0][1], bias, w[1][0], w[1][1], None, y, ws)
    else:
        B.ilinear_s8(d, x, xs, w[0][0], w[0][1], bias, None, y, ws)


@pytest.mark.parametrize("rows,k,n,gated", [(5, 8192, 256, 0), (5, 11008, 1024, 0), (5, 16384, 2048, 0), (8, 11008, 1024, 0), (16, 11008, 2048, 0), (40, 2048, 64, 0),
                                            (64, 11008, 2048, 0), (100, 8192, 512, 0), (320, 8192, 512, 0), (40, 8192, 256, 1), (64, 11008, 512, 1), (24, 16384, 100, 1)])
def test_a_guarded_workspace(rows, k, n, gated):
    xv, xs, layers, bias = product(rows, k, n, gated, rows + k)
    want, tol = (gated64(xv, xs, *layers[0], bias, *layers[1], None, "silu", "f32") if gated
                 else linear64(xv, xs, *layers[0], bias, "none", None, "f32"))
    d = B.linear_desc(rows=rows, k=k, n=n, act=B.ICNN_ACT_SILU if gated else B.ICNN_ACT_NONE, dtype=B.ICNN_F32)
    size = (B.igated_linear_s8_workspace_bytes if gated else B.ilinear_s8_workspace_bytes)(d)
    raw = torch.full((size + GUARD,), 0xA5, dtype=torch.uint8, device="cuda:0")
    raw[:size] = 0
    vector = lambda v: torch.from_numpy(v).to("cuda:0")  # noqa: E731
    XS, BI = vector(xs), vector(bias)
    for at_x, at_w in ((0, 0), (1, 0), (0, 1), (4, 8), (8, 0), (3, 2)):
        print(rows, k, n, gated, at_x, at_w, size, flush=True)
        X = Placed(rows, k, torch.int8, k, at_x, torch.from_numpy(xv))
        W = [(Placed(n, k, torch.int8, k, at_w, torch.from_numpy(w)), vector(s)) for w, s in layers]
        Y = Placed(rows, n, torch.float32)
        for t in (X, Y, *[w for w, _ in W]):
            t.snapshot()
        for _ in range(2):                             # (the second call finds the workspace as the first has left it)
            call(d, gated, X, XS, W, BI, Y, raw if size else None)
            torch.cuda.synchronize()
            assert Y.rest_untouched() and (np.abs(to_numpy(Y.view) - want) <= tol).all(), (at_x, at_w)
        assert all((t.raw == t.before).all() for t in (X, *[w for w, _ in W]))
        assert not raw[:min(size, 4096)].any() and (raw[size:] == 0xA5).all(), (at_x, at_w)


@pytest.mark.parametrize("rows,k,n,gated", [(1, 16384, 512, 0), (4, 11008, 1024, 1), (64, 256, 512, 0), (1000, 512, 4096, 0), (33, 200, 300, 1)])
def test_a_product_that_asks_for_nothing_leaves_another_one_s_workspace_alone(rows, k, n, gated):
    xv, xs, layers, bias = product(rows, k, n, gated, 3)
    d = B.linear_desc(rows=rows, k=k, n=n, dtype=B.ICNN_F32)
    assert (B.igated_linear_s8_workspace_bytes if gated else B.ilinear_s8_workspace_bytes)(d) == 0
    ws = torch.zeros(GUARD, dtype=torch.uint8, device="cuda:0")
    vector = lambda v: torch.from_numpy(v).to("cuda:0")  # noqa: E731
    for at in (0, 1, 8):
        X, W = Placed(rows, k, torch.int8, k, at, torch.from_numpy(xv)), [(Placed(n, k, torch.int8, k, at, torch.from_numpy(w)), vector(s)) for w, s in layers]
        outs = []
        for space in (ws, None):
            outs.append(torch.empty((rows, n), device="cuda:0"))
            call(d, gated, X, vector(xs), W, vector(bias), outs[-1], space)
            torch.cuda.synchronize()
        assert torch.equal(*outs) and not ws.any()
