"""Every kernel of igrouped_linear_s8 and igrouped_gated_linear_s8, at the forms that the library picks by itself for large shares only: tiles of several sizes copied through
registers, offsets that are none in each kernel, and that all of them give the same bits."""
import numpy as np
import pytest
import torch

from ff_util import ACTS, DTYPES, Placed
from paper_2006_11735_amd import binding as B
from test_gpu_feed_forward_grouped import run

pytestmark = pytest.mark.gpu


@pytest.fixture
def kernel():
    yield lambda k: B.icnn_set_tuning("ff_kernel", k)
    B.icnn_set_tuning("reset")


# whole tiles, their halves and eighths, rests of both sizes and their quarters, one way or another (see mixed_tile in csrc/ffn_plan.h)
SHARES = {"mixed": [600, 40, 100, 256, 129], "rests": [256, 257, 300, 0, 129, 128, 65, 64, 1], "popular": [3000, 100, 30, 70], "even": [300] * 20}
FULL = {"rests": [300] * 140, "most": [256] * 100 + [200] * 28, "beyond": [256] * 120 + [300, 330, 400, 511, 512, 513], "halves": [356, 296, 256] * 20, "two": [256 * 64, 256 * 64 + 100, 40]}


@pytest.mark.parametrize("share", ["mixed", "rests", "popular"])
@pytest.mark.parametrize("k", [3969, 4001, 4008, 4100, 4230, 4360])      # 32 steps of k, 33, 34 and 35: copies four, two and one step ahead, with steps left over
@pytest.mark.parametrize("n", [300, 1100])
def test_deep_products_through_registers(kernel, share, k, n):
    kernel(10)
    counts = SHARES[share]
    g = np.random.default_rng(k)
    run(counts, k, n, "f32", seed=1)
    run(counts, k, n, "bf16", "gelu", index=g.integers(-1, 500, size=sum(counts) + 5), x_rows=500, behind=5, seed=2)


@pytest.mark.parametrize("pads,between,offset", [((1, 0, 0), 0, 0), ((0, 3, 1), 0, 0), ((0, 0, 0), 8, 0), ((0, 0, 0), 0, 4), ((4, 8, 12), 12, 5)])
@pytest.mark.parametrize("share", ["mixed", "rests"])
def test_deep_products_at_odd_places(kernel, pads, between, offset, share):
    kernel(10)
    counts = SHARES[share]
    rows = sum(counts)
    run(counts, 4000, 300, "f16", "relu", pads=pads, between=between, offset=offset, index=np.random.default_rng(1).permutation(rows), seed=3)


class Operands:
    """Random operands of positions of several experts, on the GPU"""

    def __init__(self, counts, k, n, x_rows, gated, dtype, pad, seed=0):
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        experts, rows = len(counts), sum(counts)
        number = lambda *shape: torch.randint(-127, 128, shape, generator=g, device="cuda:0", dtype=torch.int8)  # noqa: E731
        real = lambda *shape: torch.rand(shape, generator=g, device="cuda:0") + 0.5  # noqa: E731
        self.x, self.xs = number(x_rows, k + pad), real(x_rows) / 70
        self.layers = [(number(experts, n, k + pad), real(experts, n) / (70 * k ** 0.5), torch.randn((experts, n), generator=g, device="cuda:0")) for _ in range(1 + gated)]
        self.index = torch.randint(-2, x_rows + 2, (rows,), generator=g, device="cuda:0", dtype=torch.int32)
        self.offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(counts).cumsum(0)]).to(device="cuda:0", dtype=torch.int32)
        self.kw = dict(rows=rows, x_rows=x_rows, k=k, n=n, experts=experts, x_stride=k + pad, w_stride=k + pad, dtype=DTYPES[dtype][1])
        self.y = torch.zeros((rows, n), dtype=DTYPES[dtype][0], device="cuda:0")

    def run(self, act):
        d = B.grouped_desc(act=ACTS.index(act), **self.kw)
        call = B.igrouped_gated_linear_s8 if len(self.layers) == 2 else B.igrouped_linear_s8
        self.y.fill_(7)
        call(d, self.x, self.xs, self.index, self.offsets, *[t for layer in self.layers for t in layer], self.y)
        torch.cuda.synchronize()
        return self.y.view(torch.uint8).clone()


@pytest.mark.parametrize("counts", [[1, 0, 3, 2], [20, 3, 0, 17, 24], [130, 0, 257, 60, 9]])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("k,n,pad", [(384, 272, 0), (333, 111, 0), (4000, 300, 0), (4001, 137, 2)])
def test_all_kernels_give_the_same_bits(kernel, counts, dtype, gated, k, n, pad):
    o = Operands(counts, k, n, 90, gated, dtype, pad)
    for act in ACTS:
        kernel(1)
        want = o.run(act)
        for which in (0, *([2] if sum(counts) <= 64 else []), *range(3, 11)):
            kernel(which)
            assert torch.equal(o.run(act), want), (which, act)


@pytest.mark.parametrize("share", list(FULL))
@pytest.mark.parametrize("k,n", [(4000, 300), (4001, 520), (4230, 300)])
def test_full_turns_of_deep_tiles_give_the_same_bits(kernel, share, k, n):
    o = Operands(FULL[share], k, n, 3000, False, "f32", 0)
    kernel(9)
    want = o.run("silu")
    for which in (10, 3, 0):
        kernel(which)
        assert torch.equal(o.run("silu"), want), which


OFFSETS = [[0, 5, 3, 40], [-7, 10, 20, 990], [500, 400, 300, 20], [2 ** 31 - 1, -2 ** 31, 0, 700], [700] * 4, [0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [0, 2 ** 31 - 1] * 20 + [0],
           [0, 700, 1, 650, 2, 600, 600, 700], [-1] * 70 + [300, 100, 650, 10 ** 6]]


@pytest.mark.parametrize("which", [0, 1, 3, *range(4, 11)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("k", [128, 4000, 4001])
def test_offsets_that_are_none_write_no_other_memory(kernel, which, gated, k):
    kernel(which)
    rows, n, x_rows = 700, 300, 650
    X, Y = Placed(x_rows, k, torch.int8, values=torch.ones((x_rows, k))), Placed(rows, n, torch.float32)
    Y.view.fill_(-3)
    Y.snapshot()
    before = Y.view.clone()
    most = max(len(o) for o in OFFSETS)
    w, one = torch.ones((most, n, k), dtype=torch.int8, device="cuda:0"), torch.ones(most * n, device="cuda:0")
    index = torch.from_numpy(np.random.default_rng(k).integers(-3, x_rows + 3, size=rows).astype(np.int32)).to("cuda:0")
    value, named = k * k if gated else k, ((index >= 0) & (index < x_rows))
    for offsets in OFFSETS:
        Y.view.copy_(before)
        d = B.grouped_desc(rows=rows, x_rows=x_rows, k=k, n=n, experts=len(offsets) - 1, dtype=B.ICNN_F32)
        at = torch.tensor(offsets, device="cuda:0").to(torch.int32)
        layers = [w, one, None] * (1 + gated)
        (B.igrouped_gated_linear_s8 if gated else B.igrouped_linear_s8)(d, X, one, index, at, *layers, Y)
        torch.cuda.synchronize()
        assert Y.rest_untouched()
        same, full = (Y.view == -3).all(1), (Y.view == value).all(1)
        # (a row of which several experts' tiles have parts may be whole in pieces only)
        parts = ((Y.view == -3) | (Y.view == value)).all()
        assert parts and same[~named].all(), (offsets, int((~(same | full)).sum()))
