"""iroute_top and icombine_rows on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from experts_util import combine64, route64
from ff_util import DTYPES, Placed, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu

OUTPUTS = ("expert", "gate", "place", "token", "offsets")


class Router:
    """An iroute_top call on logits of its own, its outputs in guarded buffers"""

    def __init__(self, logits, top, dtype="f32", score="softmax", normalise=False, scale=1.0, pad=0, offset=0):
        torch_dtype, code = DTYPES[dtype]
        self.rows, self.experts = logits.shape
        self.top, self.score, self.normalise, self.scale = top, score, normalise, scale
        self.logits = Placed(self.rows, self.experts, torch_dtype, self.experts + pad, offset, torch.from_numpy(logits).to(torch_dtype))
        self.d = B.route_desc(rows=self.rows, experts=self.experts, top=top, dtype=code, logits_stride=self.experts + pad, normalise=int(normalise), scale=scale,
                              score=B.ICNN_ROUTE_SOFTMAX if score == "softmax" else B.ICNN_ROUTE_SIGMOID)
        many = self.rows * top
        self.out = {k: Placed(1, n, torch.float32 if k == "gate" else torch.int32, n, offset)
                    for k, n in zip(OUTPUTS, (many, many, many, many, self.experts + 1))}
        size = B.iroute_top_workspace_bytes(self.d)
        self.ws = torch.full((size,), 0xEE, dtype=torch.uint8, device="cuda:0") if size else None

    def run(self, stream=None):
        B.iroute_top(self.d, self.logits, *self.out.values(), self.ws, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        return {k: to_numpy(p.view)[0] for k, p in self.out.items()}

    def check(self):
        got = self.results()
        assert all(p.rest_untouched() for p in self.out.values()) and (self.logits.raw == self.logits.before).all()
        expert, gate, place, token, offsets, rel = route64(to_numpy(self.logits.view), self.top, self.score, self.normalise, self.scale)
        for k, want in (("expert", expert), ("place", place), ("token", token), ("offsets", offsets)):
            assert (got[k] == want.reshape(-1)).all(), k
        g = got["gate"].reshape(gate.shape)
        assert (np.isnan(g) == np.isnan(gate)).all()
        off = np.abs(g - gate) - rel * np.abs(gate) - 2.0 ** -126 * max(1, abs(self.scale))
        assert not (off > 0).any(), float(np.nanmax(off))

    def go(self):
        for p in [*self.out.values(), self.logits]:
            p.snapshot()
        self.run()
        self.check()


def logits_of(rows, experts, seed, spread=1.5):
    return np.random.default_rng(seed).normal(size=(rows, experts)) * spread


@pytest.mark.parametrize("experts", [1, 2, 5, 15, 16, 17, 63, 64, 65, 100, 128, 129, 200, 256, 257, 300, 512, 513, 1000, 1024])
@pytest.mark.parametrize("rows", [1, 5, 33, 200])
def test_experts(experts, rows):
    for top in sorted({1, min(2, experts), min(8, experts), min(16, experts)}):
        Router(logits_of(rows, experts, experts + top), top, "f32", "softmax", top % 2 == 0).go()
        Router(logits_of(rows, experts, experts + top), top, "f16", "sigmoid", top % 2 == 1, 2.5).go()


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 500, 1000, 4097, 8192, 8193, 20011, 70001])
@pytest.mark.parametrize("experts,top", [(8, 2), (64, 6), (256, 8)])
def test_rows(rows, experts, top):
    Router(logits_of(rows, experts, rows), top, "bf16", "softmax", True).go()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [False, True])
def test_types_scores_strides(dtype, score, normalise):
    for pad, offset, rows in ((0, 0, 70), (3, 1, 70), (8, 8, 20), (1, 0, 300)):
        Router(logits_of(rows, 60, 3), 4, dtype, score, normalise, 1.25, pad, offset).go()
    Router(logits_of(90, 60, 4, 40.0), 5, dtype, score, normalise, -0.5).go()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("experts", [128, 256, 512, 1024])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (7, 3), (8, 8)])
def test_whole_lanes_of_experts_at_odd_places(dtype, experts, pad, offset):
    for rows in (5, 90):
        Router(logits_of(rows, experts, 7), 6, dtype, "softmax", False, 1.0, pad, offset).go()


def test_a_negative_stream_of_sigmoids_is_normalised_all_the_same():
    logits = logits_of(50, 40, 5) - 150                # each sigmoid leaves float32
    r = Router(logits, 3, "f32", "sigmoid", True)
    r.go()
    assert np.allclose(r.results()["gate"].reshape(50, 3).sum(1), 1, atol=1e-6)


@pytest.mark.parametrize("rows", [7, 100, 3000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_logits_go_to_the_lowest_index(rows, score):
    g = np.random.default_rng(rows)
    Router(g.integers(-1, 2, size=(rows, 64)).astype(float), 8, "bf16", score, True).go()
    Router(np.zeros((rows, 200)), 16, "f32", score, False).go()
    zeros = np.where(g.random((rows, 70)) < 0.5, -0.0, 0.0)
    Router(zeros, 5, "f16", score, False).go()


@pytest.mark.parametrize("rows", [9, 40, 1000])
@pytest.mark.parametrize("score,normalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_masked_experts_and_rows(rows, score, normalise):
    g = np.random.default_rng(rows)
    logits = logits_of(rows, 48, rows)
    logits[g.random((rows, 48)) < 0.9] = -np.inf       # some rows have fewer than six left
    logits[rows // 2] = -np.inf                        # one has none
    logits[:, 17] = -np.inf                            # and this expert nobody
    Router(logits, 6, "f32", score, normalise).go()
    Router(np.full((rows, 48), -np.inf), 6, "bf16", score, normalise).go()
    lowest = np.full((rows, 48), float(np.finfo(np.float32).min))
    lowest[:, 40] = 0
    Router(lowest, 3, "f32", score, normalise).go()


@pytest.mark.parametrize("score,normalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_nan_and_infinity(score, normalise):
    logits = logits_of(64, 33, 1)
    logits[3, 20] = np.nan
    logits[4, [2, 30]] = np.nan
    logits[5, 7] = np.inf
    logits[6, [7, 9]] = np.inf
    logits[7, :] = np.nan
    logits[8, :] = -np.inf
    logits[8, 11] = np.nan
    if score == "sigmoid":
        Router(logits, 4, "f32", score, normalise).go()
        return
    r = Router(logits, 4, "f32", score, normalise)
    r.go()
    expert = r.results()["expert"].reshape(64, 4)
    assert expert[3, 0] == 20 and list(expert[4, :2]) == [2, 30] and expert[5, 0] == 7 and list(expert[8]) == [11, -1, -1, -1]


def test_no_rows_leave_offsets_of_zeros():
    d = B.route_desc(rows=0, experts=40, top=2)
    offsets = torch.full((41,), 7, dtype=torch.int32, device="cuda:0")
    B.iroute_top(d, None, None, None, None, None, offsets)
    torch.cuda.synchronize()
    assert not offsets.any()


def test_rows_beyond_32_bits():
    rows, experts, stride = 40, 64, 1 << 27
    raw = torch.empty((rows - 1) * stride + experts, dtype=torch.bfloat16, device="cuda:0")
    logits = torch.from_numpy(logits_of(rows, experts, 2)).to(torch.bfloat16).cuda()
    raw.as_strided((rows, experts), (stride, 1)).copy_(logits)
    new = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device="cuda:0")  # noqa: E731
    outs = []
    for d, x in ((B.route_desc(rows=rows, experts=experts, top=2, dtype=B.ICNN_BF16, logits_stride=stride), raw),
                 (B.route_desc(rows=rows, experts=experts, top=2, dtype=B.ICNN_BF16), logits)):
        out = [new(80), new(80, torch.float32), new(80), new(80), new(65)]
        B.iroute_top(d, x, *out, new(B.iroute_top_workspace_bytes(d), torch.uint8))
        outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("rows", [20, 700])
def test_on_another_stream_and_replayed(rows):
    side = torch.cuda.Stream()
    r = Router(logits_of(rows, 128, 1), 4, "bf16", "softmax", True)
    for p in [*r.out.values(), r.logits]:
        p.snapshot()
    torch.cuda.synchronize()
    r.run(side)
    r.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.run()
    for k in range(4):
        r.logits.view.copy_(torch.from_numpy(logits_of(rows, 128, 10 + k)))
        r.logits.snapshot()
        if r.ws is not None:
            r.ws.fill_(0x5A)
        graph.replay()
        r.check()
        if k == 1:
            r.run()
            r.check()


# ---- sums of rows

def combine(rows, top, c, dtype="bf16", v_dtype=None, residual=True, in_place=False, pads=(0, 0, 0), offset=0, seed=0, place=None, v_rows=None):
    g = np.random.default_rng(seed)
    v_dtype = v_dtype or dtype
    many = rows * top if v_rows is None else v_rows
    td, tv = DTYPES[dtype][0], DTYPES[v_dtype][0]
    v = Placed(many, c, tv, c + pads[0], offset, torch.from_numpy(g.normal(size=(many, c))).to(tv))
    r = Placed(rows, c, td, c + pads[1], offset, torch.from_numpy(g.normal(size=(rows, c))).to(td)) if residual else None
    y = r if in_place else Placed(rows, c, td, c + pads[2], offset)
    gate = g.uniform(-1, 1, size=(rows, top)).astype(np.float32)
    place = g.permutation(many).reshape(rows, top) if place is None else place
    G = Placed(1, rows * top, torch.float32, None, offset, torch.from_numpy(gate.reshape(-1)))
    P = Placed(1, rows * top, torch.int32, None, offset, torch.from_numpy(place.reshape(-1)))
    tensors = [t for t in (v, r, y, G, P) if t is not None]
    vv, rr = to_numpy(v.view), None if r is None else to_numpy(r.view)
    for t in tensors:
        t.snapshot()
    d = B.combine_desc(rows=rows, top=top, c=c, v_rows=many, v_stride=v.stride, res_stride=r.stride if residual else c, y_stride=y.stride, dtype=DTYPES[dtype][1],
                       v_dtype=DTYPES[v_dtype][1])
    B.icombine_rows(d, v, G, P, r, y)
    torch.cuda.synchronize()
    assert all(t.rest_untouched() for t in tensors) and all((t.raw == t.before).all() for t in tensors if t is not y)
    want, tol = combine64(vv, gate, place, rr, dtype)
    assert (np.abs(to_numpy(y.view) - want) <= tol).all()


@pytest.mark.parametrize("c", [1, 2, 7, 8, 9, 63, 64, 100, 255, 256, 1000, 2047, 2048, 2049, 5000, 8192])
@pytest.mark.parametrize("rows,top", [(1, 1), (1, 8), (3, 2), (40, 4), (9, 16)])
def test_widths(c, rows, top):
    combine(rows, top, c, "f32", seed=c)
    combine(rows, top, c, "bf16", residual=False, seed=c)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("v_dtype", list(DTYPES))
@pytest.mark.parametrize("pads,offset", [((0, 0, 0), 0), ((8, 16, 24), 8), ((1, 3, 5), 1), ((0, 0, 0), 3)])
def test_types_and_strides(dtype, v_dtype, pads, offset):
    combine(21, 3, 264, dtype, v_dtype, pads=pads, offset=offset, seed=1)
    combine(21, 3, 77, dtype, v_dtype, in_place=True, pads=(pads[0], pads[1], pads[1]), offset=offset, seed=2)


def test_many_rows():
    combine(5000, 2, 96, "f16", seed=3)
    combine(700, 8, 1024, "bf16", seed=4)


def test_choices_without_a_place_add_nothing():
    g = np.random.default_rng(5)
    place = g.integers(-3, 60, size=(50, 5))           # -3 .. -1 and 40 .. 59 name no row
    place[7] = -1
    place[8] = 40
    place[9] = np.iinfo(np.int32).max
    place[10] = np.iinfo(np.int32).min
    place[11] = 6                                      # one row five times
    combine(50, 5, 136, "f32", place=place, v_rows=40)
    combine(50, 5, 136, "bf16", place=place, v_rows=40, residual=False)
    combine(4, 2, 40, "f32", place=np.full((4, 2), -1), v_rows=1)


def test_no_rows_of_v():
    res = torch.randn((3, 20), device="cuda:0")
    y = torch.zeros((3, 20), device="cuda:0")
    B.icombine_rows(B.combine_desc(rows=3, top=2, c=20, v_rows=0, dtype=B.ICNN_F32), None, torch.ones((3, 2), device="cuda:0"),
                    torch.zeros((3, 2), dtype=torch.int32, device="cuda:0"), res, y)
    torch.cuda.synchronize()
    assert torch.equal(y, res)


def test_a_gate_that_is_nan_and_rows_that_are_not_read():
    v = torch.full((6, 16), float("nan"), device="cuda:0")
    v[2] = 3.0
    gate = torch.tensor([[1.0, float("nan")], [float("nan"), 2.0]], device="cuda:0")
    place = torch.tensor([[2, -1], [2, 2]], dtype=torch.int32, device="cuda:0")
    y = torch.zeros((2, 16), device="cuda:0")
    B.icombine_rows(B.combine_desc(rows=2, top=2, c=16, v_rows=6, dtype=B.ICNN_F32), v, gate, place, None, y)
    torch.cuda.synchronize()
    assert (y[0] == 3).all() and y[1].isnan().all()


def test_rows_of_v_beyond_32_bits():
    stride, c = 1 << 28, 72
    v = torch.empty(17 * stride + c, dtype=torch.bfloat16, device="cuda:0")
    at = v.as_strided((18, c), (stride, 1))
    at.copy_(torch.arange(18, device="cuda:0")[:, None].expand(18, c))
    place = torch.tensor([[17, 3], [0, 16]], dtype=torch.int32, device="cuda:0")
    y = torch.zeros((2, c), dtype=torch.bfloat16, device="cuda:0")
    B.icombine_rows(B.combine_desc(rows=2, top=2, c=c, v_rows=18, v_stride=stride), v, torch.ones((2, 2), device="cuda:0"), place, None, y)
    torch.cuda.synchronize()
    assert (y[0] == 20).all() and (y[1] == 16).all()
