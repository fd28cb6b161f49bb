"""ilinear_s4, igated_linear_s4 and iquantize_weights_s4 on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from experts_util import gated_s4_64, linear_s4_64, packed4, quantize4
from ff_util import ACTS, DTYPES, Placed, to_numpy
from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu


def run(rows, k, n, group=128, dtype="bf16", act="none", *, gated=False, bias=True, residual=False, in_place=False, scales="f16", pads=(0, 0, 0), offset=0, seed=0,
        stream=None, junk=True):
    """pads: of the rows of x, residual and y; offset: elements in front of every tensor but the packed weights; junk: what is behind k in the last block is not zero"""
    g = np.random.default_rng(seed)
    torch_dtype, code = DTYPES[dtype]
    st, scode = DTYPES[scales]
    xv = g.integers(-128, 128, size=(rows, k)).astype(np.int8)
    xs = g.uniform(0.5, 1.5, size=rows).astype(np.float32) / 70
    vector = lambda v, t=torch.float32: None if v is None else Placed(1, v.numel(), t, None, offset, v.reshape(1, -1))  # noqa: E731
    layers, W, S, BI = [], [], [], []
    for _ in range(2 if gated else 1):
        w = g.integers(-8, 8, size=(n, k))
        s = torch.from_numpy(g.uniform(0.5, 1.5, size=(n, -(-k // group))) / (4.6 * k ** 0.5)).to(st)
        b = g.normal(size=n).astype(np.float32) if bias else None
        wide = np.zeros((n, -(-k // 32) * 32), int)
        wide[:, :k] = w
        if junk:
            wide[:, k:] = g.integers(-8, 8, size=(n, wide.shape[1] - k))
        p = torch.from_numpy(packed4(wide))
        layers.append((w, s.double().numpy(), b))
        W.append(Placed(1, p.numel(), torch.uint8, None, 0, p.reshape(1, -1)))
        S.append(vector(s, st)), BI.append(None if b is None else vector(torch.from_numpy(b)))
    rv = torch.from_numpy(g.normal(size=(rows, n))).to(torch_dtype) if residual else None
    X, XS = Placed(rows, k, torch.int8, k + pads[0], offset, torch.from_numpy(xv)), vector(torch.from_numpy(xs))
    R = Placed(rows, n, torch_dtype, n + pads[1], offset, rv) if residual else None
    Y = R if in_place else Placed(rows, n, torch_dtype, n + pads[2], offset)
    d = B.linear_s4_desc(rows=rows, k=k, n=n, group=group, act=ACTS.index(act), dtype=code, scale_dtype=scode, x_stride=X.stride, res_stride=R.stride if residual else n,
                         y_stride=Y.stride)
    tensors = [t for t in [X, XS, R, Y, *W, *S, *BI] if t is not None]
    for t in tensors:
        t.snapshot()
    torch.cuda.synchronize()
    if gated:
        B.igated_linear_s4(d, X, XS, W[0], S[0], BI[0], W[1], S[1], BI[1], Y, stream=stream)
    else:
        B.ilinear_s4(d, X, XS, W[0], S[0], BI[0], R, Y, stream=stream)
    torch.cuda.synchronize()
    assert all(t.rest_untouched() for t in tensors) and all((t.raw == t.before).all() for t in tensors if t is not Y)
    if gated:
        want, tol = gated_s4_64(xv, xs, *layers, act, group, dtype)
    else:
        want, tol = linear_s4_64(xv, xs, layers[0], act, None if rv is None else to_numpy(rv), group, dtype)
    off = np.abs(to_numpy(Y.view) - want) - tol
    assert (off <= 0).all(), (float(off.max()), np.unravel_index(np.argmax(off), off.shape))


ROWS = [1, 2, 3, 4, 5, 7, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 128, 129, 200, 257]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
def test_row_counts(rows, gated, group):
    run(rows, 512, 192, group, "f32", "silu" if gated else "none", gated=gated, residual=not gated, seed=rows)
    run(rows, 1001, 101, group, "f32", "silu" if gated else "none", gated=gated, residual=not gated, seed=rows)


@pytest.mark.parametrize("k", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 80, 127, 128, 130, 255, 256, 257, 272, 384, 511, 1001, 2001, 2048, 4064, 4100, 5000])
@pytest.mark.parametrize("rows,n", [(1, 33), (20, 50), (40, 70), (130, 140)])
def test_depths(k, rows, n):
    for group in (32, 64, 128, 256):
        run(rows, k, n, group, "f32", seed=k, scales="f32")
    run(rows, k, n, 128, "f32", "silu", gated=True, seed=k, scales="bf16")


@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 64, 127, 128, 129, 255, 257, 1000])
@pytest.mark.parametrize("rows,k", [(1, 512), (20, 256), (90, 256), (260, 128)])
def test_widths(n, rows, k):
    run(rows, k, n, 64, "f16", residual=True, seed=n)
    run(rows, k, n, 32, "f16", "gelu_tanh", gated=True, seed=n)
    run(rows, k, n, 128, "bf16", "gelu_tanh", gated=True, seed=n)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scales", list(DTYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [1, 37, 300])
def test_types_and_activations(dtype, scales, act, rows):
    run(rows, 384, 272, 128, dtype, act, scales=scales, residual=True, seed=1)
    run(rows, 384, 272, 64, dtype, act, scales=scales, bias=False, gated=True, seed=4)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pads,offset", [((16, 8, 24), 0), ((16, 16, 16), 16), ((0, 0, 0), 1), ((1, 5, 7), 5), ((16, 1, 0), 0), ((8, 8, 8), 8), ((4, 4, 4), 4)])
@pytest.mark.parametrize("rows,k,n", [(1, 320, 144), (29, 320, 144), (140, 640, 272), (140, 333, 111)])
def test_strides_and_offsets(dtype, pads, offset, rows, k, n):
    run(rows, k, n, 64, dtype, "gelu", residual=True, pads=pads, offset=offset, seed=7)
    run(rows, k, n, 128, dtype, "silu", gated=True, pads=pads, offset=offset, seed=8)


@pytest.mark.parametrize("rows", [1, 20, 150])
def test_residual_in_place(rows):
    run(rows, 512, 256, residual=True, in_place=True, pads=(0, 16, 16))


@pytest.mark.parametrize("rows,k,n,gated,group", [(1, 16384, 512, False, 128), (1, 16384, 256, False, 32), (2, 32768, 64, False, 64), (3, 8192, 1024, True, 128), (1, 40000, 40, True, 256),
                                                  (16, 12288, 96, False, 64), (64, 16384, 128, False, 32), (300, 8192, 256, True, 128), (512, 1024, 2048, False, 128),
                                                  (777, 512, 1111, True, 256), (1024, 2048, 1024, False, 32)])
def test_larger_products(rows, k, n, gated, group):
    run(rows, k, n, group, "bf16", "silu" if gated else "none", gated=gated, residual=not gated, seed=5)


@pytest.mark.parametrize("rows", [1, 3, 20, 100])
@pytest.mark.parametrize("group", [32, 256])
def test_the_largest_sums(rows, group):
    """Every product -128 * -8: the group's sum, sixteen times over, is 2^22"""
    k, n = 131071, 5
    x = torch.full((rows, k), -128, dtype=torch.int8, device="cuda:0")
    w = torch.full((n, -(-k // 32) * 16), 0x88, dtype=torch.uint8, device="cuda:0")
    scale, one, y = torch.ones((n, -(-k // group)), dtype=torch.float16, device="cuda:0"), torch.ones(rows, device="cuda:0"), torch.zeros((rows, n), device="cuda:0")
    B.ilinear_s4(B.linear_s4_desc(rows=rows, k=k, n=n, group=group, dtype=B.ICNN_F32), x, one, w, scale, None, None, y)
    torch.cuda.synchronize()
    assert (y.double() / (k * 1024.0) - 1).abs().max() <= (4096 + 4) * 2.0 ** -24


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_scales_that_are_nan_or_infinite_and_rows_of_zeros(rows):
    k, n, group = 512, 40, 128
    x = torch.zeros((rows, k), dtype=torch.int8, device="cuda:0")
    x[0] = 1
    w = torch.full((n, k // 2), 0x11, dtype=torch.uint8, device="cuda:0")
    scale = torch.ones((n, k // group), dtype=torch.float32, device="cuda:0")
    scale[3, 1], scale[5, 0] = float("nan"), float("inf")
    xs, y = torch.ones(rows, device="cuda:0"), torch.zeros((rows, n), device="cuda:0")
    d = B.linear_s4_desc(rows=rows, k=k, n=n, group=group, dtype=B.ICNN_F32, scale_dtype=B.ICNN_F32)
    B.ilinear_s4(d, x, xs, w, scale, None, None, y)
    torch.cuda.synchronize()
    assert y[:, 3].isnan().all() and y[0, 5] == float("inf") and y[1:, 5].isnan().all()
    rest = [i for i in range(n) if i not in (3, 5)]
    assert (y[0, rest] == k).all() and (y[1:, rest] == 0).all()


def test_no_rows_is_a_call_that_does_nothing():
    d = B.linear_s4_desc(rows=0, k=64, n=32)
    B.ilinear_s4(d, *[None] * 7)
    B.igated_linear_s4(d, *[None] * 9)


@pytest.mark.parametrize("rows", [3, 20, 300])
def test_rows_beyond_32_bits(rows):
    k, n, group, stride = 256, 128, 64, ((1 << 32) // (rows - 1) + 4096) // 4096 * 4096
    g = np.random.default_rng(3)
    x = torch.empty((rows - 1) * stride + k, dtype=torch.int8, device="cuda:0")
    y = torch.empty((rows - 1) * stride + n, dtype=torch.float16, device="cuda:0")
    xv, wv = g.integers(-127, 128, size=(rows, k)).astype(np.int8), g.integers(-8, 8, size=(n, k))
    x.as_strided((rows, k), (stride, 1)).copy_(torch.from_numpy(xv))
    xs, s = g.uniform(0.5, 1.5, size=rows).astype(np.float32) / 70, g.uniform(0.5, 1.5, size=(n, k // group)).astype(np.float32) / 70
    dev = lambda v: torch.from_numpy(v).to("cuda:0")  # noqa: E731
    XS, W, S = dev(xs), dev(packed4(wv)), dev(s)
    B.ilinear_s4(B.linear_s4_desc(rows=rows, k=k, n=n, group=group, x_stride=stride, y_stride=stride, dtype=B.ICNN_F16, scale_dtype=B.ICNN_F32), x, XS, W, S, None, None, y)
    torch.cuda.synchronize()
    want, tol = linear_s4_64(xv, xs, (wv, s, None), "none", None, group, "f16")
    assert (np.abs(to_numpy(y.as_strided((rows, n), (stride, 1))) - want) <= tol).all()


@pytest.mark.parametrize("rows", [1, 20, 150])
def test_on_another_stream_and_replayed(rows):
    run(rows, 512, 256, gated=True, stream=torch.cuda.Stream())
    k, n = 1024, 320
    g = torch.Generator(device="cuda:0").manual_seed(rows)
    x = torch.randint(-127, 128, (rows, k), generator=g, device="cuda:0", dtype=torch.int8)
    w = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda:0", dtype=torch.uint8)
    s, xs = torch.rand((n, k // 128), generator=g, device="cuda:0").half(), torch.rand(rows, generator=g, device="cuda:0")
    y = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda:0")
    calls = B.Calls([("linear_s4", (B.linear_s4_desc(rows=rows, k=k, n=n), x, xs, w, s, None, None, y))])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls.run()
    for i in range(4):
        x.random_(-127, 128, generator=g)
        calls.run()
        torch.cuda.synchronize()
        want = y.clone()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


@pytest.fixture
def kernel():
    yield lambda k: B.icnn_set_tuning("ff_kernel", k)
    B.icnn_set_tuning("reset")


@pytest.mark.parametrize("which,rows", [(1, 1), (1, 50), (2, 1), (2, 2), (2, 3), (2, 4), (3, 1), (3, 16), (3, 17), (3, 32)] +
                         [(k, m) for k in (4, 5, 6, 7) for m in (1, 31, 32, 33, 63, 64, 65, 130, 300)])
@pytest.mark.parametrize("k,n", [(16, 16), (64, 7), (300, 96), (512, 260), (1040, 129), (2320, 520)])
def test_every_kernel(kernel, which, rows, k, n):
    kernel(which)
    for dtype, pads, offset, group, scales in (("bf16", (0, 0, 0), 0, 128, "f16"), ("f32", (16, 4, 8), 0, 64, "f32"), ("f16", (1, 3, 4), 3, 256, "bf16"), ("f32", (0, 0, 0), 0, 32, "f16")):
        run(rows, k, n, group, dtype, "gelu", residual=True, pads=pads, offset=offset, scales=scales, seed=which)
        run(rows, k, n, group, dtype, "silu", gated=True, pads=pads, offset=offset, scales=scales, seed=which + 10)


@pytest.mark.parametrize("rows,which", [(2 ** 29, 0), (2 ** 29 - 3, 7)])
def test_as_many_rows_as_there_may_be(kernel, rows, which):
    """Whatever tiles one launch does not hold, another kernel has the product"""
    kernel(which)
    k, n, some = 16, 5, 70
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.ones((rows, k), dtype=torch.int8, device="cuda:0")
    x[-some:] = torch.randint(-128, 128, (some, k), generator=g, device="cuda:0").to(torch.int8)
    numbers = np.random.default_rng(3).integers(-8, 8, size=(n, k))
    w = torch.from_numpy(packed4(numbers)).to("cuda:0")
    scale, xs, y = torch.ones((n, 1), dtype=torch.float16, device="cuda:0"), torch.ones(rows, device="cuda:0"), torch.zeros((rows, n), device="cuda:0")
    B.ilinear_s4(B.linear_s4_desc(rows=rows, k=k, n=n, group=32, dtype=B.ICNN_F32), x, xs, w, scale, None, None, y)
    torch.cuda.synchronize()
    want = torch.from_numpy(numbers).double()
    assert (y[-some:].double().cpu() == x[-some:].double().cpu() @ want.T).all()           # (integers below 2^24)
    assert (y[:-some] == want.sum(1).float().to("cuda:0")).all()


@pytest.mark.parametrize("k", [2047, 2048, 2049, 4095, 4096, 4111, 8192, 8208, 16384, 16399, 32767, 32768, 32780])
def test_depths_of_single_tokens(k):
    for rows in (1, 2, 4):
        run(rows, k, 21, 128, "f32", residual=True, seed=k)
        run(rows, k, 5, 32, "bf16", "silu", gated=True, seed=k)


# ---- weights to 4 bits

@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scales", list(DTYPES))
def test_quantized_weights(group, dtype, scales):
    for n, k, pad, offset in ((1, 1, 0, 0), (3, 31, 0, 1), (5, 33, 3, 0), (40, 256, 0, 0), (17, 1001, 7, 3), (64, 640, 0, 8)):
        g = np.random.default_rng(n + k)
        td, code = DTYPES[dtype]
        st, scode = DTYPES[scales]
        w = Placed(n, k, td, k + pad, offset, torch.from_numpy(g.normal(size=(n, k))).to(td))
        p, s = Placed(1, B.iweights_s4_bytes(n, k), torch.uint8), Placed(n, -(-k // group), st, None, offset)
        for t in (w, p, s):
            t.snapshot()
        B.iquantize_weights_s4(B.quantize_s4_desc(n=n, k=k, group=group, dtype=code, scale_dtype=scode, w_stride=k + pad), w, p, s)
        torch.cuda.synchronize()
        assert all(t.rest_untouched() for t in (w, p, s)) and (w.raw == w.before).all()
        wv, got = to_numpy(w.view), to_numpy(s.view)
        _, want = quantize4(wv, group, lambda v: torch.from_numpy(v.astype(np.float32)).to(st).double().numpy())
        rel = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}[scales]       # (the quotient's rounding may move the scale's by one of its steps)
        assert (np.abs(got - want) <= rel * want).all()
        half = to_numpy(p.view).reshape(n, -1, 16)
        q = np.concatenate([half & 15, half >> 4], 2).reshape(n, -1)[:, :k].astype(int)
        q = np.where(q > 7, q - 16, q)
        wide = np.repeat(got, group, 1)[:, :k]
        assert np.abs(q).max() <= 7 and (np.abs(q - np.clip(wv / wide, -7, 7)) <= 0.5 + 8 * 2.0 ** -24).all()


def test_groups_of_zeros_nan_and_infinity():
    w = torch.zeros((6, 100), device="cuda:0")
    w[1, 40], w[2, 3], w[3, 64], w[4, :] = float("nan"), float("inf"), 1e6, 1e-9
    w[5, 0], w[5, 1], w[5, 2] = 7.0, 0.5, 1.5
    p, s = torch.full((6, 64), 0xEE, dtype=torch.uint8, device="cuda:0"), torch.zeros((6, 4), dtype=torch.float16, device="cuda:0")
    B.iquantize_weights_s4(B.quantize_s4_desc(n=6, k=100, group=32), w, p, s)
    torch.cuda.synchronize()
    assert (s[0] == 0).all() and s[1].isnan().tolist() == [False, True, False, False] and s[2].isnan().tolist() == [True, False, False, False]
    assert s[3].isnan().tolist() == [False, False, True, False] and (s[4] == 0).all()           # (1e6 / 7 leaves float16 upwards, 1e-9 / 7 downwards)
    assert s[5].tolist() == [1.0, 0.0, 0.0, 0.0] and p[5, :3].tolist() == [7, 0, 2]              # ties to even
    assert not p[:5].any()
