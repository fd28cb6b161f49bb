"""The feed-forward half of a block (ffn.FeedForward): its calls in a row, each against the definition in 64 bits on what the one before has left."""
import numpy as np
import pytest
import torch

from ff_util import DTYPES, gated64, linear64, rows64, to_numpy
from paper_2006_11735_amd import binding as B
from paper_2006_11735_amd.ffn import FeedForward, quantize_weights

pytestmark = pytest.mark.gpu


def block(rows, width, hidden, dtype, act, gated, bias, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    ff = FeedForward(r(width).abs() + 0.5, r(hidden, width) / width ** 0.5, r(hidden, width) / width ** 0.5 if gated else None, r(width, hidden) / hidden ** 0.5,
                     rows=rows, act=act, b_gate=r(hidden) if bias else None, b_up=r(hidden) if bias and gated else None, b_down=r(width) if bias else None,
                     dtype=DTYPES[dtype][0])
    ff.stream.copy_(r(rows, width))
    ff.update.copy_(r(rows, width))
    return ff


def check_rows(q, scale, u, want, c):
    tol = (c / 64 + 16) * 2.0 ** -25 + 5 * 2.0 ** -24
    assert (np.abs(scale - want) <= tol * want).all()
    assert (np.abs(q - u / want[:, None]) <= 0.5 + 127 * 5 * 2.0 ** -24).all()


@pytest.mark.parametrize("rows,width,hidden,dtype,act,gated,bias", [(1, 512, 1536, "bf16", "silu", True, False), (3, 513, 1001, "f16", "gelu_tanh", True, True),
                                                                    (17, 1024, 2048, "bf16", "gelu", False, True), (70, 640, 1792, "f32", "silu", True, False),
                                                                    (300, 1024, 4096, "bf16", "relu", False, False), (520, 768, 2048, "f16", "silu", True, True)])
def test_a_block(rows, width, hidden, dtype, act, gated, bias):
    ff = block(rows, width, hidden, dtype, act, gated, bias, rows)
    torch_dtype = DTYPES[dtype][0]
    total = (ff.stream.float() + ff.update.float()).to(torch_dtype)
    ff.run()
    torch.cuda.synchronize()
    n = to_numpy
    q, qs, h, hs = n(ff.q), n(ff.q_scale), n(ff.h), n(ff.h_scale)
    u, want = rows64(n(total), n(ff.gamma), ff.eps)
    check_rows(q, qs, u, want, width)
    (wg, sg), second, (wd, sd) = [None if w is None else tuple(n(t) for t in w) for w in ff.weights]
    bg, bu, bd = [None if b is None else n(b) for b in ff.biases]
    middle = n(ff.middle)
    if gated:
        y, tol = gated64(q, qs, wg, sg, bg, *second, bu, act, dtype)
    else:
        y, tol = linear64(q, qs, wg, sg, bg, act, None, dtype)
    assert (np.abs(middle - y) <= tol).all()
    u, want = rows64(middle, None, 0)
    check_rows(h, hs, u, want, hidden)
    y, tol = linear64(h, hs, wd, sd, bd, "none", n(total), dtype)
    assert (np.abs(n(ff.stream) - y) <= tol).all()


def test_weights_take_the_paper_s_step():
    w = torch.randn((40, 100), generator=torch.Generator().manual_seed(1)).cuda()
    q, step = quantize_weights(w)
    torch.cuda.synchronize()
    assert torch.allclose(step, w.abs().amax(1) / 127, rtol=1e-6) and (q.abs().amax(1) == 127).all()
    assert ((q * step[:, None] - w).abs() <= 0.5001 * step[:, None]).all()


def test_fewer_rows_leave_the_others_alone_and_row_counts_agree():
    ff = block(40, 512, 1024, "bf16", "silu", True, False, 5)
    start = ff.stream.clone()
    ff.run(0)
    torch.cuda.synchronize()
    assert torch.equal(ff.stream, start)
    outs = {}
    for n in (1, 4, 17, 40):
        ff.stream.copy_(start)
        ff.run(n)
        torch.cuda.synchronize()
        assert torch.equal(ff.stream[n:], start[n:])
        outs[n] = ff.stream[:n].clone()
    for n in (1, 4, 17):
        assert torch.equal(outs[n], outs[40][:n])              # whichever kernels take them
    with pytest.raises(ValueError):
        ff.run(41)


def test_a_block_as_calls_as_a_list_on_another_stream_and_replayed():
    ff = block(24, 1024, 4096, "bf16", "silu", True, True, 6)
    start = ff.stream.clone()
    functions = {"rms_norm": B.irms_norm_s8, "gated_linear": B.igated_linear_s8, "quantize_rows": B.iquantize_rows_s8, "linear": B.ilinear_s8}
    for kind, args in ff.calls(24):
        functions[kind](*args)
    torch.cuda.synchronize()
    want = ff.stream.clone()
    side = torch.cuda.Stream()
    for stream in (None, side):
        ff.stream.copy_(start)
        torch.cuda.synchronize()
        ff.run(stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(ff.stream, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ff.run()
    for k in range(4):
        ff.stream.copy_(start * (1 + k))
        ff.run()
        torch.cuda.synchronize()
        eager = ff.stream.clone()
        ff.stream.copy_(start * (1 + k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ff.stream, eager), k


def test_a_row_with_a_nan_stays_by_itself():
    ff = block(6, 512, 1024, "f32", "silu", True, False, 7)
    ff.update[2, 100] = float("nan")
    ff.run()
    torch.cuda.synchronize()
    bad = ff.stream.isnan().any(1).tolist()
    assert bad == [False, False, True, False, False, False] and ff.stream[2].isnan().all()
