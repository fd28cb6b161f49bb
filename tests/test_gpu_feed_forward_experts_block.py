"""Blocks with experts (ffn.ExpertsFeedForward) and with 4-bit weights (ffn.FeedForward, bits=4): their calls in a row, each against the definition in 64 bits on what the one
before has left."""
import numpy as np
import pytest
import torch

from experts_util import combine64, gated_s4_64, linear_s4_64, route64
from ff_util import DTYPES, gated64, linear64, rows64, to_numpy
from paper_2006_11735_amd import binding as B
from paper_2006_11735_amd.ffn import ExpertsFeedForward, FeedForward
from test_gpu_feed_forward_block import check_rows

pytestmark = pytest.mark.gpu


def experts_block(rows, width, hidden, experts, top, dtype="bf16", act="silu", gated=True, bias=False, seed=0, **kw):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    ff = ExpertsFeedForward(r(width).abs() + 0.5, r(experts, width) / width ** 0.5, r(experts, hidden, width) / width ** 0.5,
                            r(experts, hidden, width) / width ** 0.5 if gated else None, r(experts, width, hidden) / hidden ** 0.5, rows=rows, top=top, act=act,
                            b_router=r(experts) if bias else None, b_gate=r(experts, hidden) if bias else None, b_up=r(experts, hidden) if bias and gated else None,
                            b_down=r(experts, width) if bias else None, dtype=DTYPES[dtype][0], **kw)
    ff.stream.copy_(r(rows, width))
    ff.update.copy_(r(rows, width))
    return ff


@pytest.mark.parametrize("rows,width,hidden,experts,top,dtype,act,gated,bias,score,normalise", [
    (1, 512, 768, 8, 2, "bf16", "silu", True, False, "softmax", True), (3, 513, 301, 5, 3, "f16", "gelu_tanh", True, True, "sigmoid", True),
    (17, 256, 512, 16, 4, "bf16", "gelu", False, True, "softmax", False), (70, 640, 896, 6, 2, "f32", "silu", True, False, "sigmoid", False),
    (300, 512, 1024, 4, 1, "bf16", "relu", False, False, "softmax", True), (520, 384, 512, 64, 8, "f16", "silu", True, True, "softmax", True)])
def test_a_block_of_experts(rows, width, hidden, experts, top, dtype, act, gated, bias, score, normalise):
    ff = experts_block(rows, width, hidden, experts, top, dtype, act, gated, bias, rows, score=score, normalise=normalise, scale=1.5)
    torch_dtype = DTYPES[dtype][0]
    total = (ff.stream.float() + ff.update.float()).to(torch_dtype)
    ff.run()
    torch.cuda.synchronize()
    n = to_numpy
    q, qs, h, hs = n(ff.q), n(ff.q_scale), n(ff.h), n(ff.h_scale)
    u, want = rows64(n(total), n(ff.gamma), ff.eps)
    check_rows(q, qs, u, want, width)
    logits = n(ff.logits)
    y, tol = linear64(q, qs, n(ff.router[0]), n(ff.router[1]), None if ff.b_router is None else n(ff.b_router), "none", None, "f32")
    assert (np.abs(logits - y) <= tol).all()
    expert, gate, place, token, offsets, rel = route64(logits, top, score, normalise, 1.5)
    for got, want in ((ff.expert, expert), (ff.place, place), (ff.token, token), (ff.offsets, offsets)):
        assert (n(got) == want).all()
    assert (np.abs(n(ff.gate) - gate) <= rel * np.abs(gate)).all()
    (wg, sg), second, (wd, sd) = [None if w is None else tuple(n(t) for t in w) for w in ff.weights]
    bg, bu, bd = [None if b is None else n(b) for b in ff.biases]
    at = lambda t, e: None if t is None else t[e]  # noqa: E731
    middle, v = n(ff.middle), n(ff.v)
    for e in range(experts):
        rows_of = slice(offsets[e], offsets[e + 1])
        x, xs = q[token[rows_of]], qs[token[rows_of]]
        if gated:
            y, tol = gated64(x, xs, wg[e], sg[e], at(bg, e), second[0][e], second[1][e], at(bu, e), act, dtype)
        else:
            y, tol = linear64(x, xs, wg[e], sg[e], at(bg, e), act, None, dtype)
        assert (np.abs(middle[rows_of] - y) <= tol).all()
        y, tol = linear64(h[rows_of], hs[rows_of], wd[e], sd[e], at(bd, e), "none", None, dtype)
        assert (np.abs(v[rows_of] - y) <= tol).all()
    u, want = rows64(middle, None, 0)
    check_rows(h, hs, u, want, hidden)
    y, tol = combine64(v, n(ff.gate), place, n(total), dtype)
    assert (np.abs(n(ff.stream) - y) <= tol).all()


def test_fewer_rows_leave_the_others_alone_and_row_counts_agree():
    ff = experts_block(200, 512, 512, 8, 2, seed=5)
    start = ff.stream.clone()
    ff.run(0)
    torch.cuda.synchronize()
    assert torch.equal(ff.stream, start)
    outs = {}
    for n in (1, 4, 17, 33, 64, 65, 200):
        ff.stream.copy_(start)
        ff.run(n)
        torch.cuda.synchronize()
        assert torch.equal(ff.stream[n:], start[n:])
        outs[n] = ff.stream[:n].clone()
    for n in outs:
        assert torch.equal(outs[n], outs[200][:n]), n          # whichever kernels take them
    with pytest.raises(ValueError):
        ff.run(201)


FUNCTIONS = {"rms_norm": B.irms_norm_s8, "linear": B.ilinear_s8, "route": B.iroute_top, "grouped_gated_linear": B.igrouped_gated_linear_s8, "quantize_rows": B.iquantize_rows_s8,
             "grouped_linear": B.igrouped_linear_s8, "combine": B.icombine_rows, "gated_linear_s4": B.igated_linear_s4, "linear_s4": B.ilinear_s4}


def blocks():
    yield experts_block(48, 512, 1024, 8, 2, bias=True, seed=6)
    yield four_bits(24, 1024, 2048, bias=True, seed=6)


def test_blocks_as_calls_as_a_list_on_another_stream_and_replayed():
    for ff in blocks():
        start = ff.stream.clone()
        for kind, args in ff.calls(ff.rows):
            FUNCTIONS[kind](*args)
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
            ff.stream.copy_(start * (1 + k) + 0.1 * k * ff.update)
            before = ff.stream.clone()
            ff.run()
            torch.cuda.synchronize()
            eager = ff.stream.clone()
            ff.stream.copy_(before)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(ff.stream, eager), k


def test_two_captured_blocks_side_by_side():
    """Each has workspaces of its own: graphs that run at the same time do not meet."""
    ffs = [experts_block(400, 512, 512, 32, 4, seed=s) for s in (1, 2)]
    starts, wants, graphs = [ff.stream.clone() for ff in ffs], [], []
    for ff, start in zip(ffs, starts):
        ff.run()
        torch.cuda.synchronize()
        wants.append(ff.stream.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ff.run()
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in ffs]
    for _ in range(5):
        for ff, start in zip(ffs, starts):
            ff.stream.copy_(start)
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(ff.stream, want) for ff, want in zip(ffs, wants))


def test_a_row_with_a_nan_stays_by_itself():
    ff = experts_block(6, 512, 256, 8, 2, "f32", seed=7)
    ff.update[2, 100] = float("nan")
    ff.run()
    torch.cuda.synchronize()
    bad = ff.stream.isnan().any(1).tolist()
    assert bad == [False, False, True, False, False, False] and ff.stream[2].isnan().all()


# ---- weights of 4 bits

def four_bits(rows, width, hidden, dtype="bf16", act="silu", gated=True, bias=False, group=128, scales=torch.float16, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    ff = FeedForward(r(width).abs() + 0.5, r(hidden, width) / width ** 0.5, r(hidden, width) / width ** 0.5 if gated else None, r(width, hidden) / hidden ** 0.5,
                     rows=rows, act=act, b_gate=r(hidden) if bias else None, b_up=r(hidden) if bias and gated else None, b_down=r(width) if bias else None,
                     dtype=DTYPES[dtype][0], bits=4, group=group, scale_dtype=scales)
    ff.stream.copy_(r(rows, width))
    ff.update.copy_(r(rows, width))
    return ff


def unpacked(packed, n, k):
    half = to_numpy(packed).reshape(n, -1, 16).astype(int)
    q = np.concatenate([half & 15, half >> 4], 2).reshape(n, -1)[:, :k]
    return np.where(q > 7, q - 16, q)


@pytest.mark.parametrize("rows,width,hidden,dtype,act,gated,bias,group,scales", [
    (1, 512, 1536, "bf16", "silu", True, False, 128, torch.float16), (3, 513, 1001, "f16", "gelu_tanh", True, True, 32, torch.float32),
    (17, 1024, 2048, "bf16", "gelu", False, True, 64, torch.bfloat16), (70, 640, 1792, "f32", "silu", True, False, 256, torch.float16),
    (300, 1024, 4096, "bf16", "relu", False, False, 128, torch.float16)])
def test_a_block_of_4_bits(rows, width, hidden, dtype, act, gated, bias, group, scales):
    ff = four_bits(rows, width, hidden, dtype, act, gated, bias, group, scales, rows)
    total = (ff.stream.float() + ff.update.float()).to(DTYPES[dtype][0])
    ff.run()
    torch.cuda.synchronize()
    n = to_numpy
    q, qs, h, hs = n(ff.q), n(ff.q_scale), n(ff.h), n(ff.h_scale)
    u, want = rows64(n(total), n(ff.gamma), ff.eps)
    check_rows(q, qs, u, want, width)
    bg, bu, bd = [None if b is None else n(b) for b in ff.biases]
    wg, wu, wd = [None if w is None else (unpacked(w[0], *shape), n(w[1]), b)
                  for w, shape, b in zip(ff.weights, ((hidden, width), (hidden, width), (width, hidden)), (bg, bu, bd))]
    y, tol = gated_s4_64(q, qs, wg, wu, act, group, dtype) if gated else linear_s4_64(q, qs, wg, act, None, group, dtype)
    assert (np.abs(n(ff.middle) - y) <= tol).all()
    u, want = rows64(n(ff.middle), None, 0)
    check_rows(h, hs, u, want, hidden)
    y, tol = linear_s4_64(h, hs, wd, "none", n(total), group, dtype)
    assert (np.abs(n(ff.stream) - y) <= tol).all()


def test_fewer_rows_of_4_bits():
    ff = four_bits(40, 512, 1024, seed=5)
    start = ff.stream.clone()
    for n in (0, 1, 7, 40):
        ff.stream.copy_(start)
        ff.run(n)
        torch.cuda.synchronize()
        assert torch.equal(ff.stream[n:], start[n:])
