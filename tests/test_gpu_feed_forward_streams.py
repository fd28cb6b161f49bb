"""A new ffn.FeedForward whose first run splits k: on a stream that is not the one it was made on, and while a graph is captured."""
import pytest
import torch

from paper_2006_11735_amd import binding as B
from paper_2006_11735_amd.ffn import FeedForward

pytestmark = pytest.mark.gpu

WIDTH, HIDDEN, ROWS = 512, 16384, 64


def block():
    torch.full((1 << 27,), 0xFF, dtype=torch.uint8, device="cuda:0")      # (what the allocator hands out next holds no zeros)
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    ff = FeedForward(r(WIDTH).abs() + 0.5, r(HIDDEN, WIDTH) / 23, r(HIDDEN, WIDTH) / 23, r(WIDTH, HIDDEN) / 128, rows=ROWS)
    ff.stream.copy_(r(ROWS, WIDTH))
    ff.update.copy_(r(ROWS, WIDTH))
    torch.cuda.synchronize()
    assert any(B.ilinear_s8_workspace_bytes(B.linear_desc(rows=n, k=HIDDEN, n=WIDTH)) for n in (40, ROWS))
    return ff


def results(run):
    out = {}
    for n in (40, ROWS):
        ff = block()
        run(ff, n)
        torch.cuda.synchronize()
        out[n] = ff.stream.clone()
    return out


def test_the_first_run_on_another_stream():
    want = results(lambda ff, n: ff.run(n))
    side = torch.cuda.Stream()

    def on_side(ff, n):
        ff.run(n, stream=side)
    got = results(on_side)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_the_first_run_in_a_captured_graph():
    want = results(lambda ff, n: ff.run(n))
    for n in (40, ROWS):
        ff = block()
        start = ff.stream.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ff.run(n)
        for eager in (True, False, True, False, False):                   # an eager run before the first replay, and between replays
            ff.stream.copy_(start)
            ff.run(n) if eager else graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(ff.stream, want[n]), (n, eager)
