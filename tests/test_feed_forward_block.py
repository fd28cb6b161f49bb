"""What ffn.FeedForward prepares and issues, without a GPU: the library's own sizes and lists of calls, its launches stood in for."""
import pytest
import torch

from paper_2006_11735_amd import binding as B
from paper_2006_11735_amd import ffn

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="launches are stood in for")


@pytest.fixture
def events(monkeypatch):
    """What happens, in order: ("quantize", device), ("run", device, list of calls), ("wait", device)"""
    log, current = [], [None]

    class device:                                      # torch.cuda.device
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            self.before, current[0] = current[0], self.d

        def __exit__(self, *_):
            current[0] = self.before

    class Calls(B.Calls):
        def __init__(self, calls):
            self.calls = list(calls)
            super().__init__(self.calls)

        def run(self, stream=None):
            log.append(("run", current[0], self.calls))

    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda d=None: log.append(("wait", d)))
    monkeypatch.setattr(B, "iquantize_rows_s8", lambda d, x, q, scale, stream=None: log.append(("quantize", current[0])))
    monkeypatch.setattr(B, "Calls", Calls)
    return log


def block(width, hidden, rows, gated=True):
    z = torch.zeros
    return ffn.FeedForward(z(width), z(hidden, width), z(hidden, width) if gated else None, z(width, hidden), rows=rows, device="cpu")


def workspaces(ff, n):
    """(bytes that the two products of n rows ask for, the workspaces they are given)"""
    calls = [c for c in ff.calls(n) if c[0] in ("linear", "gated_linear")]
    sizes = [(B.igated_linear_s8_workspace_bytes if kind == "gated_linear" else B.ilinear_s8_workspace_bytes)(args[0]) for kind, args in calls]
    return sizes, [args[-1] for _, args in calls]


@pytest.mark.parametrize("width,hidden,gated", [(512, 16384, True), (1024, 8192, False), (512, 5461, True)])
def test_every_row_count_has_its_workspace(events, width, hidden, gated):
    ff = block(width, hidden, 700, gated)
    wanted = 0
    for n in range(1, 701):
        sizes, spaces = workspaces(ff, n)
        for size, space in zip(sizes, spaces):
            assert not size or (space is not None and space.numel() >= size), n
            wanted += size > 0
    assert wanted                                      # (there are such row counts)


def test_nothing_is_allocated_or_cleared_by_a_run(events, monkeypatch):
    """A run's stream need not be the one that clears; and what is cleared while a graph is captured is cleared only when it is replayed."""
    ff = block(512, 16384, 300)
    assert events[-1][0] == "wait"                     # what was cleared and quantised is there, for whichever stream
    kept = {n: workspaces(ff, n)[1][-1] for n in (64, 300)}
    assert all(t is not None and not t.any() for t in kept.values())
    ff = block(512, 16384, 300)

    def refuse(*_a, **_k):
        raise AssertionError("allocated")
    for name in ("zeros", "empty", "full"):
        monkeypatch.setattr(torch, name, refuse)
    for n in (0, 1, 64, 300, 64):
        ff.run(n, stream=7)
        assert events[-1][0] == "run"
    assert len({id(a[-1]) for e in events if e[0] == "run" for kind, a in e[2] if kind == "linear" and a[-1] is not None}) == 1


def test_everything_is_issued_on_the_block_s_device(events):
    """The stream that a call takes by itself is the current device's."""
    ff = block(64, 128, 8)
    ff.run(3)
    assert [e[:2] for e in events if e[0] != "wait"] == [("quantize", torch.device("cpu"))] * 3 + [("run", torch.device("cpu"))]


@pytest.mark.parametrize("name", ["columns", "transposed", "rows", "one row", "one column", "broadcast rows", "offset"])
def test_weights_are_quantised_from_their_own_numbers(events, monkeypatch, name):
    w = torch.arange(24.0 * 40).reshape(24, 40)
    w = {"columns": w[:, ::2], "transposed": w.t(), "rows": w[::3], "one row": w[3:4, ::4], "one column": w[:, 5:6], "broadcast rows": w[2].expand(6, 40),
         "offset": w[1:, 3:30]}[name]
    seen = []

    def quantise(d, x, q, scale, stream=None):
        seen.append(torch.as_strided(x, (d.rows, d.c), (d.x_stride, 1)).clone())
        assert d.x_stride >= d.c and q.shape == w.shape and q.stride() == (d.c, 1) and scale.shape == (d.rows,)
    monkeypatch.setattr(B, "iquantize_rows_s8", quantise)
    ffn.quantize_weights(w)
    assert torch.equal(seen[0], w)


def test_weights_of_other_types_or_dimensions_are_refused(events):
    for w in (torch.zeros(4, 4, dtype=torch.float64), torch.zeros(4, 4, dtype=torch.int8), torch.zeros(4), torch.zeros(2, 4, 4)):
        with pytest.raises(ValueError):
            ffn.quantize_weights(w)
