"""The feed-forward half of a transformer block in 8 bits, run through the C boundary:

    stream += update                                  (what the block's other half adds)
    q       = rms_norm(stream) * gamma, in 8 bits     irms_norm_s8
    hidden  = act(q Wgate) * (q Wup)                  igated_linear_s8      (without Wup: act(q Wgate), ilinear_s8)
    h       = hidden, in 8 bits                       iquantize_rows_s8
    stream += h Wdown                                 ilinear_s8

This is harness code, like netrun: it owns the device buffers, brings the weights to 8 bits once (a step per output channel, by the
library's own row quantisation) and issues the four calls as one list.  All arithmetic happens inside the library.

    python -m paper_2006_11735_amd.ffn --rows 1 16 512 4096 --width 4096 --hidden 16384

runs blocks of random weights and prints their times.
"""
import torch

from . import binding as B

_CODES = {torch.float32: B.ICNN_F32, torch.float16: B.ICNN_F16, torch.bfloat16: B.ICNN_BF16}
ACTS = {"none": B.ICNN_ACT_NONE, "relu": B.ICNN_ACT_RELU, "silu": B.ICNN_ACT_SILU, "gelu": B.ICNN_ACT_GELU, "gelu_tanh": B.ICNN_ACT_GELU_TANH}


def quantize_weights(w):
    """(int8 [n][k], float32 [n]) of floating weights on the GPU: per output channel the step max|w| / 127 (Section 3.1, Section 3.4.3)."""
    if w.dim() != 2 or w.dtype not in _CODES:
        raise ValueError("weights are [n][k] numbers of float32, float16 or bfloat16: got %s of %s" % (tuple(w.shape), w.dtype))
    n, k = w.shape
    if w.stride(1) != 1 or w.stride(0) < k:                    # (the library takes rows whose numbers lie next to each other, and no two rows in one place)
        w = w.contiguous()
    q, step = torch.empty((n, k), dtype=torch.int8, device=w.device), torch.empty(n, dtype=torch.float32, device=w.device)
    with torch.cuda.device(w.device):
        B.iquantize_rows_s8(B.norm_desc(rows=n, c=k, x_stride=w.stride(0), dtype=_CODES[w.dtype]), w, q, step)
    return q, step


class FeedForward:
    """`stream` and `update` are the [rows, width] buffers a program reads and writes; run(n) takes their first n rows through the block, in place."""

    def __init__(self, gamma, w_gate, w_up, w_down, *, rows, act="silu", b_gate=None, b_up=None, b_down=None, eps=1e-5, dtype=torch.bfloat16, device="cuda:0"):
        hidden, width = w_gate.shape
        if gamma.shape != (width,) or w_down.shape != (width, hidden) or (w_up is not None and w_up.shape != (hidden, width)):
            raise ValueError("gamma [width], w_gate and w_up [hidden, width], w_down [width, hidden]: got %s, %s, %s, %s" % (
                tuple(gamma.shape), tuple(w_gate.shape), None if w_up is None else tuple(w_up.shape), tuple(w_down.shape)))
        for name, b, n in (("b_gate", b_gate, hidden), ("b_up", b_up, hidden), ("b_down", b_down, width)):
            if b is not None and b.shape != (n,):
                raise ValueError("%s has shape %s, not (%d,)" % (name, tuple(b.shape), n))
        if b_up is not None and w_up is None:
            raise ValueError("b_up without w_up")
        if act not in ACTS or dtype not in _CODES or rows < 1:
            raise ValueError("act is one of %s, dtype float32, float16 or bfloat16, rows at least 1" % ", ".join(ACTS))
        if not torch.cuda.is_available():
            raise RuntimeError("FeedForward needs a GPU: there is no CPU fallback")
        self.rows, self.width, self.hidden, self.act, self.eps, self.dtype = rows, width, hidden, act, eps, dtype
        new = lambda shape, t: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        self.gamma = gamma.to(device=device, dtype=torch.float32).contiguous()
        self.weights = [None if w is None else quantize_weights(w.to(device).contiguous()) for w in (w_gate, w_up, w_down)]
        self.biases = [None if b is None else b.to(device=device, dtype=torch.float32).contiguous() for b in (b_gate, b_up, b_down)]
        self.stream, self.update = new((rows, width), dtype), new((rows, width), dtype)
        self.q, self.q_scale = new((rows, width), torch.int8), new(rows, torch.float32)
        self.middle = new((rows, hidden), dtype)
        self.h, self.h_scale = new((rows, hidden), torch.int8), new(rows, torch.float32)
        # One workspace for the calls of every row count, cleared here: a run's stream knows nothing of this one's, and what a captured run clears is cleared only when the
        # graph is replayed.  A size is the same for all counts up to a multiple of 64, and up to 4, 8, 16 and 32.
        counts = {min(c, rows) for c in (4, 8, 16, 32, *range(64, rows + 64, 64))}
        size = max(self._workspace_bytes(*self._products(c)) for c in counts)
        self._workspace = new(size, torch.uint8) if size else None
        self._lists = {}
        torch.cuda.synchronize(self.stream.device)             # what was cleared and quantised is there for runs on any stream

    def _products(self, n):
        """Descriptors of the products of n rows, up and down"""
        code = _CODES[self.dtype]
        return (B.linear_desc(rows=n, k=self.width, n=self.hidden, act=ACTS[self.act], dtype=code), B.linear_desc(rows=n, k=self.hidden, n=self.width, dtype=code))

    def _workspace_bytes(self, up, down):
        return max((B.ilinear_s8_workspace_bytes if self.weights[1] is None else B.igated_linear_s8_workspace_bytes)(up), B.ilinear_s8_workspace_bytes(down))

    def calls(self, n):
        """The block's four calls on the first n rows, as (kind, arguments)."""
        code = _CODES[self.dtype]
        norm = B.norm_desc(rows=n, c=self.width, dtype=code, gamma_dtype=B.ICNN_F32, eps=self.eps)
        up, down = self._products(n)
        rows = B.norm_desc(rows=n, c=self.hidden, dtype=code)
        (wg, sg), second, (wd, sd) = self.weights
        bg, bu, bd = self.biases
        ws = self._workspace
        if ws is not None and self._workspace_bytes(up, down) > ws.numel():            # (under another tuning than the constructor's: k stays whole)
            ws = None
        if second is None:
            first = ("linear", (up, self.q, self.q_scale, wg, sg, bg, None, self.middle, ws))
        else:
            first = ("gated_linear", (up, self.q, self.q_scale, wg, sg, bg, *second, bu, self.middle, ws))
        return [("rms_norm", (norm, self.stream, self.update, self.gamma, self.stream, self.q, self.q_scale)), first,
                ("quantize_rows", (rows, self.middle, self.h, self.h_scale)),
                ("linear", (down, self.h, self.h_scale, wd, sd, bd, self.stream, self.stream, ws))]

    def run(self, n=None, stream=None):
        n = self.rows if n is None else n
        if not 0 <= n <= self.rows:
            raise ValueError("%d rows: the buffers hold %d" % (n, self.rows))
        if n not in self._lists:
            self._lists[n] = B.Calls(self.calls(n))
        with torch.cuda.device(self.stream.device):            # (without a stream: torch's current one of this device)
            self._lists[n].run(stream)


def main():
    import argparse
    a = argparse.ArgumentParser(description="times of one block's feed-forward half in 8 bits, random weights")
    a.add_argument("--rows", type=int, nargs="+", default=[1, 16, 512, 4096])
    a.add_argument("--width", type=int, default=4096)
    a.add_argument("--hidden", type=int, default=16384)
    a.add_argument("--act", choices=sorted(ACTS), default="silu")
    a.add_argument("--steps", type=int, default=50)
    a = a.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    w = [torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16) * s[1] ** -0.5 for s in ((a.hidden, a.width), (a.hidden, a.width), (a.width, a.hidden))]
    ff = FeedForward(torch.ones(a.width), *w, rows=max(a.rows), act=a.act)
    ff.update.normal_(generator=g)
    for n in a.rows:
        for _ in range(3):
            ff.stream.normal_(generator=g)
            ff.run(n)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(a.steps):
            ff.run(n)
        end.record()
        torch.cuda.synchronize()
        us = begin.elapsed_time(end) * 1e3 / a.steps
        print("%6d rows  %9.1f us  %8.1f TOP/s  weights at %.2f TB/s" % (n, us, 6e-6 * n * a.width * a.hidden / us, 3e-6 * a.width * a.hidden / us), flush=True)


if __name__ == "__main__":
    main()
