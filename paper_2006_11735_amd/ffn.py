"""The feed-forward half of a transformer block in 8 bits, run through the C boundary:

    stream += update                                  (what the block's other half adds)
    q       = rms_norm(stream) * gamma, in 8 bits     irms_norm_s8
    hidden  = act(q Wgate) * (q Wup)                  igated_linear_s8      (without Wup: act(q Wgate), ilinear_s8)
    h       = hidden, in 8 bits                       iquantize_rows_s8
    stream += h Wdown                                 ilinear_s8

With weights of 4 bits (a scale for each group of a row's numbers) the products are igated_linear_s4 and ilinear_s4.  With experts the hidden layer is one of many:

    logits  = q Wrouter                               ilinear_s8            (float32)
    expert, gate, positions by expert                 iroute_top
    hidden  = act(q Wgate_e) * (q Wup_e)              igrouped_gated_linear_s8
    h       = hidden, in 8 bits                       iquantize_rows_s8
    v       = h Wdown_e                               igrouped_linear_s8
    stream += sum of a token's rows of v by its gates icombine_rows

This is harness code, like netrun: it owns the device buffers, brings the weights to 8 or 4 bits once (a step per output channel or group, by the
library's own quantisation) and issues the calls as one list.  All arithmetic happens inside the library.

    python -m paper_2006_11735_amd.ffn --rows 1 16 512 4096 --width 4096 --hidden 16384 [--bits 4] [--experts 8 --top 2]

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


def quantize_weights_s4(w, group=128, scale_dtype=torch.float16):
    """(packed uint8, scales [n][groups]) of floating weights on the GPU: 4-bit numbers with the step max|w| / 7 for each `group` numbers of a row."""
    if w.dim() != 2 or w.dtype not in _CODES or scale_dtype not in _CODES:
        raise ValueError("weights are [n][k] numbers of float32, float16 or bfloat16, and scales of these types: got %s of %s, %s" % (tuple(w.shape), w.dtype, scale_dtype))
    if group not in (32, 64, 128, 256):
        raise ValueError("group is 32, 64, 128 or 256: got %s" % (group,))
    n, k = w.shape
    if w.stride(1) != 1 or w.stride(0) < k:
        w = w.contiguous()
    packed = torch.empty(B.iweights_s4_bytes(n, k), dtype=torch.uint8, device=w.device)
    scale = torch.empty((n, -(-k // group)), dtype=scale_dtype, device=w.device)
    with torch.cuda.device(w.device):
        B.iquantize_weights_s4(B.quantize_s4_desc(n=n, k=k, group=group, w_stride=w.stride(0), dtype=_CODES[w.dtype], scale_dtype=_CODES[scale_dtype]), w, packed, scale)
    return packed, scale


class FeedForward:
    """`stream` and `update` are the [rows, width] buffers a program reads and writes; run(n) takes their first n rows through the block, in place."""

    def __init__(self, gamma, w_gate, w_up, w_down, *, rows, act="silu", b_gate=None, b_up=None, b_down=None, eps=1e-5, dtype=torch.bfloat16, device="cuda:0",
                 bits=8, group=128, scale_dtype=torch.float16):
        """bits: of the weights, 8 or 4; group and scale_dtype are those of the 4-bit ones' scales"""
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
        if bits not in (8, 4) or group not in (32, 64, 128, 256) or scale_dtype not in _CODES:
            raise ValueError("bits is 8 or 4, group 32, 64, 128 or 256, scale_dtype float32, float16 or bfloat16: got %s, %s, %s" % (bits, group, scale_dtype))
        if not torch.cuda.is_available():
            raise RuntimeError("FeedForward needs a GPU: there is no CPU fallback")
        self.bits, self.group, self.scale_dtype = bits, group, scale_dtype
        self.rows, self.width, self.hidden, self.act, self.eps, self.dtype = rows, width, hidden, act, eps, dtype
        new = lambda shape, t: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        self.gamma = gamma.to(device=device, dtype=torch.float32).contiguous()
        quantize = quantize_weights if bits == 8 else lambda w: quantize_weights_s4(w, group, scale_dtype)  # noqa: E731
        self.weights = [None if w is None else quantize(w.to(device).contiguous()) for w in (w_gate, w_up, w_down)]
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
        if self.bits == 4:
            kw = dict(rows=n, group=self.group, dtype=code, scale_dtype=_CODES[self.scale_dtype])
            return B.linear_s4_desc(k=self.width, n=self.hidden, act=ACTS[self.act], **kw), B.linear_s4_desc(k=self.hidden, n=self.width, **kw)
        return (B.linear_desc(rows=n, k=self.width, n=self.hidden, act=ACTS[self.act], dtype=code), B.linear_desc(rows=n, k=self.hidden, n=self.width, dtype=code))

    def _workspace_bytes(self, up, down):
        if self.bits == 4:
            return 0
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
        if self.bits == 4:
            if second is None:
                first = ("linear_s4", (up, self.q, self.q_scale, wg, sg, bg, None, self.middle))
            else:
                first = ("gated_linear_s4", (up, self.q, self.q_scale, wg, sg, bg, *second, bu, self.middle))
            last = ("linear_s4", (down, self.h, self.h_scale, wd, sd, bd, self.stream, self.stream))
        elif second is None:
            first = ("linear", (up, self.q, self.q_scale, wg, sg, bg, None, self.middle, ws))
        else:
            first = ("gated_linear", (up, self.q, self.q_scale, wg, sg, bg, *second, bu, self.middle, ws))
        if self.bits == 8:
            last = ("linear", (down, self.h, self.h_scale, wd, sd, bd, self.stream, self.stream, ws))
        return [("rms_norm", (norm, self.stream, self.update, self.gamma, self.stream, self.q, self.q_scale)), first,
                ("quantize_rows", (rows, self.middle, self.h, self.h_scale)), last]

    def run(self, n=None, stream=None):
        n = self.rows if n is None else n
        if not 0 <= n <= self.rows:
            raise ValueError("%d rows: the buffers hold %d" % (n, self.rows))
        if n not in self._lists:
            self._lists[n] = B.Calls(self.calls(n))
        with torch.cuda.device(self.stream.device):            # (without a stream: torch's current one of this device)
            self._lists[n].run(stream)


class ExpertsFeedForward:
    """The same with experts: each token's row goes through the `top` experts that its router logits pick.  Weights are [experts, hidden, width] (gate and up) and
    [experts, width, hidden] (down), the router's [experts, width]; all are brought to 8 bits, the router's too: of logits that are closer than its steps another expert may
    be picked than by its weights as they were (iroute_top takes any logits of a program that has its own).  `stream` and `update` are the [rows, width] buffers a program reads
    and writes; run(n) takes their first n rows through the block, in place."""

    def __init__(self, gamma, w_router, w_gate, w_up, w_down, *, rows, top, act="silu", score="softmax", normalise=True, scale=1.0, b_router=None, b_gate=None, b_up=None,
                 b_down=None, eps=1e-5, dtype=torch.bfloat16, device="cuda:0"):
        """score: "softmax" or "sigmoid" of the logits; normalise: gates are divided by the chosen ones' sum; scale: they are multiplied by it"""
        if w_gate.dim() != 3:
            raise ValueError("w_gate is [experts, hidden, width]: got %s" % (tuple(w_gate.shape),))
        experts, hidden, width = w_gate.shape
        if (gamma.shape != (width,) or w_router.shape != (experts, width) or w_down.shape != (experts, width, hidden)
                or (w_up is not None and w_up.shape != (experts, hidden, width))):
            raise ValueError("gamma [width], w_router [experts, width], w_gate and w_up [experts, hidden, width], w_down [experts, width, hidden]: got %s" % ", ".join(
                str(None if t is None else tuple(t.shape)) for t in (gamma, w_router, w_gate, w_up, w_down)))
        for name, b, shape in (("b_router", b_router, (experts,)), ("b_gate", b_gate, (experts, hidden)), ("b_up", b_up, (experts, hidden)), ("b_down", b_down, (experts, width))):
            if b is not None and b.shape != shape:
                raise ValueError("%s has shape %s, not %s" % (name, tuple(b.shape), shape))
        if b_up is not None and w_up is None:
            raise ValueError("b_up without w_up")
        if act not in ACTS or dtype not in _CODES or rows < 1 or score not in ("softmax", "sigmoid"):
            raise ValueError("act is one of %s, dtype float32, float16 or bfloat16, rows at least 1, score softmax or sigmoid" % ", ".join(ACTS))
        if not 1 <= top <= min(experts, 16) or experts > 1024:
            raise ValueError("top %d of %d experts: at most 16 of at most 1024" % (top, experts))
        if not torch.cuda.is_available():
            raise RuntimeError("ExpertsFeedForward needs a GPU: there is no CPU fallback")
        self.rows, self.width, self.hidden, self.experts, self.top, self.act, self.eps, self.dtype = rows, width, hidden, experts, top, act, eps, dtype
        self.score, self.normalise, self.scale = score, normalise, scale
        new = lambda shape, t: torch.zeros(shape, dtype=t, device=device)  # noqa: E731

        def quantize(w):
            q, step = quantize_weights(w.to(device).reshape(-1, w.shape[-1]))
            return q.view(w.shape), step.view(w.shape[:-1])
        self.gamma = gamma.to(device=device, dtype=torch.float32).contiguous()
        self.router, *self.weights = [None if w is None else quantize(w) for w in (w_router, w_gate, w_up, w_down)]
        self.b_router, *self.biases = [None if b is None else b.to(device=device, dtype=torch.float32).contiguous() for b in (b_router, b_gate, b_up, b_down)]
        many = rows * top
        self.stream, self.update = new((rows, width), dtype), new((rows, width), dtype)
        self.q, self.q_scale = new((rows, width), torch.int8), new(rows, torch.float32)
        self.logits = new((rows, experts), torch.float32)
        self.expert, self.place, self.token, self.offsets = new((rows, top), torch.int32), new((rows, top), torch.int32), new(many, torch.int32), new(experts + 1, torch.int32)
        self.gate = new((rows, top), torch.float32)
        self.middle, self.h, self.h_scale, self.v = new((many, hidden), dtype), new((many, hidden), torch.int8), new(many, torch.float32), new((many, width), dtype)
        # (a workspace for the router's product, cleared here, and one for its choice, for every row count as in FeedForward; the choice's size grows with the rows only up
        # to a number of chunks, which the count of rows may bring down again)
        counts = {min(c, rows) for c in (4, 8, 16, 32, *range(64, rows + 64, 64))}
        size = max(B.ilinear_s8_workspace_bytes(self._router_desc(c)) for c in counts)
        self._workspace = new(size, torch.uint8) if size else None
        size = max(B.iroute_top_workspace_bytes(self._route_desc(c)) for c in {rows, *range(1, rows + 1, 32), *range(32, rows + 1, 32)})
        self._counts = new(size, torch.uint8) if size else None
        self._lists = {}
        torch.cuda.synchronize(self.stream.device)             # what was cleared and quantised is there for runs on any stream

    def _router_desc(self, n):
        return B.linear_desc(rows=n, k=self.width, n=self.experts, dtype=B.ICNN_F32)

    def _route_desc(self, n):
        return B.route_desc(rows=n, experts=self.experts, top=self.top, dtype=B.ICNN_F32, normalise=int(self.normalise), scale=self.scale,
                            score=B.ICNN_ROUTE_SOFTMAX if self.score == "softmax" else B.ICNN_ROUTE_SIGMOID)

    def calls(self, n):
        """The block's seven calls on the first n rows, as (kind, arguments)."""
        code, many = _CODES[self.dtype], n * self.top
        norm = B.norm_desc(rows=n, c=self.width, dtype=code, gamma_dtype=B.ICNN_F32, eps=self.eps)
        router = self._router_desc(n)
        ws = self._workspace
        if ws is not None and B.ilinear_s8_workspace_bytes(router) > ws.numel():       # (under another tuning than the constructor's: k stays whole)
            ws = None
        up = B.grouped_desc(rows=many, x_rows=n, k=self.width, n=self.hidden, experts=self.experts, act=ACTS[self.act], dtype=code)
        rows = B.norm_desc(rows=many, c=self.hidden, dtype=code)
        down = B.grouped_desc(rows=many, k=self.hidden, n=self.width, experts=self.experts, dtype=code)
        (wg, sg), second, (wd, sd) = self.weights
        bg, bu, bd = self.biases
        if second is None:
            first = ("grouped_linear", (up, self.q, self.q_scale, self.token, self.offsets, wg, sg, bg, self.middle))
        else:
            first = ("grouped_gated_linear", (up, self.q, self.q_scale, self.token, self.offsets, wg, sg, bg, *second, bu, self.middle))
        return [("rms_norm", (norm, self.stream, self.update, self.gamma, self.stream, self.q, self.q_scale)),
                ("linear", (router, self.q, self.q_scale, *self.router, self.b_router, None, self.logits, ws)),
                ("route", (self._route_desc(n), self.logits, self.expert, self.gate, self.place, self.token, self.offsets, self._counts)), first,
                ("quantize_rows", (rows, self.middle, self.h, self.h_scale)),
                ("grouped_linear", (down, self.h, self.h_scale, None, self.offsets, wd, sd, bd, self.v)),
                ("combine", (B.combine_desc(rows=n, top=self.top, c=self.width, dtype=code), self.v, self.gate, self.place, self.stream, self.stream))]

    run = FeedForward.run


def main():
    import argparse
    a = argparse.ArgumentParser(description="times of one block's feed-forward half in 8 bits, random weights")
    a.add_argument("--rows", type=int, nargs="+", default=[1, 16, 512, 4096])
    a.add_argument("--width", type=int, default=4096)
    a.add_argument("--hidden", type=int, default=16384)
    a.add_argument("--act", choices=sorted(ACTS), default="silu")
    a.add_argument("--steps", type=int, default=50)
    a.add_argument("--bits", type=int, choices=(8, 4), default=8)
    a.add_argument("--group", type=int, choices=(32, 64, 128, 256), default=128, help="numbers that share a scale, of weights of 4 bits")
    a.add_argument("--experts", type=int, default=0, help="so many experts (of 8 bits) instead of one hidden layer")
    a.add_argument("--top", type=int, default=2, help="experts that a token goes through")
    a = a.parse_args()
    if a.experts and a.bits != 8:
        raise SystemExit("experts' weights have 8 bits")
    g = torch.Generator(device="cuda").manual_seed(0)
    many = (a.experts,) if a.experts else ()
    w = [torch.randn(many + s, generator=g, device="cuda", dtype=torch.bfloat16) * s[1] ** -0.5 for s in ((a.hidden, a.width), (a.hidden, a.width), (a.width, a.hidden))]
    if a.experts:
        router = torch.randn((a.experts, a.width), generator=g, device="cuda", dtype=torch.bfloat16) * a.width ** -0.5
        ff = ExpertsFeedForward(torch.ones(a.width), router, *w, rows=max(a.rows), top=a.top, act=a.act)
    else:
        ff = FeedForward(torch.ones(a.width), *w, rows=max(a.rows), act=a.act, bits=a.bits, group=a.group)
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
        per_row, layers = a.top if a.experts else 1, min(a.experts, n * a.top) if a.experts else 1       # (at most so many experts' weights are read)
        print("%6d rows  %9.1f us  %8.1f TOP/s  weights at %.2f TB/s" % (n, us, 6e-6 * n * per_row * a.width * a.hidden / us, 3e-6 * layers * a.width * a.hidden * a.bits / 8 / us),
              flush=True)


if __name__ == "__main__":
    main()
