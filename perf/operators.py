"""What is measured of the feed-forward operators in 8 bits: the work that a served transformer block's second half does.

  rows    the residual stream's addition, its root-mean-square norm and the norm's output in 8 bits with a scale per row (`irms_norm_s8`),
          and the same output of rows that are not normalised: the hidden layer between two products (`iquantize_rows_s8`)
  linear  the product of 8-bit rows and 8-bit weights with scales, bias, activation and residual in its epilogue (`ilinear_s8`)
  gated   the gated hidden layer: two such products of one input, an activation of the first times the second (`igated_linear_s8`)

8-bit outputs are returned as the values they stand for (number times scale, in bfloat16): a sum of squares in another order may move a value
across a rounding border.  Sums the operators take in 32 bits are exact integers in the kernels; the plain forms take them in float32.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MOST_ROWS = 8192 * 4096                 # numbers of the largest case of rows
MOST_PRODUCT = 4096 * 4096 * 16384      # multiply-adds of the largest product (a gated layer has two of them)


def listed():
    return [
        # the residual stream of the one token that a decoder is at: latency
        {"name": "rows_norm_1x4096_bf16", "op": "rows", "norm": True, "residual": True, "rows": 1, "c": 4096, "dtype": "bf16"},
        # a float32 stream of odd width: rows that start at no multiple of 16 bytes
        {"name": "rows_norm_517x5001_f32", "op": "rows", "norm": True, "residual": True, "rows": 517, "c": 5001, "dtype": "f32"},
        # the prompts of a batch: bandwidth
        {"name": "rows_norm_8192x4096_bf16", "op": "rows", "norm": True, "residual": True, "rows": 8192, "c": 4096, "dtype": "bf16"},
        # the hidden layer of a prompt on its way to the second product
        {"name": "rows_2048x16384_f16", "op": "rows", "norm": False, "residual": False, "rows": 2048, "c": 16384, "dtype": "f16"},
        # one token back from the hidden layer to the stream: weights read once, bandwidth
        {"name": "linear_1x16384x4096_bf16", "op": "linear", "rows": 1, "k": 16384, "n": 4096, "act": "none", "bias": False, "residual": True, "dtype": "bf16"},
        # the tokens of a small batch of requests through an ungated hidden layer
        {"name": "linear_24x2048x8192_f16", "op": "linear", "rows": 24, "k": 2048, "n": 8192, "act": "gelu", "bias": True, "residual": False, "dtype": "f16"},
        # odd in all three sizes, float32 results
        {"name": "linear_301x1001x1357_f32", "op": "linear", "rows": 301, "k": 1001, "n": 1357, "act": "relu", "bias": True, "residual": True, "dtype": "f32"},
        # the second product of a batch of prompts: the matrix cores' rate
        {"name": "linear_4096x16384x4096_bf16", "op": "linear", "rows": 4096, "k": 16384, "n": 4096, "act": "none", "bias": False, "residual": True, "dtype": "bf16"},
        # the gated hidden layer of one token: the largest share of a decoder's weights
        {"name": "gated_1x4096x16384_bf16", "op": "gated", "rows": 1, "k": 4096, "n": 16384, "act": "silu", "bias": False, "dtype": "bf16"},
        # a hidden width that no tile divides
        {"name": "gated_77x2048x5461_f16", "op": "gated", "rows": 77, "k": 2048, "n": 5461, "act": "gelu_tanh", "bias": True, "dtype": "f16"},
        # one prompt
        {"name": "gated_512x4096x8192_bf16", "op": "gated", "rows": 512, "k": 4096, "n": 8192, "act": "silu", "bias": False, "dtype": "bf16"},
        # a batch of prompts: the largest there is
        {"name": "gated_4096x4096x16384_bf16", "op": "gated", "rows": 4096, "k": 4096, "n": 16384, "act": "silu", "bias": False, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: half of them whole multiples of 64, as most models have them, the others any number."""
    v = _log(rng, lo, hi)
    return max(lo, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["rows", "linear", "gated"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "rows":
        norm = rng.random() < 0.7
        c = _size(rng, 256, 16384)
        return {"op": op, "norm": norm, "residual": norm and rng.random() < 0.8, "rows": _log(rng, 1, min(8192, MOST_ROWS // c)), "c": c,
                "dtype": dtype}
    k, n = _size(rng, 64, 16384), _size(rng, 64, 16384)
    rows = _log(rng, 1, max(1, min(4096, MOST_PRODUCT // (k * n))))
    case = {"op": op, "rows": rows, "k": k, "n": n, "act": rng.choice(ACTS[2:] if op == "gated" else ACTS), "bias": rng.random() < 0.5, "dtype": dtype}
    if op == "linear":
        case["residual"] = rng.random() < 0.5
    return case


def _weights(g, n, k):
    """8-bit weights of a layer as a conversion leaves them (normal, the largest of a row near 127) and their scales."""
    w = torch.randn((n, k), generator=g, device="cuda").mul_(36).round_().clamp_(-127, 127).to(torch.int8)
    return w, (0.5 + torch.rand(n, generator=g, device="cuda")).mul_(1 / (36 * math.sqrt(k)))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, rows = DTYPES[case["dtype"]], case["rows"]
    s = dict(case, torch_dtype=dtype)
    if case["op"] == "rows":
        c = case["c"]
        s["x"] = torch.randn((rows, c), generator=g, device="cuda").mul_(torch.rand((rows, 1), generator=g, device="cuda").add_(0.5)).to(dtype)
        s["res"] = torch.randn((rows, c), generator=g, device="cuda").to(dtype) if case["residual"] else None
        s["gamma"] = (0.5 + torch.rand(c, generator=g, device="cuda")).to(dtype) if case["norm"] else None
    else:
        k, n = case["k"], case["n"]
        s["x"] = torch.randn((rows, k), generator=g, device="cuda").mul_(34).round_().clamp_(-127, 127).to(torch.int8)
        s["x_scale"] = (0.5 + torch.rand(rows, generator=g, device="cuda")).mul_(1 / 34)
        s["w"], s["w_scale"] = _weights(g, n, k)
        s["bias"] = torch.randn(n, generator=g, device="cuda").mul_(0.1) if case["bias"] else None
        if case["op"] == "gated":
            s["w_up"], s["up_scale"] = _weights(g, n, k)
            s["up_bias"] = torch.randn(n, generator=g, device="cuda").mul_(0.1) if case["bias"] else None
        else:
            s["res"] = torch.randn((rows, n), generator=g, device="cuda").to(dtype) if case["residual"] else None
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps for such a call: its descriptor, its output buffers, and the list that it issues."""
    from paper_2006_11735_amd import binding as B
    dtype, rows = s["torch_dtype"], s["rows"]
    code = {"f32": B.ICNN_F32, "f16": B.ICNN_F16, "bf16": B.ICNN_BF16}[s["dtype"]]
    if s["op"] == "rows":
        d = B.norm_desc(rows=rows, c=s["c"], dtype=code, gamma_dtype=code, eps=1e-5)
        s["q"] = torch.empty((rows, s["c"]), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty((rows, 1), dtype=torch.float32, device="cuda")
        s["value"] = torch.empty((rows, s["c"]), dtype=torch.bfloat16, device="cuda")
        s["sum"] = torch.empty_like(s["x"]) if s["residual"] else None
        if s["norm"]:
            s["calls"] = B.Calls([("rms_norm", (d, s["x"], s["res"], s["gamma"], s["sum"], s["q"], s["scale"]))])
        else:
            s["calls"] = B.Calls([("quantize_rows", (d, s["x"], s["q"], s["scale"]))])
        return
    d = B.linear_desc(rows=rows, k=s["k"], n=s["n"], act=ACTS.index(s["act"]), dtype=code)
    s["y"] = torch.empty((rows, s["n"]), dtype=dtype, device="cuda")
    if s["op"] == "linear":
        size = B.ilinear_s8_workspace_bytes(d)
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda") if size else None
        s["calls"] = B.Calls([("linear", (d, s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], s["res"], s["y"], s["ws"]))])
    else:
        size = B.igated_linear_s8_workspace_bytes(d)
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda") if size else None
        s["calls"] = B.Calls([("gated_linear", (d, s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], s["w_up"], s["up_scale"], s["up_bias"],
                                                s["y"], s["ws"]))])


def _act(v, kind):
    if kind == "relu":
        return v.clamp_min(0)
    if kind == "silu":
        return v / (1 + torch.exp(-v))
    if kind == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _product(x, x_scale, w, w_scale, bias):
    v = torch.matmul(x.float(), w.float().t()) * x_scale[:, None] * w_scale
    return v if bias is None else v + bias


def run(s):
    if own:
        s["calls"].run()
        if s["op"] != "rows":
            return {"y": s["y"]}
        torch.mul(s["q"], s["scale"], out=s["value"])
        out = {"value": s["value"], "scale": s["scale"]}
        return dict(out, sum=s["sum"]) if s["residual"] else out
    if s["op"] == "rows":
        t, out = s["x"].float(), {}
        if s["residual"]:
            out["sum"] = (t + s["res"].float()).to(s["torch_dtype"])
            t = out["sum"].float()
        if s["norm"]:
            t = t * torch.rsqrt((t * t).mean(1, keepdim=True) + 1e-5) * s["gamma"].float()
        most = t.abs().amax(1, keepdim=True)
        out["scale"] = most / 127
        out["value"] = (torch.round(t * (127 / most)) * out["scale"]).to(torch.bfloat16)
        return out
    v = _act(_product(s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"]), s["act"])
    if s["op"] == "gated":
        v = v * _product(s["x"], s["x_scale"], s["w_up"], s["up_scale"], s["up_bias"])
    elif s["res"] is not None:
        v = v + s["res"].float()
    return {"y": v.to(s["torch_dtype"])}


def work(case):
    rows, item = case["rows"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["op"] == "rows":
        c, many = case["c"], rows * case["c"]
        # x, the residual and the sum; 8-bit numbers and scales out; gamma
        return {"bytes": many * item * (3 if case["residual"] else 1) + many + 4 * rows + (c * item if case["norm"] else 0),
                "flops": many * (7 if case["norm"] else 3)}
    k, n, layers = case["k"], case["n"], 2 if case["op"] == "gated" else 1
    per_n = k + 4 + (4 if case["bias"] else 0)
    return {"bytes": rows * (k + 4) + layers * n * per_n + rows * n * item * (2 if case.get("residual") else 1), "flops": 2.0 * layers * rows * k * n}


def exact(case, seed):
    """The definition in 64 bits.  The sum's rounding to the stream's type is part of it, and the 8-bit numbers' too."""
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "rows":
        out, t = {}, wide["x"]
        if case["residual"]:
            t = (t + wide["res"]).to(s["torch_dtype"]).double()
            out["sum"] = t
        if case["norm"]:
            t = t / (t.square().sum(1, keepdim=True) / case["c"] + 1e-5).sqrt() * wide["gamma"]
        step = t.abs().max(1, keepdim=True).values / 127
        return dict(out, scale=step, value=(t / step).round() * step)

    def layer(w, scale, bias):
        weights = s[w].double() * wide[scale][:, None]
        v = (s["x"].double() * wide["x_scale"][:, None]) @ weights.T
        return v if s[bias] is None else v + wide[bias]

    v = layer("w", "w_scale", "bias")
    if case["act"] == "relu":
        v = torch.where(v > 0, v, torch.zeros_like(v))
    elif case["act"] == "silu":
        v = v * torch.special.expit(v)
    elif case["act"] == "gelu":
        v = v * torch.special.ndtr(v)
    elif case["act"] == "gelu_tanh":
        v = v * torch.special.expit(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    if case["op"] == "gated":
        v = v * layer("w_up", "up_scale", "up_bias")
    elif case["residual"]:
        v = v + wide["res"]
    return {"y": v}
