"""What is measured of the feed-forward operators with experts and of those with weights of 4 bits: what a served transformer block's second half does where
its hidden layer is one of many, or where its weights are half as wide.

  route          the router: a token's largest logits, its gates, and all tokens' positions in the order of the experts (`iroute_top`)
  grouped        rows that lie in the order of their experts through each one's own 8-bit weights (`igrouped_linear_s8`)
  grouped_gated  the experts' gated hidden layers, rows read where the tokens have them (`igrouped_gated_linear_s8`)
  combine        the sum of a token's expert rows by its gates, on top of the stream (`icombine_rows`)
  linear_s4      the product of 8-bit rows and 4-bit weights with a scale for each group of a row's numbers (`ilinear_s4`)
  gated_s4       the gated hidden layer of such weights (`igated_linear_s4`)

Sums over k are exact integers in the kernels (over a group's numbers where weights have 4 bits); the plain forms take them in float32.
"""
import math

import numpy as np
import torch

own = False

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MOST_LOGITS = 8192 * 256                # logits of the largest router call
MOST_ROWS = 4096 * 4 * 4096             # numbers of the largest combination
MOST_PRODUCT = 8192 * 8192 * 4096       # multiply-adds of the largest product
MOST_WEIGHTS = 8 * 2 * 4096 * 8192      # bytes of all experts' weights


def listed():
    return [
        # the one token that a decoder is at: latency
        {"name": "route_1x64_top8_f32", "op": "route", "rows": 1, "experts": 64, "top": 8, "dtype": "f32", "score": "softmax", "normalise": True},
        # the prompts of a batch, many small experts
        {"name": "route_8192x256_top8_bf16", "op": "route", "rows": 8192, "experts": 256, "top": 8, "dtype": "bf16", "score": "sigmoid", "normalise": True},
        # the same one token's experts back into its stream
        {"name": "combine_1x4096_top2_bf16", "op": "combine", "rows": 1, "top": 2, "c": 4096, "dtype": "bf16"},
        # the prompts of a batch: bandwidth
        {"name": "combine_4096x4096_top4_f16", "op": "combine", "rows": 4096, "top": 4, "c": 4096, "dtype": "f16"},
        # odd in every size, a popular and a forsaken expert among seventeen, float32 results
        {"name": "grouped_301x1001x1357_f32", "op": "grouped", "rows": 301, "experts": 17, "top": 3, "k": 1001, "n": 1357, "act": "none", "bias": True, "dtype": "f32"},
        # a batch of prompts back from eight experts' hidden layers: the matrix cores' rate
        {"name": "grouped_4096x8192x4096_bf16", "op": "grouped", "rows": 4096, "experts": 8, "top": 2, "k": 8192, "n": 4096, "act": "none", "bias": False, "dtype": "bf16"},
        # the hidden layers of one token: two experts' weights read once
        {"name": "grouped_gated_1x4096x8192_bf16", "op": "grouped_gated", "rows": 1, "experts": 8, "top": 2, "k": 4096, "n": 8192, "act": "silu", "bias": False, "dtype": "bf16"},
        # a prompt through many narrow experts
        {"name": "grouped_gated_2048x2048x2048_f16", "op": "grouped_gated", "rows": 2048, "experts": 32, "top": 4, "k": 2048, "n": 2048, "act": "silu", "bias": False, "dtype": "f16"},
        # one token back from the hidden layer to the stream: weights read once
        {"name": "linear_s4_1x16384x4096_bf16", "op": "linear_s4", "rows": 1, "k": 16384, "n": 4096, "group": 128, "scales": "f16", "act": "none", "bias": False, "residual": True, "dtype": "bf16"},
        # the tokens of a small batch, sizes that no block of weights divides
        {"name": "linear_s4_24x2001x5461_f16", "op": "linear_s4", "rows": 24, "k": 2001, "n": 5461, "group": 64, "scales": "f32", "act": "gelu", "bias": True, "residual": False, "dtype": "f16"},
        # the hidden layer of one token
        {"name": "gated_s4_1x4096x16384_bf16", "op": "gated_s4", "rows": 1, "k": 4096, "n": 16384, "group": 128, "scales": "f16", "act": "silu", "bias": False, "dtype": "bf16"},
        # one prompt
        {"name": "gated_s4_512x4096x8192_bf16", "op": "gated_s4", "rows": 512, "k": 4096, "n": 8192, "group": 128, "scales": "bf16", "act": "silu", "bias": False, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: half of them whole multiples of 64, as most models have them, the others any number."""
    v = _log(rng, lo, hi)
    return max(lo, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["route", "combine", "grouped", "grouped_gated", "linear_s4", "gated_s4"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    case = {"op": op, "dtype": dtype}
    if op == "route":
        experts = _log(rng, 4, 512)
        return dict(case, rows=_log(rng, 1, min(16384, MOST_LOGITS // experts)), experts=experts, top=rng.randint(1, min(8, experts)),
                    score=rng.choice(["softmax", "sigmoid"]), normalise=rng.random() < 0.6)
    if op == "combine":
        c, top = _size(rng, 256, 8192), rng.randint(1, 8)
        return dict(case, rows=_log(rng, 1, min(4096, MOST_ROWS // (2 * c * top))), top=top, c=c)
    gated = op in ("grouped_gated", "gated_s4")
    case["act"] = rng.choice(ACTS[2:] if gated else ACTS)
    case["bias"] = rng.random() < 0.5
    k, n = _size(rng, 64, 8192), _size(rng, 64, 8192)
    macs = k * n * (2 if gated else 1)
    if op in ("grouped", "grouped_gated"):
        experts = _log(rng, 2, max(2, min(64, MOST_WEIGHTS // macs)))
        top = rng.randint(1, min(4, experts))
        return dict(case, rows=_log(rng, 1, max(1, min(4096, MOST_PRODUCT // (macs * top)))), experts=experts, top=top, k=k, n=n)
    case.update(rows=_log(rng, 1, max(1, min(1024, MOST_PRODUCT // (4 * macs)))), k=k, n=n, group=rng.choice([32, 64, 128, 256]),
                scales=rng.choice(["f16", "bf16", "f32"]))
    if op == "linear_s4":
        case["residual"] = rng.random() < 0.5
    return case


def _normal8(shape, g, spread):
    return torch.randn(shape, generator=g, device="cuda").mul_(spread).round_().clamp_(-127, 127).to(torch.int8)


def _rows8(rows, k, g):
    """8-bit rows as the norm leaves them, and their scales."""
    return _normal8((rows, k), g, 34), (0.5 + torch.rand(rows, generator=g, device="cuda")).mul_(1 / 34)


def _weights8(experts, n, k, g):
    """All experts' weights, normal with the largest of a row near 127, and a scale per output."""
    w = torch.empty((experts, n, k), dtype=torch.int8, device="cuda")
    for e in range(experts):
        w[e] = _normal8((n, k), g, 36)
    return w, (0.5 + torch.rand((experts, n), generator=g, device="cuda")).mul_(1 / (36 * math.sqrt(k)))


def _weights4(n, k, group, dtype, g):
    """4-bit weights as numbers, and their groups' scales."""
    w = torch.randn((n, k), generator=g, device="cuda").mul_(2.6).round_().clamp_(-8, 7).to(torch.int8)
    return w, (0.5 + torch.rand((n, -(-k // group)), generator=g, device="cuda")).mul_(1 / (2.6 * math.sqrt(k))).to(dtype)


def _groups(rows, experts, top, g):
    """Which tokens go to which expert, some experts more in demand than others: the tokens in the experts' order and each expert's first position."""
    score = torch.rand((rows, experts), generator=g, device="cuda") * torch.rand(experts, generator=g, device="cuda")
    chosen = score.topk(top, dim=1).indices.reshape(-1)
    order = torch.sort(chosen, stable=True).indices
    counts = torch.bincount(chosen, minlength=experts).cpu()
    bounds = [0] + torch.cumsum(counts, 0).tolist()
    return (order // top).to(torch.int32), bounds


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, rows, dtype = case["op"], case["rows"], DTYPES[case["dtype"]]
    s = dict(case, torch_dtype=dtype)
    if op == "route":
        s["logits"] = torch.randn((rows, case["experts"]), generator=g, device="cuda").mul_(1.5).to(dtype)
    elif op == "combine":
        many = rows * case["top"]
        s["v"] = torch.randn((many, case["c"]), generator=g, device="cuda").to(dtype)
        s["res"] = torch.randn((rows, case["c"]), generator=g, device="cuda").to(dtype)
        gate = torch.rand((rows, case["top"]), generator=g, device="cuda") + 0.05
        s["gate"] = gate / gate.sum(1, keepdim=True)
        s["place"] = torch.randperm(many, generator=g, device="cuda").to(torch.int32).view(rows, case["top"])
    elif op in ("grouped", "grouped_gated"):
        k, n, experts = case["k"], case["n"], case["experts"]
        s["token"], s["bounds"] = _groups(rows, experts, case["top"], g)
        s["offsets"] = torch.tensor(s["bounds"], dtype=torch.int32, device="cuda")
        s["positions"] = rows * case["top"]
        # the first product reads each token's row where it is, the second one the rows that the first has left in the experts' order
        s["x"], s["x_scale"] = _rows8(rows if op == "grouped_gated" else s["positions"], k, g)
        for name in ("", "up_")[:2 if op == "grouped_gated" else 1]:
            s[name + "w"], s[name + "scale"] = _weights8(experts, n, k, g)
            s[name + "bias"] = torch.randn((experts, n), generator=g, device="cuda").mul_(0.1) if case["bias"] else None
    else:
        k, n = case["k"], case["n"]
        s["x"], s["x_scale"] = _rows8(rows, k, g)
        for name in ("", "up_")[:2 if op == "gated_s4" else 1]:
            s[name + "w"], s[name + "scale"] = _weights4(n, k, case["group"], DTYPES[case["scales"]], g)
            s[name + "bias"] = torch.randn(n, generator=g, device="cuda").mul_(0.1) if case["bias"] else None
        s["res"] = torch.randn((rows, n), generator=g, device="cuda").to(dtype) if case.get("residual") else None
    if own:
        _plan(s)
    return s


def _packed4(w):
    """Blocks of 32 numbers in 16 bytes: byte j has number j in its low half and number 16 + j in its high one."""
    n, k = w.shape
    blocks = torch.nn.functional.pad(w, (0, -k % 32)).view(n, -1, 2, 16)
    return ((blocks[:, :, 0] & 15) | (blocks[:, :, 1] << 4)).reshape(n, -1).contiguous()


def _plan(s):
    """What a program keeps for such a call: its descriptor, its output buffers, weights in the operator's layout, and the list that it issues."""
    from paper_2006_11735_amd import binding as B
    codes = {"f32": B.ICNN_F32, "f16": B.ICNN_F16, "bf16": B.ICNN_BF16}
    op, rows, code, dtype = s["op"], s["rows"], codes[s["dtype"]], s["torch_dtype"]
    new = lambda shape, t: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
    if op == "route":
        d = B.route_desc(rows=rows, experts=s["experts"], top=s["top"], dtype=code, normalise=int(s["normalise"]),
                         score=B.ICNN_ROUTE_SOFTMAX if s["score"] == "softmax" else B.ICNN_ROUTE_SIGMOID)
        many, size = rows * s["top"], B.iroute_top_workspace_bytes(d)
        s["out"] = {"expert": new((rows, s["top"]), torch.int32), "gate": new((rows, s["top"]), torch.float32), "place": new((rows, s["top"]), torch.int32),
                    "token": new(many, torch.int32), "offsets": new(s["experts"] + 1, torch.int32)}
        s["ws"] = new(size, torch.uint8) if size else None
        s["calls"] = B.Calls([("route", (d, s["logits"], *s["out"].values(), s["ws"]))])
    elif op == "combine":
        d = B.combine_desc(rows=rows, top=s["top"], c=s["c"], v_rows=rows * s["top"], dtype=code, v_dtype=code)
        s["out"] = {"y": new((rows, s["c"]), dtype)}
        s["calls"] = B.Calls([("combine", (d, s["v"], s["gate"], s["place"], s["res"], s["out"]["y"]))])
    elif op in ("grouped", "grouped_gated"):
        d = B.grouped_desc(rows=s["positions"], x_rows=s["x"].shape[0], k=s["k"], n=s["n"], experts=s["experts"], act=ACTS.index(s["act"]), dtype=code)
        s["out"] = {"y": new((s["positions"], s["n"]), dtype)}
        if op == "grouped":
            s["calls"] = B.Calls([("grouped_linear", (d, s["x"], s["x_scale"], None, s["offsets"], s["w"], s["scale"], s["bias"], s["out"]["y"]))])
        else:
            s["calls"] = B.Calls([("grouped_gated_linear", (d, s["x"], s["x_scale"], s["token"], s["offsets"], s["w"], s["scale"], s["bias"],
                                                            s["up_w"], s["up_scale"], s["up_bias"], s["out"]["y"]))])
    else:
        d = B.linear_s4_desc(rows=rows, k=s["k"], n=s["n"], group=s["group"], act=ACTS.index(s["act"]), dtype=code, scale_dtype=codes[s["scales"]])
        s["out"] = {"y": new((rows, s["n"]), dtype)}
        packed = _packed4(s["w"])
        if op == "linear_s4":
            s["calls"] = B.Calls([("linear_s4", (d, s["x"], s["x_scale"], packed, s["scale"], s["bias"], s["res"], s["out"]["y"]))])
        else:
            s["calls"] = B.Calls([("gated_linear_s4", (d, s["x"], s["x_scale"], packed, s["scale"], s["bias"], _packed4(s["up_w"]), s["up_scale"],
                                                       s["up_bias"], s["out"]["y"]))])


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


def _route(s):
    rows, experts, top = s["rows"], s["experts"], s["top"]
    logits = s["logits"].float()
    best, expert = torch.sort(logits, dim=1, descending=True, stable=True)
    best, expert = best[:, :top], expert[:, :top]
    if s["score"] == "softmax":
        every = torch.exp(logits - best[:, :1])
        gate = torch.exp(best - best[:, :1])
        gate = gate / (gate if s["normalise"] else every).sum(1, keepdim=True)
    else:
        gate = 1 / (1 + torch.exp(-best))
        if s["normalise"]:
            gate = gate / gate.sum(1, keepdim=True)
    flat = expert.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    hits = torch.zeros(experts, dtype=torch.int64, device=flat.device).index_add_(0, flat, torch.ones_like(flat))
    offsets = torch.cat([hits.new_zeros(1), torch.cumsum(hits, 0)])
    return {"expert": expert.to(torch.int32), "gate": gate, "place": place.view(rows, top).to(torch.int32), "token": (order // top).to(torch.int32),
            "offsets": offsets.to(torch.int32)}


def _grouped(s):
    y = torch.zeros((s["positions"], s["n"]), dtype=s["torch_dtype"], device="cuda")
    for e in range(s["experts"]):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if lo == hi:
            continue
        if s["op"] == "grouped":
            x, xs = s["x"][lo:hi].float(), s["x_scale"][lo:hi, None]
        else:
            at = s["token"][lo:hi].long()
            x, xs = s["x"][at].float(), s["x_scale"][at, None]

        def product(name):
            v = torch.matmul(x, s[name + "w"][e].float().t()) * xs * s[name + "scale"][e]
            return v if s[name + "bias"] is None else v + s[name + "bias"][e]
        v = _act(product(""), s["act"])
        if s["op"] == "grouped_gated":
            v = v * product("up_")
        y[lo:hi] = v.to(s["torch_dtype"])
    return y


def _product4(s, name):
    wide = s[name + "scale"].float().repeat_interleave(s["group"], dim=1)[:, :s["k"]] * s[name + "w"].float()
    v = torch.matmul(s["x"].float(), wide.t()) * s["x_scale"][:, None]
    return v if s[name + "bias"] is None else v + s[name + "bias"]


def run(s):
    if own:
        s["calls"].run()
        return s["out"]
    op = s["op"]
    if op == "route":
        return _route(s)
    if op == "combine":
        v = s["v"].float()[s["place"].long()]
        return {"y": (s["res"].float() + (v * s["gate"][:, :, None]).sum(1)).to(s["torch_dtype"])}
    if op in ("grouped", "grouped_gated"):
        return {"y": _grouped(s)}
    v = _act(_product4(s, ""), s["act"])
    if op == "gated_s4":
        v = v * _product4(s, "up_")
    elif s["res"] is not None:
        v = v + s["res"].float()
    return {"y": v.to(s["torch_dtype"])}


def work(case):
    op, rows, item = case["op"], case["rows"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if op == "route":
        e, top = case["experts"], case["top"]
        # logits in; expert, gate, place and token of each choice, the experts' first positions out
        return {"bytes": rows * (e * item + 16 * top) + 4 * (e + 1), "flops": rows * e * (1 + top)}
    if op == "combine":
        c, top = case["c"], case["top"]
        return {"bytes": rows * (c * item * (top + 2) + 8 * top), "flops": 2 * rows * top * c}
    k, n, gated = case["k"], case["n"], op in ("grouped_gated", "gated_s4")
    layers = 2 if gated else 1
    if op in ("grouped", "grouped_gated"):
        many = rows * case["top"]
        # each of the experts that these positions can reach once: as many as there are, or one a position
        per_expert = layers * n * (k + 4 + (4 if case["bias"] else 0))
        x = rows * (k + 4) + 4 * many if gated else many * (k + 4)
        return {"bytes": min(case["experts"], many) * per_expert + x + many * n * item + 4 * (case["experts"] + 1), "flops": 2.0 * layers * many * k * n}
    scale = {"f32": 4, "f16": 2, "bf16": 2}[case["scales"]]
    per_n = 16 * -(-k // 32) + scale * -(-k // case["group"]) + (4 if case["bias"] else 0)
    return {"bytes": rows * (k + 4) + layers * n * per_n + rows * n * item * (2 if case.get("residual") else 1), "flops": 2.0 * layers * rows * k * n}


def exact(case, seed):
    """The definition in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        logits = s["logits"].double().cpu().numpy()
        expert = np.argsort(-logits, axis=1, kind="stable")[:, :case["top"]]
        chosen = np.take_along_axis(logits, expert, 1)
        if case["score"] == "softmax":
            over = chosen if case["normalise"] else logits
            gate = np.exp(chosen - np.logaddexp.reduce(over, axis=1, keepdims=True))
        else:
            gate = 0.5 + 0.5 * np.tanh(0.5 * chosen)
            if case["normalise"]:
                gate /= gate.sum(1, keepdims=True)
        many = expert.size
        order = np.lexsort((np.arange(many), expert.reshape(-1)))
        place = np.argsort(order, kind="stable").reshape(expert.shape)
        offsets = np.searchsorted(expert.reshape(-1)[order], np.arange(case["experts"] + 1), side="left")
        whole = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
        return {"expert": whole(expert), "gate": torch.from_numpy(gate).cuda(), "place": whole(place), "token": whole(order // case["top"]), "offsets": whole(offsets)}
    if op == "combine":
        y = s["res"].double()
        for j in range(case["top"]):
            y = y + s["gate"][:, j, None].double() * s["v"].double().index_select(0, s["place"][:, j].long())
        return {"y": y}

    def act(v):
        if case["act"] == "relu":
            return torch.where(v > 0, v, torch.zeros_like(v))
        if case["act"] == "silu":
            return v * torch.special.expit(v)
        if case["act"] == "gelu":
            return v * torch.special.ndtr(v)
        if case["act"] == "gelu_tanh":
            return v * torch.special.expit(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return v

    x = s["x"].double() * s["x_scale"].double()[:, None]
    if op in ("grouped", "grouped_gated"):
        if op == "grouped_gated":
            x = x.index_select(0, s["token"].long())
        y = torch.empty((s["positions"], case["n"]), dtype=torch.float64, device="cuda")
        for e, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
            def layer(name):
                v = (x[lo:hi] @ s[name + "w"][e].double().T) * s[name + "scale"][e].double()
                return v + s[name + "bias"][e].double() if case["bias"] else v
            if hi > lo:
                y[lo:hi] = act(layer("")) * layer("up_") if op == "grouped_gated" else act(layer(""))
        return {"y": y}

    def layer(name):
        w = torch.zeros((case["n"], case["k"]), dtype=torch.float64, device="cuda")
        for i in range(s[name + "scale"].shape[1]):
            at = slice(i * case["group"], min((i + 1) * case["group"], case["k"]))
            w[:, at] = s[name + "w"][:, at].double() * s[name + "scale"][:, i, None].double()
        v = x @ w.T
        return v + s[name + "bias"].double() if case["bias"] else v
    v = act(layer(""))
    if op == "gated_s4":
        v = v * layer("up_")
    elif case["residual"]:
        v = v + s["res"].double()
    return {"y": v}
