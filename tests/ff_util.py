"""The feed-forward operators' definitions in 64 bits (numpy, on the CPU), and tensors placed with strides and offsets in guarded buffers."""
import math

import numpy as np
import torch

from paper_2006_11735_amd import binding as B

DTYPES = {"f32": (torch.float32, B.ICNN_F32), "f16": (torch.float16, B.ICNN_F16), "bf16": (torch.bfloat16, B.ICNN_BF16)}
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
# half a unit in the last place, relative, and the least spacing's half (subnormals)
ROUNDING = {"f32": (2.0 ** -24, 2.0 ** -150), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -134)}
_ERF = np.vectorize(math.erf, otypes=[np.float64])


class Placed:
    """`rows` x `width` elements of a device buffer, `stride` apart, the first `offset` elements in; the rest holds a guard pattern."""

    def __init__(self, rows, width, dtype, stride=None, offset=0, values=None):
        self.rows, self.width, self.stride = rows, width, width if stride is None else stride
        item = torch.empty(0, dtype=dtype).element_size()
        size = max(0, rows - 1) * self.stride + width + offset + 32
        self.raw = torch.full((size * item,), 0xA5, dtype=torch.uint8, device="cuda:0")
        flat = self.raw.view(dtype)
        self.view = flat.as_strided((rows, width), (self.stride, 1), offset)
        self.before = None
        if values is not None:
            self.view.copy_(values)
        self.address = flat.data_ptr() + offset * item

    def data_ptr(self):
        return self.address

    def snapshot(self):
        self.before = self.raw.clone()

    def rest_untouched(self):
        """whether all bytes but the rows' are what they were at the snapshot"""
        now = self.raw.clone()
        old = self.before.clone()
        for t in (now, old):
            t.view(self.view.dtype).as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).zero_()
        return bool((now == old).all())


def act64(v, kind):
    if kind == "relu":
        return np.maximum(v, 0)
    if kind == "silu":
        return v / (1 + np.exp(-v))
    if kind == "gelu":
        return v * 0.5 * (1 + _ERF(v / math.sqrt(2)))
    if kind == "gelu_tanh":
        return v * 0.5 * (1 + np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def product64(x, xs, w, ws, bias):
    """(value, what its float32 error scales with): the sum is an exact integer, so three products and an addition round"""
    acc = x.astype(np.float64) @ w.astype(np.float64).T
    p = acc * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
    b = 0 if bias is None else bias.astype(np.float64)
    return p + b, np.abs(p) + np.abs(b)


def linear64(x, xs, w, ws, bias, act, res, dtype):
    """(y, tolerance).  v is off by up to 4 roundings of its terms, 2^-22 of them.  The activations' slope is at most 1.13; their own error is that of exp, whose
    argument v log2(e) is rounded (|v| 2^-23 relative), a reciprocal, erf (a few units of 1) and four products: together below (4 + |v|) 2^-21 |v|."""
    v, size = product64(x, xs, w, ws, bias)
    y = act64(v, act)
    tol = 1.13 * 2.0 ** -22 * size + (0 if act in ("none", "relu") else (4 + np.abs(v)) * 2.0 ** -21 * np.abs(v))
    if res is not None:
        y = y + res.astype(np.float64)
        tol = tol + 2.0 ** -24 * np.abs(y)
    rel, least = ROUNDING[dtype]
    return y, tol * (1 + rel) + rel * np.abs(y) + least


def gated64(x, xs, w, ws, bias, w2, ws2, bias2, act, dtype):
    g, tol_g = linear64(x, xs, w, ws, bias, act, None, "f32")
    u, tol_u = linear64(x, xs, w2, ws2, bias2, "none", None, "f32")
    y = g * u
    tol = tol_g * np.abs(u) + tol_u * np.abs(g) + tol_g * tol_u + 2.0 ** -24 * np.abs(y)
    rel, least = ROUNDING[dtype]
    return y, tol * (1 + rel) + rel * np.abs(y) + least


def rows64(s, gamma, eps):
    """(u, scale) of rows that are already the sums: gamma None = no norm"""
    u = s.astype(np.float64)
    if gamma is not None:
        u = u / np.sqrt((u * u).mean(1, keepdims=True) + eps) * gamma.astype(np.float64)
    return u, np.abs(u).max(1) / 127


def to_numpy(t):
    return t.detach().to("cpu").to(torch.float64).numpy() if t.is_floating_point() else t.detach().cpu().numpy()
