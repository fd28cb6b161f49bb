"""Definitions in 64 bits (numpy, on the CPU) of the operators with experts and of those with 4-bit weights, with what float32 may be off."""
import numpy as np

from ff_util import ROUNDING, act64

UNIT = 2.0 ** -24                                      # a float32 rounding


def route64(logits, top, score, normalise, scale):
    """(expert, gate, place, token, offsets, relative tolerance of the gates) of float64 logits"""
    rows, experts = logits.shape
    order = np.argsort(np.where(np.isnan(logits), -np.inf, -logits), axis=1, kind="stable")[:, :top] if rows else np.zeros((0, top), int)
    l = np.take_along_axis(logits, order, 1)
    none = l == -np.inf
    expert = np.where(none, -1, order)
    with np.errstate(all="ignore"):
        most = logits.max(1, keepdims=True) if rows else np.zeros((0, 1))
        if score == "softmax":
            e, every = np.exp(l - most), np.exp(logits - most)
            gate = e / np.where(none, 0, e).sum(1, keepdims=True) if normalise else e / np.where(logits == -np.inf, 0, every).sum(1, keepdims=True)
        else:
            # (sigmoids over their sum: the common factor exp(shift) of those that are all tiny cancels)
            shift = np.minimum(most, 0) if normalise else 0
            gate = np.where(l > 0, 1 / (1 + np.exp(-l)), np.exp(np.minimum(l, 0) - shift) / (1 + np.exp(np.minimum(l, 0)))) if normalise else 1 / (1 + np.exp(-l))
            gate = np.where(np.isnan(l), np.nan, gate)
            if normalise:
                gate = gate / np.where(none, 0, gate).sum(1, keepdims=True)
        # The difference to the maximum is rounded (a relative error of exp as large as its rounding: |l - most| units) in numerator and sum; exp is within two
        # units, sums of P + 6 numbers and a division within three, sigmoids' own additions and divisions, the scale: 34 units
        away = np.where(np.isfinite(l - most), np.abs(l - most), 0).max(1, keepdims=True) if rows else np.zeros((0, 1))
        away = np.maximum(away, np.where(np.isfinite(l), np.abs(l), 0).max(1, keepdims=True)) if score == "sigmoid" and rows else away
    gate = np.where(none, 0, gate * scale)
    flat = expert.reshape(-1)
    chosen = np.nonzero(flat >= 0)[0]
    sort = chosen[np.argsort(flat[chosen], kind="stable")]
    place = np.full(flat.shape, -1)
    place[sort] = np.arange(len(sort))
    token = np.full(flat.shape, -1)
    token[:len(sort)] = sort // top
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[chosen], minlength=experts))])
    return expert, gate, place.reshape(expert.shape), token, offsets, (2 * away + 34) * UNIT


def combine64(v, gate, place, res, dtype):
    ok = (place >= 0) & (place < len(v))
    rows = v[np.where(ok, place, 0)] * ok[:, :, None]
    terms = np.where(ok[:, :, None], gate.astype(np.float64)[:, :, None] * rows, 0)
    y, size = terms.sum(1), np.abs(terms).sum(1)
    if res is not None:
        y, size = y + res, size + np.abs(res)
    tol = (place.shape[1] + 2) * UNIT * size           # a product and an addition a term, the residual's
    rel, least = ROUNDING[dtype]
    return y, tol * (1 + rel) + rel * np.abs(y) + least


def quantize4(w, group, scale_type):
    """(numbers, scales) of float64 weights: scale_type a numpy function that rounds"""
    n, k = w.shape
    q, s = np.zeros((n, k)), np.zeros((n, -(-k // group)))
    for i in range(s.shape[1]):
        at = slice(i * group, (i + 1) * group)
        with np.errstate(all="ignore"):
            s[:, i] = scale_type(np.abs(w[:, at]).max(1) / 7)
            q[:, at] = np.where(s[:, i, None] > 0, np.clip(np.rint(w[:, at] / s[:, i, None]), -7, 7), 0)
    return q, s


def packed4(w):
    """Numbers in [-8, 7] as the operators have them: blocks of 32 in 16 bytes, number j in byte j's lower half, 16 + j in its upper one"""
    n, k = w.shape
    p = np.zeros((n, -(-k // 32) * 32), np.int64)
    p[:, :k] = w
    p = p.reshape(n, -1, 2, 16) & 15
    return (p[:, :, 0] | p[:, :, 1] << 4).astype(np.uint8).reshape(n, -1)


def product4(x, xs, w, scales, group, bias):
    """(value, tolerance): sums of groups, or of parts of them by blocks of 32, are exact integers; each is scaled and added in float32, in any order: as many roundings
    as blocks and one for the product; the row's scale and the bias round three times more."""
    k = x.shape[1]
    v, size = 0, 0
    for b in range(0, k, 32):
        acc = (x[:, b:b + 32].astype(np.float64) @ w[:, b:b + 32].astype(np.float64).T) * scales[:, b // group].astype(np.float64)
        v, size = v + acc, size + np.abs(acc)
    xs = xs.astype(np.float64)[:, None]
    b = 0 if bias is None else bias.astype(np.float64)
    v, size = v * xs + b, size * xs + np.abs(b)
    return v, (-(-k // 32) + 4) * UNIT * size


def _act(v, tol, act):
    # the slope of an activation is at most 1.13; its own error as in ff_util.linear64
    return act64(v, act), 1.13 * tol + (0 if act in ("none", "relu") else (4 + np.abs(v)) * 2.0 ** -21 * np.abs(v))


def rounded(y, tol, dtype):
    rel, least = ROUNDING[dtype]
    return y, tol * (1 + rel) + rel * np.abs(y) + least


def linear_s4_64(x, xs, layer, act, res, group, dtype):
    v, tol = _act(*product4(x, xs, layer[0], layer[1], group, layer[2]), act)
    if res is not None:
        v = v + res
        tol = tol + UNIT * np.abs(v)
    return rounded(v, tol, dtype)


def gated_s4_64(x, xs, gate, up, act, group, dtype):
    g, tg = _act(*product4(x, xs, gate[0], gate[1], group, gate[2]), act)
    u, tu = product4(x, xs, up[0], up[1], group, up[2])
    y = g * u
    return rounded(y, tg * np.abs(u) + tu * np.abs(g) + tg * tu + UNIT * np.abs(y), dtype)
