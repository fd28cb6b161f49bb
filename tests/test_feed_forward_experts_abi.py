"""What the operators with experts and those with 4-bit weights refuse, on the host, before anything is launched."""
import ctypes

import pytest

from paper_2006_11735_amd import binding as B
from test_feed_forward_abi import accepted, code

X, XS, IX, OF, W, WS, BI, W2, WS2, BI2, R, Y, G, P, T, SP = (k << 28 for k in range(1, 17))


def size_code(fn, *args):
    with pytest.raises(B.IcnnError) as e:
        fn(*args)
    return e.value.code


def test_the_descriptors_have_the_layout_of_the_header():
    sizes = {B.icnn_route_desc: 40, B.icnn_grouped_desc: 72, B.icnn_combine_desc: 56, B.icnn_linear_s4_desc: 56, B.icnn_quantize_s4_desc: 32}
    assert {t: ctypes.sizeof(t) for t in sizes} == sizes
    d = B.grouped_desc(rows=3, k=40, n=8, experts=2, w_stride=48)
    assert (d.x_rows, d.x_stride, d.w_stride, d.expert_stride, d.y_stride, d.dtype) == (3, 40, 48, 384, 8, B.ICNN_BF16)
    d = B.combine_desc(rows=3, top=2, c=10, dtype=B.ICNN_F32)
    assert (d.v_rows, d.v_stride, d.res_stride, d.y_stride, d.v_dtype) == (6, 10, 10, 10, B.ICNN_F32)
    d = B.route_desc(rows=3, experts=10, top=2)
    assert (d.logits_stride, d.dtype, d.scale, d.score) == (10, B.ICNN_F32, 1.0, B.ICNN_ROUTE_SOFTMAX)
    d = B.linear_s4_desc(rows=3, k=40, n=8)
    assert (d.x_stride, d.res_stride, d.y_stride, d.group, d.scale_dtype) == (40, 8, 8, 128, B.ICNN_F16)


# ---- the router

@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 30), B.ICNN_E_SHAPE), (dict(experts=0), B.ICNN_E_SHAPE), (dict(experts=1025, logits_stride=2000), B.ICNN_E_SHAPE),
    (dict(top=0), B.ICNN_E_SHAPE), (dict(top=17), B.ICNN_E_SHAPE), (dict(experts=3), B.ICNN_E_SHAPE), (dict(logits_stride=63), B.ICNN_E_SHAPE),
    (dict(logits_stride=1 << 41), B.ICNN_E_SHAPE), (dict(dtype=B.ICNN_S8), B.ICNN_E_PARAM), (dict(score=2), B.ICNN_E_PARAM), (dict(score=-1), B.ICNN_E_PARAM),
    (dict(normalise=2), B.ICNN_E_PARAM), (dict(scale=float("nan")), B.ICNN_E_PARAM), (dict(scale=float("inf")), B.ICNN_E_PARAM)])
def test_route_descriptors(kw, want):
    d = B.route_desc(**{**dict(rows=10, experts=64, top=4), **kw})
    assert code(B.iroute_top, d, X, W, G, P, T, OF, SP) == want
    assert size_code(B.iroute_top_workspace_bytes, d) == want


def test_route_pointers_and_overlaps():
    d = B.route_desc(rows=10, experts=64, top=4)
    good = [X, W, G, P, T, OF]
    assert accepted(B.iroute_top, d, *good)
    for k in range(6):
        assert code(B.iroute_top, d, *[None if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_NULL, k
        assert code(B.iroute_top, d, *[p + 2 if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_ALIGN, k
    for k in range(1, 6):                              # every output on another one, and on the logits
        for j in range(6):
            if j != k:
                assert code(B.iroute_top, d, *[good[j] + 16 if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_UNSUPPORTED, (k, j)
    many = B.route_desc(rows=1000, experts=64, top=4)
    assert B.iroute_top_workspace_bytes(d) == 0 and B.iroute_top_workspace_bytes(many) > 0
    assert code(B.iroute_top, many, *good) == B.ICNN_E_NULL and code(B.iroute_top, many, *good, SP + 8) == B.ICNN_E_ALIGN
    assert code(B.iroute_top, many, *good, T + 16) == B.ICNN_E_UNSUPPORTED and accepted(B.iroute_top, many, *good, SP)
    assert code(B.iroute_top, B.route_desc(rows=0, experts=64, top=4), *[None] * 6) == B.ICNN_E_NULL
    with pytest.raises(B.IcnnError) as e:
        B._check(B._lib.iroute_top(None, *good, SP, 0))
    assert e.value.code == B.ICNN_E_NULL


# ---- sums of rows

@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 30), B.ICNN_E_SHAPE), (dict(v_rows=-1), B.ICNN_E_SHAPE), (dict(v_rows=1 << 31), B.ICNN_E_SHAPE), (dict(c=0), B.ICNN_E_SHAPE),
    (dict(c=(1 << 20) + 1), B.ICNN_E_SHAPE), (dict(top=0), B.ICNN_E_SHAPE), (dict(top=17), B.ICNN_E_SHAPE), (dict(v_stride=63), B.ICNN_E_SHAPE),
    (dict(res_stride=63), B.ICNN_E_SHAPE), (dict(y_stride=63), B.ICNN_E_SHAPE), (dict(dtype=B.ICNN_U8), B.ICNN_E_PARAM), (dict(v_dtype=B.ICNN_S32), B.ICNN_E_PARAM)])
def test_combine_descriptors(kw, want):
    d = B.combine_desc(**{**dict(rows=10, top=4, c=64), **kw})
    assert code(B.icombine_rows, d, X, G, P, R, Y) == want


def test_combine_pointers_and_overlaps():
    d = B.combine_desc(rows=10, top=4, c=64)
    good = [X, G, P, R, Y]
    assert accepted(B.icombine_rows, d, *good) and accepted(B.icombine_rows, d, X, G, P, None, Y) and accepted(B.icombine_rows, d, X, G, P, R, R)
    for k in range(5):
        if k != 3:
            assert code(B.icombine_rows, d, *[None if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_NULL, k
        assert code(B.icombine_rows, d, *[p + 1 if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_ALIGN, k
    for y in (X, X + 40 * 128 - 2, G + 12, P + 156, R + 2, R - 128):
        assert code(B.icombine_rows, d, X, G, P, R, y) == B.ICNN_E_UNSUPPORTED, y
    assert B.icombine_rows(B.combine_desc(rows=0, top=4, c=64), *[None] * 5, stream=0) == 0
    with pytest.raises(B.IcnnError) as e:
        B._check(B._lib.icombine_rows(None, *good, 0))
    assert e.value.code == B.ICNN_E_NULL


# ---- products grouped by expert

@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 31, x_rows=5), B.ICNN_E_SHAPE), (dict(x_rows=-1), B.ICNN_E_SHAPE), (dict(k=0), B.ICNN_E_SHAPE), (dict(k=131072), B.ICNN_E_SHAPE),
    (dict(n=0), B.ICNN_E_SHAPE), (dict(n=(1 << 22) + 1), B.ICNN_E_SHAPE), (dict(experts=0), B.ICNN_E_SHAPE), (dict(experts=1025), B.ICNN_E_SHAPE),
    (dict(x_stride=63), B.ICNN_E_SHAPE), (dict(w_stride=63), B.ICNN_E_SHAPE), (dict(y_stride=31), B.ICNN_E_SHAPE), (dict(expert_stride=2047), B.ICNN_E_SHAPE),
    (dict(w_stride=128, expert_stride=31 * 128 + 63), B.ICNN_E_SHAPE), (dict(expert_stride=1 << 41), B.ICNN_E_SHAPE), (dict(rows=1 << 24, n=1 << 13), B.ICNN_E_SHAPE),
    (dict(n=1 << 22, experts=1024, rows=1 << 11), B.ICNN_E_SHAPE), (dict(dtype=B.ICNN_S8), B.ICNN_E_PARAM), (dict(act=5), B.ICNN_E_PARAM), (dict(act=-1), B.ICNN_E_PARAM)])
def test_grouped_descriptors(kw, want):
    d = B.grouped_desc(**{**dict(rows=10, k=64, n=32, experts=4), **kw})
    assert code(B.igrouped_linear_s8, d, X, XS, IX, OF, W, WS, BI, Y) == want
    assert code(B.igrouped_gated_linear_s8, d, X, XS, IX, OF, W, WS, BI, W2, WS2, BI2, Y) == want


def test_grouped_pointers_and_overlaps():
    d = B.grouped_desc(rows=10, k=64, n=32, experts=4)
    good = [X, XS, IX, OF, W, WS, BI, Y]
    assert accepted(B.igrouped_linear_s8, d, *good) and accepted(B.igrouped_linear_s8, d, X + 1, XS, None, OF, W + 3, WS, None, Y)
    for k in (0, 1, 3, 4, 5, 7):
        assert code(B.igrouped_linear_s8, d, *[None if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_NULL, k
    for k in (1, 2, 3, 5, 6, 7):
        assert code(B.igrouped_linear_s8, d, *[p + 1 if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_ALIGN, k
    for y in (X, X + 638, XS + 36, IX + 36, OF + 16, W + 4 * 2048 - 2, WS + 4 * 128 - 4, BI + 4):
        assert code(B.igrouped_linear_s8, d, X, XS, IX, OF, W, WS, BI, y) == B.ICNN_E_UNSUPPORTED, y
    gated = [X, XS, IX, OF, W, WS, BI, W2, WS2, BI2, Y]
    assert accepted(B.igrouped_gated_linear_s8, d, *gated)
    for k in (0, 1, 3, 4, 5, 7, 8, 10):
        assert code(B.igrouped_gated_linear_s8, d, *[None if i == k else p for i, p in enumerate(gated)]) == B.ICNN_E_NULL, k
    for y in (W2 + 100, WS2, BI2 + 500):
        assert code(B.igrouped_gated_linear_s8, d, *gated[:-1], y) == B.ICNN_E_UNSUPPORTED, y
    fewer = B.grouped_desc(rows=10, x_rows=9, k=64, n=32, experts=4)
    assert code(B.igrouped_linear_s8, fewer, X, XS, None, OF, W, WS, BI, Y) == B.ICNN_E_SHAPE and accepted(B.igrouped_linear_s8, fewer, *good)
    assert B.igrouped_linear_s8(B.grouped_desc(rows=10, x_rows=0, k=64, n=32, experts=4), *good, stream=0) == 0
    for fn, n in ((B._lib.igrouped_linear_s8, 9), (B._lib.igrouped_gated_linear_s8, 12)):
        with pytest.raises(B.IcnnError) as e:
            B._check(fn(None, *[X] * (n - 1), 0))
        assert e.value.code == B.ICNN_E_NULL


# ---- weights of 4 bits

@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 31), B.ICNN_E_SHAPE), (dict(k=0), B.ICNN_E_SHAPE), (dict(k=131072), B.ICNN_E_SHAPE), (dict(n=0), B.ICNN_E_SHAPE),
    (dict(n=(1 << 22) + 1), B.ICNN_E_SHAPE), (dict(rows=1 << 26, n=256), B.ICNN_E_SHAPE), (dict(x_stride=63), B.ICNN_E_SHAPE), (dict(y_stride=31), B.ICNN_E_SHAPE),
    (dict(res_stride=31), B.ICNN_E_SHAPE), (dict(group=16), B.ICNN_E_PARAM), (dict(group=96), B.ICNN_E_PARAM), (dict(group=512), B.ICNN_E_PARAM), (dict(group=0), B.ICNN_E_PARAM),
    (dict(dtype=B.ICNN_S8), B.ICNN_E_PARAM), (dict(scale_dtype=B.ICNN_U8), B.ICNN_E_PARAM), (dict(act=5), B.ICNN_E_PARAM)])
def test_s4_descriptors(kw, want):
    d = B.linear_s4_desc(**{**dict(rows=10, k=64, n=32), **kw})
    assert code(B.ilinear_s4, d, X, XS, W, WS, BI, R, Y) == want
    if "res_stride" not in kw:
        assert code(B.igated_linear_s4, d, X, XS, W, WS, BI, W2, WS2, BI2, Y) == want


def test_s4_pointers_and_overlaps():
    d = B.linear_s4_desc(rows=10, k=64, n=32)
    good = [X, XS, W, WS, BI, R, Y]
    assert accepted(B.ilinear_s4, d, *good) and accepted(B.ilinear_s4, d, X + 1, XS, W, WS + 2, None, None, Y) and accepted(B.ilinear_s4, d, X, XS, W, WS, BI, R, R)
    for k in (0, 1, 2, 3, 6):
        assert code(B.ilinear_s4, d, *[None if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_NULL, k
    for k, by in ((1, 2), (2, 8), (3, 1), (4, 2), (5, 1), (6, 1)):
        assert code(B.ilinear_s4, d, *[p + by if i == k else p for i, p in enumerate(good)]) == B.ICNN_E_ALIGN, k
    for y in (X, X + 638, W + 1022, XS + 36, WS + 62, BI + 64, R + 2, R - 64):
        assert code(B.ilinear_s4, d, X, XS, W, WS, BI, R, y) == B.ICNN_E_UNSUPPORTED, y
    gated = [X, XS, W, WS, BI, W2, WS2, BI2, Y]
    for k in (0, 1, 2, 3, 5, 6, 8):
        assert code(B.igated_linear_s4, d, *[None if i == k else p for i, p in enumerate(gated)]) == B.ICNN_E_NULL, k
    for y in (W2 + 16, WS2, BI2):
        assert code(B.igated_linear_s4, d, *gated[:-1], y) == B.ICNN_E_UNSUPPORTED, y
    for fn, n in ((B._lib.ilinear_s4, 8), (B._lib.igated_linear_s4, 10)):
        with pytest.raises(B.IcnnError) as e:
            B._check(fn(None, *[X] * (n - 1), 0))
        assert e.value.code == B.ICNN_E_NULL


def test_quantising_to_4_bits():
    assert B.iweights_s4_bytes(3, 1) == 48 and B.iweights_s4_bytes(5, 64) == 160 and B.iweights_s4_bytes(1, 65) == 48
    assert size_code(B.iweights_s4_bytes, 0, 5) == B.ICNN_E_SHAPE and size_code(B.iweights_s4_bytes, 5, 1 << 20) == B.ICNN_E_SHAPE
    for kw, want in ((dict(n=0), B.ICNN_E_SHAPE), (dict(k=0), B.ICNN_E_SHAPE), (dict(w_stride=63), B.ICNN_E_SHAPE), (dict(n=1 << 22, k=131071), B.ICNN_E_SHAPE),
                     (dict(group=31), B.ICNN_E_PARAM), (dict(dtype=B.ICNN_S8), B.ICNN_E_PARAM), (dict(scale_dtype=-1), B.ICNN_E_PARAM)):
        assert code(B.iquantize_weights_s4, B.quantize_s4_desc(**{**dict(n=32, k=64), **kw}), X, W, WS) == want, kw
    d = B.quantize_s4_desc(n=32, k=64)
    assert accepted(B.iquantize_weights_s4, d, X, W, WS)
    for k, by in ((0, 2), (1, 8), (2, 1)):
        args = [X, W, WS]
        args[k] += by
        assert code(B.iquantize_weights_s4, d, *args) == B.ICNN_E_ALIGN
        args[k] = None
        assert code(B.iquantize_weights_s4, d, *args) == B.ICNN_E_NULL
    for args in ((X, X + 16, WS), (X, W, X + 100), (X, W, W + 1020)):
        assert code(B.iquantize_weights_s4, d, *args) == B.ICNN_E_UNSUPPORTED, args


def test_lists_of_calls_refuse_as_the_calls_do():
    grouped, s4 = B.grouped_desc(rows=10, k=64, n=32, experts=4), B.linear_s4_desc(rows=10, k=64, n=32)
    for call in (("route", (B.route_desc(rows=10, experts=64, top=4), X, W, None, P, T, OF, None)), ("combine", (B.combine_desc(rows=10, top=4, c=64), X, None, P, R, Y)),
                 ("grouped_linear", (grouped, X, XS, None, None, W, WS, BI, Y)), ("grouped_gated_linear", (grouped, X, XS, IX, OF, W, WS, BI, None, WS2, BI, Y)),
                 ("linear_s4", (s4, X, XS, W, None, BI, R, Y)), ("gated_linear_s4", (s4, X, XS, W, WS, BI, W2, None, BI, Y))):
        with pytest.raises(B.IcnnError) as e:
            B.Calls([call]).run(stream=0)
        assert e.value.code == B.ICNN_E_NULL, call[0]
    nothing = [("combine", (B.combine_desc(rows=0, top=4, c=64), *[None] * 5)), ("grouped_linear", (B.grouped_desc(rows=0, k=64, n=32, experts=4), *[None] * 8)),
               ("grouped_gated_linear", (B.grouped_desc(rows=0, k=64, n=32, experts=4), *[None] * 11)), ("linear_s4", (B.linear_s4_desc(rows=0, k=64, n=32), *[None] * 7)),
               ("gated_linear_s4", (B.linear_s4_desc(rows=0, k=64, n=32), *[None] * 9))]
    B.Calls(nothing).run(stream=0)


def test_blocks_refuse_shapes_that_do_not_fit():
    import torch
    from paper_2006_11735_amd.ffn import ExpertsFeedForward, FeedForward
    z = torch.zeros
    good = dict(gamma=z(8), w_router=z(4, 8), w_gate=z(4, 16, 8), w_up=z(4, 16, 8), w_down=z(4, 8, 16), rows=4, top=2)
    for kw in (dict(gamma=z(9)), dict(w_router=z(8, 4)), dict(w_gate=z(16, 8)), dict(w_up=z(4, 16, 9)), dict(w_down=z(4, 16, 8)), dict(b_router=z(5)), dict(b_gate=z(4, 8)),
               dict(b_down=z(8)), dict(w_up=None, b_up=z(4, 16)), dict(act="tanh"), dict(dtype=torch.float64), dict(rows=0), dict(top=0), dict(top=5), dict(score="linear")):
        with pytest.raises(ValueError):
            ExpertsFeedForward(**{**good, **kw})
    good = dict(gamma=z(8), w_gate=z(16, 8), w_up=z(16, 8), w_down=z(8, 16), rows=4)
    for kw in (dict(bits=2), dict(bits=4, group=48), dict(bits=4, scale_dtype=torch.int8)):
        with pytest.raises(ValueError):
            FeedForward(**{**good, **kw})
