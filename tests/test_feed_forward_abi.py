"""What the feed-forward operators refuse, on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2006_11735_amd import binding as B


def code(fn, *args):
    with pytest.raises(B.IcnnError) as e:
        fn(*args, stream=0)
    assert B.icnn_last_error() != ""
    return e.value.code


def accepted(fn, *args):
    """No refusal: the launch itself fails where there is no GPU (where there is one, nothing is launched on these addresses)."""
    return torch.cuda.is_available() or code(fn, *args) == B.ICNN_E_LAUNCH


X, R, G, S, Q, SC = (k << 24 for k in range(1, 7))


def test_the_descriptors_have_the_layout_of_the_header():
    assert ctypes.sizeof(B.icnn_norm_desc) == 5 * 8 + 4 * 4 and ctypes.sizeof(B.icnn_linear_desc) == 5 * 8 + 4 * 4
    d = B.norm_desc(rows=3, c=40, dtype=B.ICNN_F16, x_stride=48)
    assert (d.x_stride, d.res_stride, d.q_stride, d.gamma_dtype) == (48, 40, 40, B.ICNN_F16) and abs(d.eps - 1e-5) < 1e-12
    d = B.linear_desc(rows=3, k=40, n=8, y_stride=9)
    assert (d.x_stride, d.w_stride, d.res_stride, d.y_stride, d.dtype) == (40, 40, 8, 9, B.ICNN_BF16)
    with pytest.raises(AttributeError):
        B.linear_desc(colour=1)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 31), B.ICNN_E_SHAPE), (dict(c=0), B.ICNN_E_SHAPE), (dict(c=(1 << 20) + 1), B.ICNN_E_SHAPE),
    (dict(x_stride=63), B.ICNN_E_SHAPE), (dict(res_stride=63), B.ICNN_E_SHAPE), (dict(sum_stride=0), B.ICNN_E_SHAPE), (dict(q_stride=-64), B.ICNN_E_SHAPE),
    (dict(x_stride=1 << 41), B.ICNN_E_SHAPE), (dict(rows=1 << 20, x_stride=1 << 25), B.ICNN_E_SHAPE),
    (dict(dtype=B.ICNN_U8), B.ICNN_E_PARAM), (dict(dtype=6), B.ICNN_E_PARAM), (dict(dtype=B.ICNN_F32, gamma_dtype=B.ICNN_F16), B.ICNN_E_PARAM),
    (dict(eps=-1e-9), B.ICNN_E_PARAM), (dict(eps=float("nan")), B.ICNN_E_PARAM), (dict(eps=float("inf")), B.ICNN_E_PARAM)])
def test_norm_descriptors(kw, want):
    d = B.norm_desc(**{**dict(rows=10, c=64), **kw})
    assert code(B.irms_norm_s8, d, X, R, G, S, Q, SC) == want
    if not set(kw) & {"res_stride", "sum_stride", "gamma_dtype", "eps"}:
        assert code(B.iquantize_rows_s8, d, X, Q, SC) == want


def test_norm_pointers_and_overlaps():
    d = B.norm_desc(rows=10, c=64)
    for k in (0, 2, 4, 5):                                    # (the residual and the sum may be absent)
        args = [X, R, G, S, Q, SC]
        args[k] = None
        assert code(B.irms_norm_s8, d, *args) == B.ICNN_E_NULL, k
    for k in (0, 1, 2, 3, 5):
        args = [X, R, G, S, Q, SC]
        args[k] += 1
        assert code(B.irms_norm_s8, d, *args) == B.ICNN_E_ALIGN, k
    for args in ([X, R, G, S, X, SC], [X, R, G, S, Q, X + 1276], [X, R, G, X + 2, Q, SC], [X, R, G, R + 128, Q, SC], [X, R, G, Q, Q, SC], [X, R, G, S, Q, Q + 636],
                 [X, R, G, G, Q, SC], [X, R, G, S, R, SC], [X, R, G, S, G + 126, SC], [X, R, G, S, S + 1, SC]):
        assert code(B.irms_norm_s8, d, *args) == B.ICNN_E_UNSUPPORTED, args
    wider = B.norm_desc(rows=10, c=64, sum_stride=128)
    assert code(B.irms_norm_s8, wider, X, R, G, X, Q, SC) == B.ICNN_E_UNSUPPORTED       # in place with another stride
    halves = B.norm_desc(rows=10, c=64, x_stride=128, sum_stride=128, res_stride=128)
    assert accepted(B.irms_norm_s8, halves, X, R, G, X + 128, Q, SC)                    # the other half of a buffer's rows
    assert accepted(B.irms_norm_s8, d, X, R, G, X, Q, SC) and accepted(B.irms_norm_s8, d, X, R, G, R, Q, SC) and accepted(B.irms_norm_s8, d, X, None, G, None, Q, SC)
    assert code(B.iquantize_rows_s8, d, None, Q, SC) == B.ICNN_E_NULL and code(B.iquantize_rows_s8, d, X, Q, None) == B.ICNN_E_NULL
    assert code(B.iquantize_rows_s8, d, X, X + 1270, SC) == B.ICNN_E_UNSUPPORTED and code(B.iquantize_rows_s8, d, X, Q, Q) == B.ICNN_E_UNSUPPORTED
    with pytest.raises(B.IcnnError) as e:
        B._check(B._lib.irms_norm_s8(None, X, R, G, S, Q, SC, 0))
    assert e.value.code == B.ICNN_E_NULL


W, WS, BI, Y, W2, WS2 = (k << 24 for k in range(11, 17))


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.ICNN_E_SHAPE), (dict(rows=1 << 31), B.ICNN_E_SHAPE), (dict(k=0), B.ICNN_E_SHAPE), (dict(n=0), B.ICNN_E_SHAPE), (dict(n=(1 << 31) - 1, y_stride=1 << 31), B.ICNN_E_SHAPE), (dict(k=131072), B.ICNN_E_SHAPE),
    (dict(x_stride=63), B.ICNN_E_SHAPE), (dict(w_stride=63), B.ICNN_E_SHAPE), (dict(y_stride=31), B.ICNN_E_SHAPE), (dict(res_stride=31), B.ICNN_E_SHAPE),
    (dict(w_stride=1 << 41), B.ICNN_E_SHAPE), (dict(rows=1 << 30, y_stride=1 << 20), B.ICNN_E_SHAPE),
    (dict(dtype=B.ICNN_S8), B.ICNN_E_PARAM), (dict(dtype=-1), B.ICNN_E_PARAM), (dict(act=5), B.ICNN_E_PARAM), (dict(act=-1), B.ICNN_E_PARAM)])
def test_linear_descriptors(kw, want):
    d = B.linear_desc(**{**dict(rows=10, k=64, n=32), **kw})
    assert code(B.ilinear_s8, d, X, SC, W, WS, BI, R, Y) == want
    if "res_stride" not in kw:
        assert code(B.igated_linear_s8, d, X, SC, W, WS, BI, W2, WS2, None, Y) == want
        with pytest.raises(B.IcnnError) as e:
            B.ilinear_s8_workspace_bytes(d)
        assert e.value.code == want
        with pytest.raises(B.IcnnError) as e:
            B.igated_linear_s8_workspace_bytes(d)
        assert e.value.code == want


def test_linear_pointers_and_overlaps():
    d = B.linear_desc(rows=10, k=64, n=32)
    for k in (0, 1, 2, 3, 6):
        args = [X, SC, W, WS, BI, R, Y]
        args[k] = None
        assert code(B.ilinear_s8, d, *args) == B.ICNN_E_NULL, k
    for k in (1, 3, 4, 5, 6):
        args = [X, SC, W, WS, BI, R, Y]
        args[k] += 1
        assert code(B.ilinear_s8, d, *args) == B.ICNN_E_ALIGN, k
    assert code(B.ilinear_s8, d, X, SC, W, WS, BI, R, Y, G + 8) == B.ICNN_E_ALIGN
    for y in (X, X + 638, X - 638, W, SC + 36, WS, BI + 64, R + 2, R - 64):
        assert code(B.ilinear_s8, d, X, SC, W, WS, BI, R, y) == B.ICNN_E_UNSUPPORTED, y
    assert accepted(B.ilinear_s8, d, X, SC, W, WS, BI, R, R) and accepted(B.ilinear_s8, d, X + 1, SC, W + 3, WS, None, None, Y)
    for k in (0, 1, 2, 3, 5, 6, 8):
        args = [X, SC, W, WS, BI, W2, WS2, BI, Y]
        args[k] = None
        assert code(B.igated_linear_s8, d, *args) == B.ICNN_E_NULL, k
    for y in (X, W, W2 + 2046, WS2, BI + 126):
        assert code(B.igated_linear_s8, d, X, SC, W, WS, None, W2, WS2, BI, y) == B.ICNN_E_UNSUPPORTED, y
    with pytest.raises(B.IcnnError) as e:
        B._check(B._lib.ilinear_s8(None, X, SC, W, WS, BI, R, Y, None, 0))
    assert e.value.code == B.ICNN_E_NULL


def test_lists_of_calls_refuse_as_the_calls_do():
    norm, linear = B.norm_desc(rows=10, c=64), B.linear_desc(rows=10, k=64, n=32)
    for call in (("rms_norm", (norm, X, R, None, S, Q, SC)), ("quantize_rows", (norm, None, Q, SC)), ("linear", (linear, X, SC, W, WS, BI, R, None, None)),
                 ("gated_linear", (linear, X, SC, W, WS, BI, None, WS2, BI, Y, None))):
        with pytest.raises(B.IcnnError) as e:
            B.Calls([call]).run(stream=0)
        assert e.value.code == B.ICNN_E_NULL, call[0]
    nothing = [("rms_norm", (B.norm_desc(rows=0, c=64), None, None, None, None, None, None)), ("quantize_rows", (B.norm_desc(rows=0, c=64), None, None, None)),
               ("linear", (B.linear_desc(rows=0, k=64, n=32), *[None] * 8)), ("gated_linear", (B.linear_desc(rows=0, k=64, n=32), *[None] * 10))]
    B.Calls(nothing).run(stream=0)
    missing = B.icnn_call(kind=B.ICNN_CALL_LINEAR)
    with pytest.raises(B.IcnnError) as e:
        B._check(B._lib.icnn_run_calls(1, ctypes.byref(missing), 0))
    assert e.value.code == B.ICNN_E_NULL


def test_a_block_refuses_shapes_that_do_not_fit():
    from paper_2006_11735_amd.ffn import FeedForward
    z = torch.zeros
    good = dict(gamma=z(8), w_gate=z(16, 8), w_up=z(16, 8), w_down=z(8, 16), rows=4)
    for kw in (dict(gamma=z(9)), dict(w_up=z(16, 9)), dict(w_down=z(16, 8)), dict(b_gate=z(8)), dict(b_down=z(16)), dict(w_up=None, b_up=z(16)), dict(act="tanh"),
               dict(dtype=torch.float64), dict(rows=0)):
        with pytest.raises(ValueError):
            FeedForward(**{**good, **kw})


def test_workspaces_are_asked_for_where_k_is_long_and_outputs_are_few():
    size = lambda **kw: B.ilinear_s8_workspace_bytes(B.linear_desc(**kw))  # noqa: E731
    assert size(rows=64, k=16384, n=512) > 4096 and size(rows=1, k=16384, n=512) == 0 and size(rows=4096, k=16384, n=4096) == 0
    assert size(rows=64, k=256, n=512) == 0 and size(rows=0, k=16384, n=512) == 0
    try:
        B.icnn_set_tuning("ff_split", 1)
        assert size(rows=64, k=16384, n=512) == 0
    finally:
        B.icnn_set_tuning("reset")
