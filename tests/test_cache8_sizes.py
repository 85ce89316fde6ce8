"""Sizes and factors at the ends of what rotary positions and the operators over a paged cache of codes take (no GPU needed)."""
import ctypes

import pytest

from tests.test_cache8_refusals import P, calls, config, xkv  # noqa: F401  (the fixture)


def rope(x, heads, rows=1, d_h=2, n=2):
    ts = (x.xkv_rope_tensor * 2)(*(x.xkv_rope_tensor(x=P, y=P, x_row=0, x_head=d_h, y_row=0, y_head=d_h, heads=h) for h in heads))
    return x._lib.xkv_rope(ctypes.byref(x.make_rope(d_h=d_h)), 0, 0, ts, n, rows, P, 1, None)


@pytest.fixture()
def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls that are not refused would run")


def test_heads_of_both_tensors_together(xkv, no_gpu):  # noqa: F811
    fits = (xkv.XKV_ERR_CUDA, xkv.XKV_ERR_ARCH)          # passes the checks, and then finds no device
    assert rope(xkv, (1 << 30, 1 << 30)) == xkv.XKV_ERR_UNSUPPORTED
    assert rope(xkv, ((1 << 31) - 1, 0), n=1) == xkv.XKV_ERR_UNSUPPORTED
    assert rope(xkv, ((1 << 31) - 1025, 1)) == xkv.XKV_ERR_UNSUPPORTED
    assert rope(xkv, ((1 << 31) - 1026, 1)) in fits
    assert rope(xkv, (1 << 30, (1 << 30) - 1025)) in fits
    assert rope(xkv, (1 << 10, 1 << 10), rows=(1 << 21) - 1) in fits


def test_tokens_of_an_append(xkv, no_gpu):  # noqa: F811
    cfg = config(xkv)                                    # G * H_q = 16
    assert calls(xkv, cfg, n=1 << 27)["append"] == xkv.XKV_ERR_UNSUPPORTED
    assert calls(xkv, cfg, n=(1 << 27) - 1)["append"] in (xkv.XKV_ERR_CUDA, xkv.XKV_ERR_ARCH)
    assert calls(xkv, cfg, n=1 << 27)["assign"] in (xkv.XKV_ERR_CUDA, xkv.XKV_ERR_ARCH)


def test_a_gain_that_the_inverse_cannot_divide_by(xkv):  # noqa: F811
    for gain in (1e-39, 1e-45, 1e39):
        with pytest.raises(xkv.XKVError):
            xkv.make_rope(d_h=64, gain=gain)
    for gain in (1e-37, 1e38):
        assert xkv.make_rope(d_h=64, gain=gain).gain == ctypes.c_float(gain).value
    plan = xkv.make_rope(d_h=64)
    t = xkv.xkv_rope_tensor(x=P, y=P, x_row=64, x_head=64, y_row=64, y_head=64, heads=1)
    for plan.gain in (1e-39, float("inf"), float("nan"), 0.0):
        assert xkv._lib.xkv_rope(ctypes.byref(plan), 2, 0, ctypes.byref(t), 1, 1, P, 1, None) == xkv.XKV_ERR_INVALID_ARG
