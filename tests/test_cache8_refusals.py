"""What rotary positions and the operators over a paged cache of codes refuse on the host (no GPU needed; addresses are never followed)."""
import ctypes
import math

import pytest

P = 0x10000          # an aligned address that nothing reads


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import build
    build.build()
    from paper_2503_18893_b200 import xkv as m
    return m


def config(x, **over):
    kw = dict(G=2, batch=3, H_kv=2, H_q=8, d_h=128, page=16, n_pages=40, max_pages=12)
    kw.update(over)
    return x.make_cache8_config(**kw)


def calls(x, cfg, **over):
    a = dict(l0=0, l1=2, n=8, new=4, cap=16, q=P, k=P, v=P, K=P, V=P, K8=P, V8=P, ks=P, vs=P, table=P, len=P, slot=P, pos=P, first=P, held=P,
             want=P, ring=P, state=P, ws=P, ws_bytes=1 << 40, out=P, lse=P, flags=P)
    a.update(over)
    c, L = ctypes.byref(cfg) if cfg is not None else None, x._lib
    return dict(
        assign=L.xkv_page_assign(c, a["held"], a["want"], a["table"], a["ring"], a["state"], a["first"], a["len"], a["pos"], a["slot"], a["n"],
                                 a["flags"], None),
        append=L.xkv_cache8_append(c, a["l0"], a["l1"], a["k"], a["v"], a["slot"], a["n"], a["K8"], a["V8"], a["ks"], a["vs"], a["flags"], None),
        read=L.xkv_cache8_read(c, a["l0"], a["l1"], a["table"], a["len"], a["K8"], a["V8"], a["ks"], a["vs"], a["cap"], a["K"], a["V"], a["flags"],
                               None),
        attend=L.xkv_cache8_attend(c, a["l0"], a["l1"], a["q"], a["first"], a["n"], a["new"], a["table"], a["len"], a["K8"], a["V8"], a["ks"],
                                   a["vs"], a["ws"], a["ws_bytes"], a["out"], a["lse"], a["flags"], None))


ALL = {"assign", "append", "read", "attend"}
CODES = {"append", "read", "attend"}


@pytest.mark.parametrize("over", [dict(G=0), dict(batch=0), dict(H_kv=0), dict(H_q=7), dict(H_q=2 * 17), dict(d_h=96), dict(page=8), dict(page=48),
                                  dict(page=256), dict(n_pages=0), dict(max_pages=0), dict(max_pages=(1 << 18) + 1), dict(softmax_scale=-1.0),
                                  dict(softmax_scale=math.inf), dict(softmax_scale=math.nan)])
def test_configurations(xkv, over):
    assert set(calls(xkv, config(xkv, **over)).values()) == {xkv.XKV_ERR_INVALID_ARG}
    with pytest.raises(xkv.XKVError):
        xkv.xkv_cache8_workspace_bytes(config(xkv, **over), 4)


def test_struct_size_and_null(xkv):
    cfg = config(xkv)
    cfg.struct_size = 8
    assert set(calls(xkv, cfg).values()) == {xkv.XKV_ERR_INVALID_ARG}
    assert set(calls(xkv, None).values()) == {xkv.XKV_ERR_INVALID_ARG}


def test_sizes_beyond_32_bits(xkv):
    assert set(calls(xkv, config(xkv, batch=40000)).values()) == {xkv.XKV_ERR_UNSUPPORTED}
    assert set(calls(xkv, config(xkv, n_pages=(1 << 25) + 1)).values()) == {xkv.XKV_ERR_UNSUPPORTED}
    assert calls(xkv, config(xkv, batch=300), cap=1 << 22)["read"] == xkv.XKV_ERR_UNSUPPORTED
    assert calls(xkv, config(xkv), n=(1 << 27))["attend"] == xkv.XKV_ERR_UNSUPPORTED


@pytest.mark.parametrize("over,who", [
    (dict(l0=-1), CODES), (dict(l1=3), CODES), (dict(l0=1, l1=1), CODES), (dict(n=-1), {"assign", "append", "attend"}), (dict(n=3), {"attend"}),
    (dict(new=0), {"attend"}), (dict(new=9), {"attend"}), (dict(cap=0), {"read"}), (dict(cap=(1 << 22) + 1), {"read"}),
    (dict(first=None), {"assign", "attend"}), (dict(q=None), {"attend"}), (dict(q=P + 8), {"attend"}), (dict(k=None), {"append"}), (dict(k=P + 8), {"append"}),
    (dict(v=None), {"append"}), (dict(v=P + 2), {"append"}), (dict(K=None, V=None), {"read"}), (dict(K=P + 8), {"read"}), (dict(V=P + 8), {"read"}),
    (dict(K8=None), CODES), (dict(K8=P + 8), CODES), (dict(V8=None), CODES), (dict(V8=P + 4), CODES), (dict(ks=None), CODES), (dict(vs=P + 2), CODES),
    (dict(table=None), {"assign", "read", "attend"}), (dict(table=P + 2), {"assign", "read", "attend"}), (dict(len=None), {"assign", "read", "attend"}),
    (dict(slot=None), {"assign", "append"}), (dict(slot=P + 1), {"assign", "append"}), (dict(pos=None), {"assign"}), (dict(pos=None, slot=None), {"assign", "append"}),
    (dict(held=None), {"assign"}), (dict(want=None), {"assign"}), (dict(ring=None), {"assign"}), (dict(state=None), {"assign"}), (dict(state=P + 2), {"assign"}),
    (dict(ws=None), {"attend"}), (dict(ws=P + 4), {"attend"}), (dict(ws_bytes=1), {"attend"}), (dict(out=None), {"attend"}), (dict(out=P + 2), {"attend"}),
    (dict(lse=P + 2), {"attend"}), (dict(flags=P + 2), ALL)])
def test_arguments(xkv, over, who):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls that are not refused would run")
    for name, st in calls(xkv, config(xkv), **over).items():
        if name in who:
            assert st == xkv.XKV_ERR_INVALID_ARG, (name, st)
        else:                                          # passes the checks, and then finds no device
            assert st in (xkv.XKV_ERR_CUDA, xkv.XKV_ERR_ARCH), (name, st)


ROPE = dict(d_h=128)


@pytest.mark.parametrize("over", [dict(d_h=0), dict(d_h=127), dict(d_h=1026), dict(rot=0), dict(rot=3), dict(rot=130), dict(d_h=512, rot=258),
                                  dict(base=0.0), dict(base=-1.0), dict(base=math.nan), dict(base=math.inf), dict(gain=-1.0), dict(gain=math.inf),
                                  dict(scaling="linear", factor=0.0), dict(scaling="ntk", factor=2.0, rot=2), dict(scaling="llama3", factor=8.0),
                                  dict(scaling="llama3", factor=8.0, original=8192.0, low=4.0, high=4.0), dict(scaling="yarn", factor=4.0),
                                  dict(scaling="yarn", factor=4.0, original=4096.0, beta_fast=0.0), dict(scaling="yarn", factor=4.0, original=4096.0, base=1.0),
                                  dict(scaling="yarn", factor=1e-5, original=4096.0)])
def test_rotations_that_are_refused(xkv, over):
    with pytest.raises(xkv.XKVError):
        xkv.make_rope(**{**ROPE, **over})


def test_words_that_are_not_known(xkv):
    for kw in (dict(layout="other"), dict(scaling="dynamic")):
        with pytest.raises(ValueError):
            xkv.make_rope(d_h=64, **kw)
    with pytest.raises(ValueError):
        xkv.xkv_rope(xkv.make_rope(d_h=64), None, None, direction="back")


def test_frequencies(xkv):
    """Turns per position against the formulas: to the precision of 64-bit arithmetic, and of a fraction in steps of 2^-64 (off by half
    a step, 2^-65, whatever the frequency)."""
    from tests import _cache8_ref as R
    for scaling in xkv.XKV_ROPE_SCALINGS:
        for rot in (4, 64, 128, 256):
            kw = dict(base=500000.0, factor=8.0, original=8192.0) if scaling != "none" else {}
            plan = xkv.make_rope(d_h=256, rot=rot, scaling=scaling, **kw)
            f, gain = R.frequencies(rot, scaling=scaling, **kw)
            assert abs(plan.gain - gain) <= 2.0 ** -23 * gain
            for i in range(rot // 2):
                assert abs(plan.turns[i] * 2.0 ** -64 - float(f[i]) / (2 * math.pi)) <= 2.0 ** -49 * float(f[i]) + 2.0 ** -65
            assert not any(plan.turns[rot // 2:])
    assert xkv.make_rope(d_h=64, scaling="yarn", factor=4.0, original=4096.0, gain=1.0).gain == 1.0


def test_rope_arguments(xkv):
    L, plan = xkv._lib, xkv.make_rope(d_h=64)

    def call(direction=0, kind=0, n=1, rows=6, pos=P, n_pos=3, plan=plan, **t):
        kw = dict(x=P, y=P + 65536, x_row=64, x_head=64, y_row=64, y_head=64, heads=1)
        kw.update(t)
        ts = (xkv.xkv_rope_tensor * 2)(xkv.xkv_rope_tensor(**kw), xkv.xkv_rope_tensor(**kw))
        return L.xkv_rope(ctypes.byref(plan) if plan is not None else None, direction, kind, ts, n, rows, pos, n_pos, None)

    for kw in (dict(plan=None), dict(direction=3), dict(direction=-1), dict(kind=3), dict(n=0), dict(n=3), dict(rows=-1), dict(rows=7), dict(n_pos=0),
               dict(pos=None), dict(pos=P + 2), dict(x=None), dict(y=None), dict(x=P + 1), dict(kind=2, x=P + 2), dict(heads=-1),
               dict(y=P, y_row=128), dict(y=P, y_head=128)):
        assert call(**kw) == xkv.XKV_ERR_INVALID_ARG, kw
    assert call(rows=3 << 30, heads=2) == xkv.XKV_ERR_UNSUPPORTED
    for field, value in (("struct_size", 4), ("rot", 300), ("rot", 7), ("layout", 2), ("gain", -1.0)):
        p = xkv.make_rope(d_h=64)
        setattr(p, field, value)
        assert call(plan=p) == xkv.XKV_ERR_INVALID_ARG, field


def test_the_binding_checks_tensors(xkv):
    import torch
    cfg, t = config(xkv), torch.zeros(4)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="held: the tensor"):
        xkv.xkv_page_assign(cfg, t, i, i, i, i, None, i)
    with pytest.raises(ValueError, match="current CUDA device"):
        xkv.xkv_page_assign(cfg, i, i, i, i, i, None, i)
    with pytest.raises(ValueError, match="k: the tensor"):
        xkv.xkv_cache8_append(cfg, 0, 2, t, t, i, t, t, t, t)
    with pytest.raises(ValueError, match="neither"):
        xkv.xkv_cache8_read(cfg, 0, 2, i, i, t, t, t, t, None, None)
    with pytest.raises(ValueError, match="q: the tensor"):
        xkv.xkv_cache8_attend(cfg, 0, 2, torch.zeros((2, 3, 8, 128)), None, 1, i, i, t, t, t, t, t, t)
    plan = xkv.make_rope(d_h=64)
    with pytest.raises(ValueError, match="pos: the tensor"):
        xkv.xkv_rope(plan, torch.zeros((3, 1, 64)), torch.zeros(3))
    with pytest.raises(ValueError, match="current CUDA device"):
        xkv.xkv_rope(plan, torch.zeros((3, 1, 64)), i)


def test_workspace_bytes(xkv):
    cfg = config(xkv)
    assert xkv.xkv_cache8_workspace_bytes(cfg, 1) > 0
    with pytest.raises(xkv.XKVError):
        xkv.xkv_cache8_workspace_bytes(cfg, 0)
