"""What the operators over an uncompressed cache refuse on the host (no GPU needed; addresses are never followed)."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import build
    build.build()
    from paper_2503_18893_b200 import xkv as m
    return m


P = 0x10000          # an aligned address that nothing reads


def calls(x, cfg, **over):
    """Status of every entry point with good arguments but for `over`."""
    a = dict(l0=0, l1=2, n=8, keep=16, q=P, K=P, V=P, ws=P, ws_bytes=1 << 40, out=P, lse=P, len=P, path=P, path_len=P, pos=P, first=P, mask=P,
             draft=P, vis=P, seen=P, decay=1.0, w=P, src=P, since=P, flags=P)
    a.update(over)
    c, L = ctypes.byref(cfg) if cfg is not None else None, x._lib
    return dict(
        attend=L.xkv_tree_attend(c, a["l0"], a["l1"], a["q"], a["n"], a["mask"], a["draft"], a["K"], a["V"], a["len"], a["ws"], a["ws_bytes"],
                                 a["out"], a["lse"], a["flags"], None),
        commit=L.xkv_tree_commit(c, a["l0"], a["l1"], a["K"], a["V"], a["len"], a["path"], a["path_len"], a["n"], a["pos"], a["first"], a["flags"], None),
        weigh=L.xkv_cache_weigh(c, a["l0"], a["l1"], a["q"], a["n"], a["lse"], a["K"], a["len"], a["vis"], a["seen"], a["decay"], a["w"], a["flags"], None),
        select=L.xkv_evict_select(c, a["l0"], a["l1"], a["w"], a["pos"], a["since"], a["len"], a["keep"], a["src"], a["flags"], None),
        compact=L.xkv_evict_compact(c, a["l0"], a["l1"], a["K"], a["V"], a["src"], a["keep"], a["w"], a["pos"], a["flags"], None))


def config(x, **over):
    kw = dict(G=2, batch=1, H_kv=2, H_q=8, d_h=128, cap=100)
    kw.update(over)
    return x.make_cache_config(**kw)


ALL = {"attend", "commit", "weigh", "select", "compact"}


@pytest.mark.parametrize("over", [dict(G=0), dict(batch=0), dict(H_kv=0), dict(H_q=7), dict(H_q=2 * 17), dict(d_h=96), dict(d_h=256), dict(cap=0),
                                  dict(cap=(1 << 22) + 1), dict(softmax_scale=-1.0), dict(softmax_scale=math.inf), dict(softmax_scale=math.nan)])
def test_configurations(xkv, over):
    got = calls(xkv, config(xkv, **over))
    assert set(got.values()) == {xkv.XKV_ERR_INVALID_ARG}, got
    with pytest.raises(xkv.XKVError):
        xkv.xkv_tree_workspace_bytes(config(xkv, **over), 4)


def test_struct_size_and_null(xkv):
    cfg = config(xkv)
    cfg.struct_size = 8
    assert set(calls(xkv, cfg).values()) == {xkv.XKV_ERR_INVALID_ARG}
    assert set(calls(xkv, None).values()) == {xkv.XKV_ERR_INVALID_ARG}


def test_sizes_beyond_32_bits(xkv):
    assert set(calls(xkv, config(xkv, batch=40000)).values()) == {xkv.XKV_ERR_UNSUPPORTED}
    assert set(calls(xkv, config(xkv, batch=300, cap=1 << 22)).values()) == {xkv.XKV_ERR_UNSUPPORTED}
    big = config(xkv, cap=xkv.XKV_EVICT_MAX_ROWS + 1)
    assert calls(xkv, big)["select"] == xkv.XKV_ERR_UNSUPPORTED


@pytest.mark.parametrize("over,who", [
    (dict(l0=-1), ALL), (dict(l1=3), ALL), (dict(l0=1, l1=1), ALL), (dict(l0=2, l1=1), ALL),
    (dict(n=0), {"attend", "commit", "weigh"}), (dict(n=257), {"attend", "commit", "weigh"}), (dict(n=101), {"attend"}),
    (dict(keep=0), {"select", "compact"}), (dict(keep=101), {"select", "compact"}),
    (dict(q=None), {"attend", "weigh"}), (dict(q=P + 8), {"attend", "weigh"}), (dict(K=None), {"attend", "commit", "weigh", "compact"}),
    (dict(K=P + 2), {"attend", "commit", "weigh", "compact"}), (dict(V=None), {"attend", "commit", "compact"}), (dict(V=P + 8), {"attend", "commit", "compact"}),
    (dict(ws=None), {"attend"}), (dict(ws=P + 4), {"attend"}), (dict(ws_bytes=1000), {"attend"}), (dict(out=None), {"attend"}), (dict(out=P + 2), {"attend"}),
    (dict(lse=P + 2), {"attend", "weigh"}), (dict(lse=None), {"weigh"}), (dict(len=None), {"commit"}), (dict(len=P + 1), {"attend", "commit", "weigh", "select"}),
    (dict(path=None), {"commit"}), (dict(path=P + 2), {"commit"}), (dict(path_len=P + 1), {"commit"}), (dict(first=None), {"commit"}),
    (dict(pos=P + 2), {"commit", "select", "compact"}), (dict(mask=P + 2), {"attend"}), (dict(draft=P + 2), {"attend"}), (dict(vis=P + 2), {"weigh"}),
    (dict(seen=P + 3), {"weigh"}), (dict(decay=-0.1), {"weigh"}), (dict(decay=1.5), {"weigh"}), (dict(decay=math.nan), {"weigh"}),
    (dict(w=None), {"weigh", "select"}), (dict(w=P + 2), {"weigh", "select", "compact"}), (dict(src=None), {"select", "compact"}),
    (dict(src=P + 2), {"select", "compact"}), (dict(since=P + 2), {"select"}), (dict(flags=P + 2), ALL)])
def test_arguments(xkv, over, who):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls that are not refused would run")
    got = calls(xkv, config(xkv, cap=100), **over)
    for name, st in got.items():
        if name in who:
            assert st == xkv.XKV_ERR_INVALID_ARG, (name, st)
        else:                                          # passes the checks, and then finds no device
            assert st in (xkv.XKV_ERR_CUDA, xkv.XKV_ERR_ARCH), (name, st)


def test_the_binding_checks_tensors(xkv):
    import torch
    cfg = config(xkv)
    t = torch.zeros(4)
    with pytest.raises(ValueError, match="K: the tensor"):
        xkv.xkv_tree_commit(cfg, 0, 2, t, t, t, t, None, 4)
    with pytest.raises(TypeError, match="weights"):
        xkv.xkv_evict_select(cfg, 0, 2, 12345, None, None, None, 4, t)
    with pytest.raises(ValueError, match="current CUDA device"):
        xkv.xkv_evict_select(cfg, 0, 2, torch.zeros((2, 1, 2, 100)), None, None, None, 4, t)


def test_workspace_bytes(xkv):
    cfg = config(xkv)
    small, large = xkv.xkv_tree_workspace_bytes(cfg, 32), xkv.xkv_tree_workspace_bytes(cfg, 33)
    assert large == 2 * small                          # 128 query rows a head, more than 128
    for n in (0, 257):
        with pytest.raises(xkv.XKVError):
            xkv.xkv_tree_workspace_bytes(cfg, n)


def test_fault_injection_masks(xkv):
    for mask in (1, 16, 128, xkv.XKV_INJECT_CACHE_NO_LOAD | 2):
        with pytest.raises(xkv.XKVError):
            xkv.xkv_debug_set_cache_fault_injection(mask)
    xkv.xkv_debug_set_cache_fault_injection(xkv.XKV_INJECT_CACHE_NO_LOAD | xkv.XKV_INJECT_CACHE_NO_HANDOVER)
    xkv.xkv_debug_set_cache_fault_injection(0)
