"""A wait that runs out in a call without a flag word shows in what the call returns."""
import pytest
import torch

from tests import test_gpu_cache_weigh as W
from tests import test_gpu_tree_attend as T

pytestmark = pytest.mark.gpu


@pytest.fixture()
def xkv():
    from paper_2503_18893_b200 import xkv as m
    yield m
    m.xkv_debug_set_cache_fault_injection(0)


@pytest.mark.parametrize("inject", ["XKV_INJECT_CACHE_NO_LOAD", "XKV_INJECT_CACHE_NO_HANDOVER"])
# problems of one CTA and of several, both numbers of query rows, sequences without drafts
@pytest.mark.parametrize("shape", [dict(n=5, lens=[3000]), dict(n=64, lens=[40000], H_kv=2, H_q=8), dict(n=70, lens=[900], d=64),
                                   dict(batch=40, n=3, lens=[5 * b for b in range(40)], drafts=[b % 4 for b in range(40)], H_kv=8, H_q=16),
                                   dict(batch=3, n=150, lens=[0, 300, 30], drafts=[150, 0, 33], H_kv=2, H_q=4, d=64, G=2)])
def test_tree_attend(xkv, inject, shape):
    s = T.make(**shape, seed=1)
    c, n = s["c"], s["n"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cfg, ln, dl = xkv.make_cache_config(**c), i32(s["lens"]), i32(s["drafts"])
    ws = torch.zeros(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")

    def call(lse):
        out = torch.full((c["G"], c["batch"], n, c["H_q"], c["d_h"]), 7.0, dtype=torch.bfloat16, device="cuda")
        xkv.xkv_tree_attend(cfg, 0, c["G"], s["q"], n, s["mask"], dl, s["K"], s["V"], ln, ws, out, lse)
        torch.cuda.synchronize()
        return out
    lse = torch.full((c["G"], c["batch"], n, c["H_q"]), 7.0, device="cuda")
    there = (torch.arange(n)[None] < torch.tensor(s["drafts"])[:, None]).cuda()
    xkv.xkv_debug_set_cache_fault_injection(getattr(xkv, inject))
    for with_lse in (True, False):
        out = call(lse if with_lse else None)
        for l in range(c["G"]):
            assert torch.isnan(out[l][there]).all() and torch.isnan(lse[l][there]).all()
            assert (out[l][~there] == 7).all() and (lse[l][~there] == 7).all()
    xkv.xkv_debug_set_cache_fault_injection(0)
    out = call(lse)
    T.check(s, out, lse)


@pytest.mark.parametrize("inject", ["XKV_INJECT_CACHE_NO_LOAD", "XKV_INJECT_CACHE_NO_HANDOVER"])
@pytest.mark.parametrize("d", [64, 128])
def test_cache_weigh(xkv, inject, d):
    # (a hand-over is missed by a CTA's fifth tile)
    s = W.make(n=3, lens=[128 * 148 * 6 - 5, 0, 700], batch=3, H_kv=1, H_q=4, seed=2, d=d)
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    cfg, ln, vis, seen = xkv.make_cache_config(**s["c"]), i32(s["lens"]), i32(s["visible"]), i32(s["seen"])

    def call():
        w = s["w"].clone()
        xkv.xkv_cache_weigh(cfg, 0, 1, s["q"], 3, s["lse"], s["K"], ln, vis, seen, 0.5, w)
        torch.cuda.synchronize()
        return w
    s["decay"] = 0.5
    xkv.xkv_debug_set_cache_fault_injection(getattr(xkv, inject))
    w = call()
    for b, n in enumerate(s["lens"]):
        assert torch.isnan(w[0, b, :, :n]).all() and torch.equal(w[0, b, :, n:], s["w"][0, b, :, n:])
    xkv.xkv_debug_set_cache_fault_injection(0)
    W.check(s, call())
