"""Waits of the attention over codes that run out: the call ends with a flag and NaN, and the next one is right again."""
import time

import pytest
import torch

from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu


@pytest.fixture()
def xkv():
    from paper_2503_18893_b200 import xkv as m
    yield m
    m.xkv_debug_set_cache_fault_injection(0)


@pytest.mark.parametrize("inject", ["XKV_INJECT_CACHE_NO_LOAD", "XKV_INJECT_CACHE_NO_HANDOVER"])
@pytest.mark.parametrize("lens,news,kw", [([9000], [1], dict(H_kv=2)), ([700, 40, 300], [4, 3, 1], dict(H_kv=2, d=64)), ([3000], [8], dict(H_kv=2)),
                                          ([2000], [30], dict(H_kv=2)), ([1500, 600], [100, 70], dict(H_kv=2)), ([400] * 30, [1] * 30, dict(H_kv=8))])
def test_attend_gives_up(xkv, inject, lens, news, kw):
    c = A.Case(xkv, lens, news, page=16, seed=5, **kw)
    out, lse = c.run()
    c.check(out, lse) if sum(lens) < 1000 else A.check_large(c, out, lse)
    for _ in range(2):
        xkv.xkv_debug_set_cache_fault_injection(getattr(xkv, inject))
        began = time.perf_counter()
        bad, bad_lse = c.run()
        torch.cuda.synchronize()
        flags = int(c.flags)
        assert time.perf_counter() - began < 2.0
        if inject == "XKV_INJECT_CACHE_NO_LOAD":
            assert flags == xkv.XKV_FLAG_TIMEOUT and bool(bad.isnan().all()) and bool(bad_lse.isnan().all())
        else:                                   # a CTA whose tiles all have room ahead of the hand-over gives up as well: nobody multiplies
            assert flags == xkv.XKV_FLAG_TIMEOUT and bool(bad.isnan().any())
        xkv.xkv_debug_set_cache_fault_injection(0)
        again, lse2 = c.run()
        assert int(c.flags) == 0 and torch.equal(again, out) and torch.equal(lse2, lse)


def test_without_a_flag_word_nan_tells(xkv):
    c = A.Case(xkv, [900], [1], H_kv=1, page=32, seed=6)
    out, _ = c.run()
    ws = torch.empty(xkv.xkv_cache8_workspace_bytes(c.cfg, 1), dtype=torch.uint8, device="cuda")
    xkv.xkv_debug_set_cache_fault_injection(xkv.XKV_INJECT_CACHE_NO_LOAD)
    e, bad = torch.float8_e4m3fn, torch.zeros_like(c.q)
    xkv.xkv_cache8_attend(c.cfg, 0, 1, c.q, None, 1, A.dev(c.table), A.dev(c.lens), c.K.view(e), c.V.view(e), c.ks, c.vs, ws, bad)
    torch.cuda.synchronize()
    assert bool(bad.isnan().all())
    xkv.xkv_debug_set_cache_fault_injection(0)
    again, _ = c.run()
    assert torch.equal(again, out)
