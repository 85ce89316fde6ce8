"""Waits of the kernels over an uncompressed cache that run out: the call ends with a flag, and the next one is right again."""
import time

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
@pytest.mark.parametrize("shape", [dict(n=5, lens=[3000]), dict(n=64, lens=[40000], H_kv=2, H_q=8), dict(n=70, lens=[900], d=64)])
def test_tree_attend_gives_up(xkv, inject, shape):
    s = T.make(**shape, seed=1)
    good = T.call(xkv, s)
    T.check(s, good[0], good[1])
    for _ in range(2):
        xkv.xkv_debug_set_cache_fault_injection(getattr(xkv, inject))
        began = time.perf_counter()
        flags = T.call(xkv, s)[2]
        torch.cuda.synchronize()
        assert flags.item() == xkv.XKV_FLAG_TIMEOUT
        assert time.perf_counter() - began < 2.0
        xkv.xkv_debug_set_cache_fault_injection(0)
        again = T.call(xkv, s)
        assert again[2].item() == 0 and torch.equal(again[0], good[0]) and torch.equal(again[1], good[1])


@pytest.mark.parametrize("inject", ["XKV_INJECT_CACHE_NO_LOAD", "XKV_INJECT_CACHE_NO_HANDOVER"])
def test_cache_weigh_gives_up(xkv, inject):
    # (the accumulators are four: a hand-over is missed by a CTA's fifth tile)
    s = W.make(n=3, lens=[128 * 148 * 6], H_kv=1, H_q=4, seed=2)
    good = W.call(xkv, s)[0]
    for _ in range(2):
        xkv.xkv_debug_set_cache_fault_injection(getattr(xkv, inject))
        began = time.perf_counter()
        flags = W.call(xkv, s)[1]
        torch.cuda.synchronize()
        assert flags.item() == xkv.XKV_FLAG_TIMEOUT
        assert time.perf_counter() - began < 2.0
        xkv.xkv_debug_set_cache_fault_injection(0)
        w, flags = W.call(xkv, s)
        assert flags.item() == 0 and torch.equal(w, good)


def test_other_masks_are_refused(xkv):
    with pytest.raises(xkv.XKVError):
        xkv.xkv_debug_set_cache_fault_injection(1)
