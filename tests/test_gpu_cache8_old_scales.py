"""Rows appended to a page that holds some already, whatever power of two its scale is; and to one whose scale is 0 or not finite."""
import math

import pytest
import torch

from tests import test_gpu_cache8_codes as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("old", [-126, -100, -70, -65, -61, -60, -59, 0, 119, 120, 121, 125, 126, 127])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_every_power_of_two(xkv, old, d, page):
    for size in (0.0, 2.0 ** -80, 2.0 ** -58, 1.0, 2.0 ** 100):
        p = C.Pool(xkv, 1, 2, d, page, 3, seed=old + 200)
        p.ks[0, 1], p.vs[0, 1] = 2.0 ** old, 2.0 ** old
        p.append(C.rows(p, 3, size), C.rows(p, 3, size), [page + 5, page + 6, page + 7])
        assert int(p.flags) == 0


@pytest.mark.parametrize("old", [0.0, 2.0 ** -130, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_scales_that_are_no_power_of_two(xkv, old, d, page):
    """0: the page held nothing, its rows become 0.  Not finite: NaN.  The scale is that of the new rows alone."""
    p, fresh = C.Pool(xkv, 1, 2, d, page, 3, seed=3), C.Pool(xkv, 1, 2, d, page, 3, seed=3)
    k, v, slot = C.rows(p, 3), C.rows(p, 3, 100.0), C.dev([page + 5, page + 6, page + 7])
    p.ks[0, 1], p.vs[0, 1] = old, old
    fresh.ks[0, 1], fresh.vs[0, 1] = 2.0 ** -60, 2.0 ** -60
    before = [t.clone().view(torch.uint8) for t in (p.K, p.V)]
    for q in (p, fresh):
        xkv.xkv_cache8_append(q.cfg, 0, 1, k, v, slot, q.K, q.V, q.ks, q.vs, q.flags)
    for codes, scale, codes_f, scale_f, was in ((p.K, p.ks, fresh.K, fresh.ks, before[0]), (p.V, p.vs, fresh.V, fresh.vs, before[1])):
        assert torch.equal(scale[0, 1], scale_f[0, 1])
        raw = codes.view(torch.uint8)
        assert torch.equal(raw[0, 1, :, 5:8], codes_f.view(torch.uint8)[0, 1, :, 5:8])
        held = raw[0, 1, :, :5]
        assert bool((held == 0).all()) if abs(old) < 1 else bool(codes.float()[0, 1, :, :5].isnan().all())
        assert torch.equal(raw[0, 1, :, 8:], was[0, 1, :, 8:]) and torch.equal(raw[0, [0, 2]], was[0, [0, 2]])
