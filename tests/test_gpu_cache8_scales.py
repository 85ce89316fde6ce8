"""Attention over codes: pages' scales as memory may hold them.  What the calls say has no influence has none, in blocks of few query rows
and of many."""
import math

import pytest
import torch

from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu
NEWS = [1, 4, 20]                                # with four query heads: blocks of 8, 16 and 128 query rows


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("other", [math.nan, math.inf, -math.inf, 2.0 ** 127, 2.0 ** 100])
@pytest.mark.parametrize("new", NEWS)
@pytest.mark.parametrize("page", [16, 64])
def test_a_page_that_holds_nothing_whatever_its_other_scale(xkv, new, page, other):
    c = A.Case(xkv, [200, 90], [new, 1], H_kv=1, page=page, seed=7)
    at = c.table[0][1]
    for zero, rest in ((c.ks, c.vs), (c.vs, c.ks)):
        keep = zero[0, at, 0].item(), rest[0, at, 0].item()
        zero[0, at, 0], rest[0, at, 0] = 0.0, 1.0
        want, want_lse = c.run()
        c.check(want, want_lse)
        rest[0, at, 0] = other
        out, lse = c.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        zero[0, at, 0], rest[0, at, 0] = keep


@pytest.mark.parametrize("bad", [math.nan, math.inf, 2.0 ** 127])
@pytest.mark.parametrize("which", ["ks", "vs"])
@pytest.mark.parametrize("new", [20, 100])
def test_scales_of_a_page_that_a_token_does_not_see(xkv, new, which, bad):
    """Tokens before the page's rows are as without; those that see it get NaN where its scale is not finite."""
    c = A.Case(xkv, [150], [new], H_kv=1, page=16, seed=new)
    clean, clean_lse = c.run()
    j = (150 - new + 1 + 15) // 16               # the first page that begins with a row behind the first token's
    sees = max(0, 16 * j - (150 - new))          # the first token that sees it
    getattr(c, which)[0, c.table[0][j], 0] = bad
    out, lse = c.run()
    assert 0 < sees < new and torch.equal(out[0, :sees], clean[0, :sees]) and torch.equal(lse[0, :sees], clean_lse[0, :sees])
    if bad != 2.0 ** 127:
        assert bool(out[0, sees:].isnan().all()) and bool(lse[0, sees:].isnan().all())


@pytest.mark.parametrize("new", NEWS)
@pytest.mark.parametrize("v_scale", [2.0 ** -90, 2.0 ** -60, 2.0 ** 118])
def test_values_scales_at_the_ends_of_their_range(xkv, new, v_scale):
    c = A.Case(xkv, [300, 30], [new, 1], H_kv=1, page=16, seed=9, spread=0.5)
    c.vs[:] = v_scale
    far, far_lse = c.run()
    c.vs[:] = 1.0
    out, lse = c.run()
    c.check(out, lse)
    # weights, sums and results differ by a power of two; the exponent of a weight is rounded with v_scale's in it, 2^-17 at most
    assert bool(((far.double() / v_scale - out.double()).abs() <= 2.0 ** -7 * out.double().abs() + 2.0 ** -16 * 448).all())
    assert bool(((far_lse - lse).abs() <= 2.0 ** -16).all())


@pytest.mark.parametrize("new", NEWS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_query_of_zeros_over_faint_keys(xkv, new, d):
    """Its logits are all 0, however small the keys' scales; a row behind a token's own stays out."""
    for k_scale in (2.0 ** -60, 2.0 ** -90, 2.0 ** -100, 2.0 ** -126):
        c = A.Case(xkv, [200, 30], [new, 1], H_kv=1, d=d, page=16, seed=5)
        c.ks[:] = k_scale
        c.q[0, 0] = 0.0
        c.q[0, new - 1, 1] = 0.0
        out, lse = c.run()
        c.check(out, lse)
        assert not bool(out.isnan().any())


@pytest.mark.parametrize("new", NEWS)
@pytest.mark.parametrize("scale", [1e-12, 1e-30, 1e-37, 1e-44])
def test_a_tiny_softmax_scale(xkv, new, scale):
    for k_scale in (2.0 ** -7, 2.0 ** -60):
        c = A.Case(xkv, [200, 30], [new, 1], H_kv=1, page=16, seed=6, scale=scale)
        c.ks[:] = k_scale
        c.q[0, new - 1] = 0.0
        out, lse = c.run()
        c.check(out, lse)
        assert not bool(out.isnan().any())


@pytest.mark.parametrize("new", NEWS)
def test_a_factor_beyond_fp32(xkv, new):
    """Keys that are exactly 0 have logit 0 whatever scale and query say."""
    c = A.Case(xkv, [120], [new], H_kv=1, page=16, seed=8)
    c.ks[:] = 2.0 ** 100
    c.q[:] = 2.0 ** 100
    c.K[:] = 0
    out, lse = c.run()
    rows = torch.arange(120 - new + 1, 121, dtype=torch.float64, device="cuda")
    assert bool(((lse[0].double() - rows.log()[:, None]).abs() <= 2.0 ** -18).all()) and not bool(out.isnan().any())
