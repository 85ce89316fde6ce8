"""Attention over codes: what can go wrong, in blocks of 8, 16 and 128 query rows alike."""
import math

import pytest
import torch

from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu
WIDTHS = [(1, 4), (2, 4), (4, 4), (3, 5), (5, 4), (20, 4), (40, 1), (9, 16)]      # tokens of the first sequence, query heads of a KV head


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,n_rep", [w for w in WIDTHS if w[0] > 1])
def test_nan_in_a_new_row(xkv, new, n_rep, d):
    """Tokens before the row are as without; those that see it get NaN in those elements, or everywhere where it is the key's."""
    c = A.Case(xkv, [150, 300], [new, 1], H_kv=2, n_rep=n_rep, d=d, page=16, seed=d + new)
    clean, clean_lse = c.run()
    for tok in {0, new // 2, new - 1}:
        row = 150 - new + tok
        p, off = c.table[0][row // 16], row % 16
        keep = c.V[0, p, 1, off].clone(), c.K[0, p, 1, off].clone()
        c.V[0, p, 1, off, 3], c.V[0, p, 1, off, d - 1] = A.NAN_CODE, 0xFF
        out, lse = c.run()
        c.check(out, lse)
        assert torch.equal(out[0, :tok], clean[0, :tok]) and torch.equal(out[0, new:], clean[0, new:])
        assert torch.equal(out[0, :, :n_rep], clean[0, :, :n_rep])          # the other KV head's
        hit = out[0, tok:new, n_rep:].isnan()
        assert bool(hit[..., [3, d - 1]].all()) and int(hit.sum()) == 2 * (new - tok) * n_rep
        c.V[0, p, 1, off] = keep[0]
        c.K[0, p, 1, off, 5] = A.NAN_CODE
        out, lse = c.run()
        assert torch.equal(out[0, :tok], clean[0, :tok]) and torch.equal(lse[0, :tok], clean_lse[0, :tok])
        assert bool(out[0, tok:new, n_rep:].isnan().all()) and bool(lse[0, tok:new, n_rep:].isnan().all())
        assert torch.equal(out[0, new:], clean[0, new:]) and torch.equal(out[0, :, :n_rep], clean[0, :, :n_rep])
        c.K[0, p, 1, off] = keep[1]


@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_queries_that_are_not_finite(xkv, new, n_rep):
    c = A.Case(xkv, [200, 201], [new, 1], H_kv=1, n_rep=n_rep, seed=3)
    clean, clean_lse = c.run()
    hit = torch.zeros((new + 1, n_rep), dtype=torch.bool, device="cuda")
    for t, h, e, what in ((new - 1, 0, 9, math.nan), (new, n_rep - 1, 100, math.inf), (0, n_rep // 2, 127, -math.inf)):
        c.q[0, t, h, e] = what
        hit[t, h] = True
    out, lse = c.run()
    assert bool(out[0][hit].isnan().all()) and torch.equal(out[0][~hit], clean[0][~hit]) and torch.equal(lse[0][~hit], clean_lse[0][~hit])


@pytest.mark.parametrize("bad", [-1, 10 ** 6, -(1 << 31)])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_pages_out_of_range(xkv, new, n_rep, page, bad):
    c = A.Case(xkv, [500, 300], [new, 1], H_kv=1, n_rep=n_rep, page=page, seed=6)
    c.table[0][1] = bad                          # one that every token would see
    c.table[0][(500 - new) // page] = bad        # and the one with the first new rows
    c.table[1][-(-300 // page) - 1] = bad
    out, lse = c.run()
    c.check(out, lse)
    assert int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE
    c.table[0] = [bad] * len(c.table[0])         # nothing is left
    out, lse = c.run()
    c.check(out, lse)
    assert bool((out[0, :new] == 0).all()) and bool((lse[0, :new] == -math.inf).all())


@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_scales_of_zero(xkv, new, n_rep):
    c = A.Case(xkv, [300], [new], H_kv=1, n_rep=n_rep, page=32, seed=7)
    c.ks[0, c.table[0][1], 0] = 0.0
    c.vs[0, c.table[0][2], 0] = 0.0
    c.vs[0, c.table[0][(300 - new) // 32], 0] = 0.0
    out, lse = c.run()
    c.check(out, lse)


@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_scales_far_apart(xkv, new, n_rep):
    for k_loud in (-6, -8, -30):
        c = A.Case(xkv, [300], [new], H_kv=1, n_rep=n_rep, page=64, seed=11)
        c.vs[0, c.table[0][0], 0], c.vs[0, c.table[0][3], 0] = 2.0 ** 20, 2.0 ** -20
        c.ks[0, c.table[0][0], 0] = 2.0 ** k_loud
        out, lse = c.run()
        c.check(out, lse)


@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_logits_that_climb_from_tile_to_tile(xkv, new, n_rep):
    c = A.Case(xkv, [2000], [new], H_kv=1, n_rep=n_rep, page=64, seed=14)
    for i, p in enumerate(c.table[0]):
        c.ks[0, p] = 2.0 ** (i // 4 - 11)
    out, lse = c.run()
    A.check_large(c, out, lse)


@pytest.mark.parametrize("new,n_rep", WIDTHS)
def test_a_result_on_another_stream(xkv, new, n_rep):
    c = A.Case(xkv, [700, 90], [new, 1], H_kv=2, n_rep=n_rep, page=16, seed=22)
    want, want_lse = c.run()
    e = torch.float8_e4m3fn
    ws = torch.empty(xkv.xkv_cache8_workspace_bytes(c.cfg, c.max_new), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(c.q), torch.zeros(c.q.shape[:3], device="cuda")
    first, table, lens = A.dev(c.first), A.dev(c.table), A.dev(c.lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())   # all that the call reads or writes is ready
    xkv.xkv_cache8_attend(c.cfg, 0, 1, c.q, first, c.max_new, table, lens, c.K.view(e), c.V.view(e), c.ks, c.vs, ws, out, lse, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
