"""xkv_tree_attend where a row's maximum grows in the middle of a CTA's tiles, so that what it has summed up is rescaled between two
products -- at the second, a middle and the last step -- and where a CTA goes on to another problem behind a partial result."""
import math

import pytest
import torch

from tests import _cache_ref as R
from tests.test_gpu_tree_attend import call, make

pytestmark = pytest.mark.gpu

TILE = 128


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def segments(problems, tiles):
    """(problem, first tile, end) of every CTA's part of a list of `problems` x `tiles` tiles in even pieces."""
    ctas = min(torch.cuda.get_device_properties(0).multi_processor_count, 148, problems * tiles)
    out = []
    for c in range(ctas):
        u, end = problems * tiles * c // ctas, problems * tiles * (c + 1) // ctas
        while u < end:
            p, t = divmod(u, tiles)
            n = min(tiles - t, end - u)
            out.append((p, t, t + n))
            u += n
    return out


def check_head(s, out, lse, l, b, h, scale):
    c, rep = s["c"], s["c"]["H_q"] // s["c"]["H_kv"]
    dl, ln = s["drafts"][b], s["lens"][b]
    at = torch.cat([torch.ones((dl, ln), dtype=torch.bool), s["sees"][b, :dl, :dl]], 1).repeat_interleave(rep, 0).cuda()
    q = s["q"][l, b, :dl, h * rep:(h + 1) * rep].reshape(dl * rep, -1)
    want, wl, mag, top = R.head_attend(q, s["K"][l, b, h, :ln + dl], s["V"][l, b, h, :ln + dl], at, scale)
    tol, tl = R.attend_bounds(want, wl, mag, top, c["d_h"])
    got = out[l, b, :dl, h * rep:(h + 1) * rep].reshape(dl * rep, -1).double()
    gl = lse[l, b, :dl, h * rep:(h + 1) * rep].reshape(-1).double()
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol).all(), (l, b, h, ((got - want).abs() / tol).max().item())
    assert ((gl - wl).abs() <= tl).all(), (l, b, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,H_kv,rep,rows", [(8, 4, 4, 40000), (1, 8, 1, 30000), (33, 4, 4, 20000), (64, 4, 4, 20000)])
def test_a_maximum_that_jumps_inside_a_segment(xkv, n, H_kv, rep, rows, d):
    """Two thirds of the query rows meet a row 2^9 above all before, three times in a segment, and the rows behind it lie as high:
    the 64 rows of a step, 2^-9 each, are an eighth of the next such row, so that a sum that is lost or scaled wrongly shows.
    Values are one on average; noise in the logits is small against the threshold of 2^8."""
    s = make(n=n, lens=[rows], H_kv=H_kv, H_q=H_kv * rep, d=d, seed=n + d, tree="chain", spare=0)
    step = 64 if n * rep > 128 else TILE
    tiles = -(-(rows + n) // TILE)
    height = torch.zeros((H_kv, tiles * TILE))           # log2 of a row's weight, relative to its segment's first rows
    several = 0
    for p, t0, t1 in segments(H_kv, tiles):
        begin, steps = t0 * TILE, (t1 - t0) * TILE // step
        several += steps >= 6
        for i, at in enumerate(sorted({1, steps // 2, steps - 1} & set(range(1, steps)))):
            height[p, begin + at * step + 3 + 11 * i:t1 * TILE] = 9.0 * (i + 1)
    assert several >= 100
    high = torch.arange(n * H_kv * rep).reshape(n, H_kv * rep) % 3 != 0          # the others' first element is zero: no jump
    scale = 1 / math.sqrt(d)
    s["V"] = (s["V"].float() + 1).to(torch.bfloat16)
    s["q"] = (s["q"].float() * 0.1).to(torch.bfloat16)
    s["q"][0, 0, ..., 0] = torch.where(high, 4.0, 0.0).to(torch.bfloat16).cuda()
    s["K"][0, 0, ..., 0] = (height[:, :rows + n] * math.log(2) / (4 * scale)).to(torch.bfloat16).cuda()
    out, lse, flags = call(xkv, s)
    assert flags.item() == 0
    for h in range(H_kv):
        check_head(s, out, lse, 0, 0, h, scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [6, 40])
def test_a_partial_result_and_then_another_problem(xkv, n, d):
    """Problems of about as many tiles as a CTA takes: nearly every CTA ends one, leaves a partial result and begins the next."""
    lens = [900 + 37 * b for b in range(20)]
    s = make(G=2, batch=20, n=n, lens=lens, H_kv=2, H_q=8, d=d, seed=d, spare=0)
    first = call(xkv, s)
    for l in range(2):
        for b in range(20):
            for h in range(2):
                check_head(s, first[0], first[1], l, b, h, 1 / math.sqrt(d))
    for _ in range(20):
        out, lse, _ = call(xkv, s)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [7, 130])
def test_values_that_are_not_finite_over_many_problems_of_a_cta(xkv, n, d):
    """More than 32 problems a CTA; drafts whose values are not finite in some of the sequences, one of them the last before the
    ragged end: every other sequence, and every token that does not attend to them, keeps its bits."""
    batch, H = 300, 16
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 25, (batch,), generator=g).tolist()
    drafts = torch.randint(1, n + 1, (batch,), generator=g).tolist()
    for b in range(0, batch, 4):
        drafts[b] = n
    s = make(batch=batch, n=n, lens=lens, drafts=drafts, H_kv=H, H_q=H, d=d, seed=n, spare=0, tree="any")
    clean, clean_lse, _ = call(xkv, s)
    bad = torch.zeros((batch, n), dtype=torch.bool)
    for b in range(0, batch, 3):
        for j in {int(torch.randint(0, drafts[b], (1,), generator=g)), drafts[b] - 1 if b % 2 else 0}:
            bad[b, j] = True
            s["V"][0, b, :, lens[b] + j, (b + j) % 5::9] = (math.nan, math.inf, -math.inf)[(b + j) % 3]
    for _ in range(3):
        out, lse, flags = call(xkv, s)
        assert flags.item() == 0 and torch.equal(lse, clean_lse)
        hit = (s["sees"] & bad[:, None]).any(2) & (torch.arange(n) < torch.tensor(drafts)[:, None])
        assert hit.any(1).sum() > 50
        hit = hit.cuda()
        assert torch.equal(out[0][~hit], clean[0][~hit])
        assert not torch.isfinite(out[0][hit]).all(-1).any()
        assert torch.isfinite(clean[0][hit]).all()
