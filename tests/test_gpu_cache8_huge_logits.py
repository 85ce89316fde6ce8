"""Attention over codes where logits are far beyond what fp32 tells apart from their neighbours: the rows of the largest share the weight."""
import math

import pytest
import torch

from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("new,n_rep", [(1, 4), (4, 4), (20, 4), (60, 7)])
def test_logits_of_every_size(xkv, new, n_rep, order):
    rows, d, page = 1000, 64, 16
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    codes = codes[codes.float().isfinite() & (codes.float() != 0)]
    codes = codes[codes.float().argsort()]                       # every value, up
    c = A.Case(xkv, [rows], [new], H_kv=1, n_rep=n_rep, d=d, page=page, seed=1)
    c.ks[:], c.vs[:] = 1.0, 2.0 ** -8
    at = torch.arange(rows) * len(codes) // rows
    at = at.flip(0) if order == "down" else at[torch.randperm(rows, generator=torch.Generator().manual_seed(2))] if order == "mixed" else at
    key = codes.view(torch.uint8)[at].view(torch.float8_e4m3fn)
    pages = torch.tensor(c.table[0], device="cuda")[torch.arange(rows, device="cuda") // page]
    off = torch.arange(rows, device="cuda") % page
    c.K[:] = 0
    c.K[0, pages, 0, off, 0] = key.view(torch.uint8).cuda()
    V = (c.V[0, pages, 0, off].view(torch.float8_e4m3fn).double() * 2.0 ** -8)
    for e in range(0, 110, 3):                   # logits up to 448 * 2^e / 8: in units of two, from 80 to 2^114
        c.q[:] = 0
        sign = torch.where(torch.arange(new * n_rep).view(new, n_rep) % 2 == 0, 1.0, -1.0).cuda()
        c.q[0, :, :, 0] = sign * 2.0 ** e
        out, lse = c.run()
        for s in (1.0, -1.0):
            z = s * 2.0 ** e * c.scale * key.double().cuda()
            seen = torch.arange(rows, device="cuda") <= torch.arange(rows - new, rows, device="cuda")[:, None]
            p = torch.softmax(z.expand(new, -1).masked_fill(~seen, -math.inf), -1)
            total = torch.logsumexp(z.expand(new, -1).masked_fill(~seen, -math.inf), -1)
            want, mag = p @ V, p @ V.abs()
            hit = sign == s
            got = out[0].double()
            # a logit is rounded to 24 bits, where its neighbours are 1 / 28 of it away at the least: what matters is below 2^12 of them
            off_by = 2.0 ** -23 * min(448.0 * 2.0 ** e, 4096.0)
            bound = (2.0 ** -8 + 2.0 ** -10 + 2 * off_by) * mag + 2.0 ** -33
            assert bool(((got - want[:, None]).abs() <= bound[:, None])[hit].all()), (e, s, float(((got - want[:, None]).abs() / bound[:, None])[hit].max()))
            assert bool(((lse[0].double() - total[:, None]).abs() <= 2.0 ** -20 * (1 + total.abs()[:, None]))[hit].all())
