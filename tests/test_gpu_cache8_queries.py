"""Attention over codes: a query's small elements beside its largest one, seen in the logarithm of the sum of a single row."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens,n_rep", [(1, 4), (3, 4), (5, 4)])         # blocks of 8, 16 and 128 query rows
def test_every_element_counts(xkv, tokens, n_rep, d):
    """One row a sequence, which only the last of its tokens sees: its logit is the log-sum-exp.  An element of 2^-e (1 + i/128) beside a
    largest one of 1 (a power of two, the worst for a split) meets the row's only key element, 256."""
    cases = [(e, i) for e in range(0, 26) for i in (0, 1, 3, 5, 37, 64, 85, 127)]
    batch = len(cases)
    f8 = torch.float8_e4m3fn
    K, V = (torch.zeros((1, 1, 1, 16, d), device="cuda").to(f8) for _ in range(2))
    K[0, 0, 0, 0, 1] = 256.0
    ones = torch.ones((1, 1, 1), device="cuda")
    cfg = xkv.make_cache8_config(G=1, batch=batch, H_kv=1, H_q=n_rep, d_h=d, page=16, n_pages=1, max_pages=1, softmax_scale=1.0)
    q = torch.zeros((1, batch * tokens, n_rep, d), dtype=torch.bfloat16, device="cuda")
    small = torch.tensor([2.0 ** -e * (1 + i / 128) for e, i in cases], device="cuda", dtype=torch.float64)
    sign = torch.tensor([(-1.0) ** i for i in range(batch)], device="cuda", dtype=torch.float64)
    q[0, :, :, 0] = 1.0
    q[0, :, :, 1] = (small * sign).to(torch.bfloat16).repeat_interleave(tokens)[:, None]
    table, length = torch.zeros((batch, 1), dtype=torch.int32, device="cuda"), torch.ones(batch, dtype=torch.int32, device="cuda")
    first = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * tokens
    ws = torch.empty(xkv.xkv_cache8_workspace_bytes(cfg, tokens), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    xkv.xkv_cache8_attend(cfg, 0, 1, q, first, tokens, table, length, K, V, ones, ones, ws, out, lse)
    got = lse[0].view(batch, tokens, n_rep).double()
    assert bool((got[:, :tokens - 1] == -math.inf).all())
    # 2^-21 of the largest element, times the key's 256; the logit, its maximum and their logarithm in fp32
    z = 256.0 * small * sign
    bound = 256.0 * 2.0 ** -21 * small.clamp_min(1.0) + 2.0 ** -21 * (z.abs() + 16.0)
    off = (got[:, tokens - 1] - z[:, None]).abs()
    assert bool((off <= bound[:, None]).all()), [(cases[i], float(off[i].max())) for i in (off > bound[:, None]).any(1).nonzero().flatten().tolist()]
