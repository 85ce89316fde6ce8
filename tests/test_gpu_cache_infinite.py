"""Logits that are minus infinity, infinite and NaN keys, values and queries in what is attended to, over an uncompressed cache."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def attend(xkv, q, K, V, rows, n):
    G, batch, H_kv, cap, d = K.shape
    cfg = xkv.make_cache_config(G=G, batch=batch, H_kv=H_kv, H_q=q.shape[3], d_h=d, cap=cap)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    xkv.xkv_tree_attend(cfg, 0, G, q, n, None, None, K, V, torch.tensor([rows], dtype=torch.int32, device="cuda"), ws, out, lse)
    return cfg, out, lse


def inputs(rows, n, H_q, d=128, seed=0):
    g = torch.Generator().manual_seed(seed)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    return bf(1, 1, n, H_q, d), bf(1, 1, 1, rows + n, d), bf(1, 1, 1, rows + n, d)


@pytest.mark.parametrize("n,H_q", [(1, 4), (40, 4)])
@pytest.mark.parametrize("rows", [5, 700, 40000])
def test_logits_of_minus_infinity(xkv, rows, n, H_q):
    """One dimension of the keys is -inf: a query that is positive there has no finite logit."""
    q, K, V = inputs(rows, n, H_q)
    q[..., 0] = 1.0
    K[..., 0] = -math.inf
    _, out, lse = attend(xkv, q, K, V, rows, n)
    assert (out == 0).all() and (lse == -math.inf).all()
    # half of the rows finite again: the others weigh nothing
    K[0, 0, 0, ::2, 0] = 0.5
    cfg, out, lse = attend(xkv, q, K, V, rows, n)
    for i in ([0, n - 1] if rows < 1000 else [0]):
        at = list(range(0, rows + i + 1, 2))
        k, v = K[0, 0, 0, at].double(), V[0, 0, 0, at].double()
        for h in range(H_q):
            z = k @ q[0, 0, i, h].double() / math.sqrt(128)
            p = torch.softmax(z, 0)
            # weights and the output are rounded to bf16, logits err by less than 128 * 2^-23 of 16 (sum of |q_i k_i| / sqrt(d))
            assert ((out[0, 0, i, h].double() - p @ v).abs() <= 2.0 ** -8 * (p @ v).abs() + (2.0 ** -8 + 1e-3) * (p @ v.abs())).all()
            assert abs(lse[0, 0, i, h].item() - torch.logsumexp(z, 0).item()) < 1e-3
    # such rows have drawn no weight
    w = torch.full((1, 1, 1, rows + n), math.nan, device="cuda")
    xkv.xkv_cache_weigh(cfg, 0, 1, q, n, lse, K, None, torch.tensor([[rows + i + 1 for i in range(n)]], dtype=torch.int32, device="cuda"),
                        torch.zeros(1, dtype=torch.int32, device="cuda"), 1.0, w)
    assert (w[0, 0, 0, 1::2] == 0).all() and torch.isfinite(w).all() and (w[0, 0, 0, :rows:2] > 0).all()


def test_a_query_that_is_nan_stays_alone(xkv):
    q, K, V = inputs(500, 40, 4, seed=1)
    _, clean, clean_lse = attend(xkv, q, K, V, 500, 40)
    q[0, 0, 17, 2, 5] = math.nan
    _, out, lse = attend(xkv, q, K, V, 500, 40)
    assert torch.isnan(out[0, 0, 17, 2]).all() and torch.isnan(lse[0, 0, 17, 2])
    out[0, 0, 17, 2], lse[0, 0, 17, 2] = clean[0, 0, 17, 2], clean_lse[0, 0, 17, 2]
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("rows", [100, 30000])
def test_a_committed_row_that_is_not_finite_reaches_everyone(xkv, rows):
    q, K, V = inputs(rows, 3, 4, seed=2)
    V[0, 0, 0, 50, 7] = math.inf
    _, out, lse = attend(xkv, q, K, V, rows, 3)
    assert not torch.isfinite(out[..., 7]).any() and torch.isfinite(out[..., 8:]).all() and torch.isfinite(lse).all()
    V[0, 0, 0, 50, 7] = 0
    K[0, 0, 0, 60] = math.nan
    _, out, lse = attend(xkv, q, K, V, rows, 3)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
