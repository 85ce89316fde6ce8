"""xkv_cache_weigh where it can go wrong beside its definition's cases: tokens without a log-sum-exp over keys that are not finite,
and the number of queries at which another pass over the keys begins."""
import math

import pytest
import torch

from tests.test_gpu_cache_weigh import call, check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("n,rep,d", [(3, 4, 128), (3, 4, 64), (20, 2, 128), (40, 4, 128), (40, 4, 64)])
@pytest.mark.parametrize("rows", [90, 700])
def test_a_token_that_attended_to_nothing_adds_nothing(xkv, n, rep, d, rows):
    """Its log-sum-exp is minus infinity, and rows whose keys are not finite are among those that it is said to have seen."""
    s = make(n=n, lens=[rows], H_kv=2, H_q=2 * rep, d=d, seed=n + rows, visible=[[rows] * n])
    s["lse"][0, 0, 1] = -math.inf
    s["lse"][0, 0, 2, rep:] = -math.inf          # only the heads of the second KV head
    clean, _ = call(xkv, s)
    check(s, clean)
    # every query but those is turned down: the rows below are seen by nobody else
    s["visible"] = torch.tensor([[rows if i in (1, 2) else rows // 3 for i in range(n)]])
    s["lse"][0, 0, 2] = -math.inf
    s["K"][0, 0, 0, rows // 2, 5] = math.nan
    s["K"][0, 0, 1, rows // 2 + 1] = math.inf
    s["K"][0, 0, 1, rows - 1, 3] = -math.inf
    w, flags = call(xkv, s)
    assert flags.item() == 0
    check(s, w)
    assert torch.equal(w[..., rows // 3:rows], s["w"][..., rows // 3:rows])


# a pass holds 128 queries of a KV head
@pytest.mark.parametrize("n,rep", [(128, 1), (129, 1), (64, 2), (32, 4), (33, 4), (255, 1), (256, 1), (16, 8), (17, 8), (8, 16), (9, 16)])
def test_queries_around_a_pass(xkv, n, rep):
    s = make(n=n, lens=[300], H_kv=1, H_q=rep, d=64 if n % 2 else 128, seed=n)
    w, flags = call(xkv, s)
    assert flags.item() == 0
    check(s, w)
