"""xkv_cache_weigh against its definition in 64 bits."""
import math

import pytest
import torch

from tests import _cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def make(*, G=1, batch=1, H_kv=2, H_q=8, d=128, n=3, lens=(200,), visible=None, seen=None, decay=1.0, spare=2, seed=0):
    g = torch.Generator().manual_seed(seed)
    cap = max(lens) + spare
    K = torch.randn((G, batch, H_kv, cap, d), generator=g)
    w = torch.rand((G, batch, H_kv, cap), generator=g)
    seen = list(seen) if seen is not None else list(lens)
    for b in range(batch):
        K[:, b, :, lens[b]:] = math.nan
        w[:, b, :, seen[b]:lens[b]] = math.nan       # a row that is new holds anything
        w[:, b, :, lens[b]:] = 7.0
    if decay == 0.0:
        w[:] = torch.where(w == 7.0, w, torch.full_like(w, math.nan))
    q = torch.randn((G, batch, n, H_q, d), generator=g)
    if visible is None:
        visible = torch.tensor([[max(0, ln - n + 1 + i) for i in range(n)] for ln in lens])
    else:
        visible = torch.tensor(visible)
    lse = torch.randn((G, batch, n, H_q), generator=g) + 5
    return dict(c=dict(G=G, batch=batch, H_kv=H_kv, H_q=H_q, d_h=d, cap=cap), n=n, K=K.to(torch.bfloat16).cuda(), q=q.to(torch.bfloat16).cuda(),
                lse=lse.cuda(), w=w.cuda(), lens=list(lens), visible=visible, seen=seen, decay=decay)


def call(xkv, s, layers=None, scale=0.0, w=None):
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    w = s["w"].clone() if w is None else w
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    l0, l1 = layers or (0, s["c"]["G"])
    xkv.xkv_cache_weigh(xkv.make_cache_config(**s["c"], softmax_scale=scale), l0, l1, s["q"], s["n"], s["lse"], s["K"], i32(s["lens"]),
                        i32(s["visible"]), i32(s["seen"]), s["decay"], w, flags)
    return w, flags


def check(s, w, scale=0.0, layers=None):
    want, err = R.weigh_ref(s["q"], s["lse"].cpu(), s["K"], s["lens"], s["visible"], s["seen"], s["decay"], s["w"],
                            scale or 1 / math.sqrt(s["c"]["d_h"]))
    l0, l1 = layers or (0, s["c"]["G"])
    assert torch.equal(w[:l0].nan_to_num(9), s["w"][:l0].nan_to_num(9)) and torch.equal(w[l1:].nan_to_num(9), s["w"][l1:].nan_to_num(9))
    for b, ln in enumerate(s["lens"]):
        assert torch.equal(w[:, b, :, ln:], s["w"][:, b, :, ln:])
        d = (w[l0:l1, b, :, :ln].double() - want[l0:l1, b, :, :ln]).abs()
        assert torch.isfinite(d).all()
        assert (d <= err[l0:l1, b, :, :ln]).all(), (b, (d / err[l0:l1, b, :, :ln]).max().item())


CASES = [
    dict(n=1, lens=[1]), dict(n=1, lens=[127]), dict(n=1, lens=[128], spare=0), dict(n=1, lens=[129]), dict(n=1, lens=[1000], H_kv=1, H_q=1),
    dict(n=1, lens=[500], H_kv=1, H_q=16, d=64), dict(n=5, lens=[300]), dict(n=33, lens=[290], H_kv=1, H_q=7), dict(n=64, lens=[260], d=64),
    # more than 256 queries a head: another pass over the keys; an odd and an even number of tiles
    dict(n=65, lens=[130], H_kv=1, H_q=4), dict(n=100, lens=[300], H_kv=1, H_q=7), dict(n=256, lens=[400], H_kv=1, H_q=3, d=64),
    # tokens that were turned down, that saw next to nothing; none at all
    dict(n=6, lens=[200], visible=[[195, 0, 196, 0, 0, 197]]), dict(n=40, lens=[333], visible=[[1 + 8 * i if i % 3 else 0 for i in range(40)]]),
    dict(n=4, lens=[200], visible=[[0, 0, 0, 0]], decay=0.5), dict(n=3, lens=[150], visible=[[150, 1, 128]]),
    # new rows, decay, no earlier weights
    dict(n=2, lens=[200], seen=[150], decay=0.9), dict(n=2, lens=[200], seen=[0]), dict(n=2, lens=[200], decay=0.0),
    dict(n=130, lens=[260], seen=[130], decay=0.25, H_kv=1, H_q=2),
    # batches
    dict(batch=3, n=4, lens=[5, 0, 300], seen=[1, 0, 300]), dict(G=2, batch=2, n=3, lens=[129, 700], d=64), dict(batch=40, n=1, lens=[7 * i for i in range(40)], H_kv=1, H_q=2),
    dict(batch=2, n=1, lens=[0, 0]),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_cache_weigh(xkv, i):
    s = make(**CASES[i], seed=i)
    w, flags = call(xkv, s)
    assert flags.item() == 0
    check(s, w)


def test_long_cache_and_scale_and_layers(xkv):
    s = make(G=3, n=2, lens=[128 * 400 + 5], H_kv=1, H_q=4, seed=50)
    w, _ = call(xkv, s, layers=(1, 2), scale=0.05)
    check(s, w, scale=0.05, layers=(1, 2))


def test_a_token_that_attended_to_nothing(xkv):
    s = make(n=3, lens=[90], seed=51)
    s["lse"][0, 0, 1] = -math.inf
    w, _ = call(xkv, s)
    check(s, w)


def test_defaults(xkv):
    s = make(n=2, lens=[140], spare=0, seed=52)
    s["visible"] = torch.tensor([[140, 140]])
    w = s["w"].clone()
    xkv.xkv_cache_weigh(xkv.make_cache_config(**s["c"]), 0, 1, s["q"], 2, s["lse"], s["K"], None, None, None, 1.0, w)
    check(s, w)


def test_out_of_range_is_clamped_and_reported(xkv):
    s = make(batch=2, n=2, lens=[90, 60], seed=53)
    s["K"] = s["K"].nan_to_num(0.5)
    s["w"] = s["w"].nan_to_num(0.5)
    cap = s["c"]["cap"]
    for k, v, to in (("lens", [cap + 5, 60], [cap, 60]), ("lens", [90, -3], [90, 0]), ("seen", [95, 60], [90, 60]), ("seen", [90, -1], [90, 0]),
                     ("visible", [[91, 50], [1, 1]], [[90, 50], [1, 1]]), ("visible", [[9, -50], [1, 1]], [[9, 0], [1, 1]])):
        t = dict(s, visible=torch.tensor([[20, 30], [0, 0]]), seen=[0, 0])
        t[k] = torch.tensor(v) if k == "visible" else v
        w, flags = call(xkv, t)
        assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE, k
        t[k] = torch.tensor(to) if k == "visible" else to
        check(t, w)


def test_the_same_call_twice_and_in_a_graph(xkv):
    s = make(batch=2, n=20, lens=[3000, 411], H_kv=2, H_q=14, seed=54)
    a, b = call(xkv, s)[0], call(xkv, s)[0]
    assert torch.equal(a, b)
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    args = (s["q"], 20, s["lse"], s["K"], i32(s["lens"]), i32(s["visible"]), i32(s["seen"]), 1.0)
    w = s["w"].clone()
    cfg = xkv.make_cache_config(**s["c"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        xkv.xkv_cache_weigh(cfg, 0, 1, *args, w)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, a)


def test_weights_of_its_own_attention_add_up(xkv):
    """A row's weights are a softmax: with the log-sum-exp of xkv_tree_attend they add up to the number of queries."""
    s = make(n=1, lens=[3001], H_kv=2, H_q=8, spare=0, seed=55)
    c = s["c"]
    cfg = xkv.make_cache_config(**c)
    out, lse = torch.empty_like(s["q"]), torch.empty((1, 1, 1, 8), device="cuda")
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, 1), dtype=torch.uint8, device="cuda")
    xkv.xkv_tree_attend(cfg, 0, 1, s["q"], 1, None, None, s["K"], s["K"], None, ws, out, lse)
    w = torch.full((1, 1, 2, 3001), math.nan, device="cuda")
    xkv.xkv_cache_weigh(cfg, 0, 1, s["q"], 1, lse, s["K"], None, None, None, 0.0, w)
    # both err in their logits by less than 128 * 2^-23 of 12 (|q| |k| scale), and round a few times
    torch.testing.assert_close(w.double().sum(-1), torch.full((1, 1, 2), 4.0, dtype=torch.float64, device="cuda"), rtol=5e-4, atol=0)
