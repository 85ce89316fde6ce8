"""xkv_tree_attend against its definition in 64 bits: head layouts, lengths, masks, ragged batches, rows that hold anything."""
import math

import pytest
import torch

from tests import _cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def make(*, G=1, batch=1, H_kv=2, H_q=8, d=128, n=5, lens=(100,), drafts=None, spare=3, seed=0, tree="tree", fill=math.nan):
    g = torch.Generator().manual_seed(seed)
    cap = max(lens) + n + spare
    c = dict(G=G, batch=batch, H_kv=H_kv, H_q=H_q, d_h=d, cap=cap)
    K = torch.randn((G, batch, H_kv, cap, d), generator=g)
    V = torch.randn((G, batch, H_kv, cap, d), generator=g)
    drafts = list(drafts or [n] * batch)
    for b in range(batch):                       # what is behind the last draft is anything
        K[:, b, :, lens[b] + drafts[b]:] = fill
        V[:, b, :, lens[b] + drafts[b]:] = fill
    q = torch.randn((G, batch, n, H_q, d), generator=g)
    if tree == "tree":
        sees = torch.stack([R.random_tree(n, g) for _ in range(batch)])
    elif tree == "chain":
        sees = torch.ones((batch, n, n), dtype=torch.bool).tril()
    elif tree == "none":
        sees = torch.zeros((batch, n, n), dtype=torch.bool)
    else:                                        # no order at all: also later drafts, also not itself
        sees = torch.rand((batch, n, n), generator=g) < 0.4
    to = lambda t: t.to(torch.bfloat16).cuda()
    return dict(c=c, q=to(q), K=to(K), V=to(V), sees=sees, n=n, lens=list(lens), drafts=drafts,
                mask=None if tree == "chain" else R.words(sees).cuda())


def call(xkv, s, layers=None, scale=0.0, out=None, lse=None, stream=None, ws=None, flags=None):
    c, n = s["c"], s["n"]
    cfg = xkv.make_cache_config(**c, softmax_scale=scale)
    out = torch.full((c["G"], c["batch"], n, c["H_q"], c["d_h"]), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    lse = torch.full((c["G"], c["batch"], n, c["H_q"]), 7.0, device="cuda") if lse is None else lse
    if ws is None:
        ws = torch.full((xkv.xkv_tree_workspace_bytes(cfg, n),), 255, dtype=torch.uint8, device="cuda")       # NaNs
    ln = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
    dl = torch.tensor(s["drafts"], dtype=torch.int32, device="cuda")
    l0, l1 = layers or (0, c["G"])
    flags = torch.zeros(1, dtype=torch.int32, device="cuda") if flags is None else flags
    xkv.xkv_tree_attend(cfg, l0, l1, s["q"], n, s["mask"], dl, s["K"], s["V"], ln, ws, out, lse, flags, stream)
    return out, lse, flags


def check(s, out, lse, layers=None, scale=0.0, heads=None):
    c, n = s["c"], s["n"]
    rep = c["H_q"] // c["H_kv"]
    scale = scale or 1 / math.sqrt(c["d_h"])
    l0, l1 = layers or (0, c["G"])
    for l in range(c["G"]):
        for b in range(c["batch"]):
            dl, ln = s["drafts"][b], s["lens"][b]
            if not l0 <= l < l1:
                assert (out[l, b] == 7).all() and (lse[l, b] == 7).all()
                continue
            assert (out[l, b, dl:] == 7).all() and (lse[l, b, dl:] == 7).all()
            if not dl:
                continue
            at = torch.cat([torch.ones((dl, ln), dtype=torch.bool), s["sees"][b, :dl, :dl]], 1).repeat_interleave(rep, 0).cuda()
            for h in heads or range(c["H_kv"]):
                q = s["q"][l, b, :dl, h * rep:(h + 1) * rep].reshape(dl * rep, -1)
                want, wl, mag, top = R.head_attend(q, s["K"][l, b, h, :ln + dl], s["V"][l, b, h, :ln + dl], at, scale)
                tol, tl = R.attend_bounds(want, wl, mag, top, c["d_h"])
                got = out[l, b, :dl, h * rep:(h + 1) * rep].reshape(dl * rep, -1).double()
                gl = lse[l, b, :dl, h * rep:(h + 1) * rep].reshape(-1).double()
                empty = ~at.any(1)
                assert (got[empty] == 0).all() and (gl[empty] == -math.inf).all()
                assert torch.isfinite(got).all()
                worst = ((got - want).abs() / tol).max().item()
                assert worst <= 1, (l, b, h, worst)
                assert ((gl - wl).abs()[~empty] <= tl[~empty]).all(), (l, b, h)


CASES = [
    # one token: a decode step, at every kind of length
    dict(n=1, lens=[0], tree="chain"), dict(n=1, lens=[1], tree="chain"), dict(n=1, lens=[126], tree="chain"), dict(n=1, lens=[127], tree="chain"),
    dict(n=1, lens=[128], tree="chain"), dict(n=1, lens=[129], tree="chain", spare=0), dict(n=1, lens=[1000], tree="chain", H_kv=1, H_q=1),
    dict(n=1, lens=[777], tree="tree", H_kv=2, H_q=32),
    # trees, on and across the borders of tiles and mask words
    dict(n=5, lens=[300], d=64), dict(n=31, lens=[97]), dict(n=32, lens=[96], d=64), dict(n=33, lens=[95]), dict(n=64, lens=[1]),
    dict(n=33, lens=[250], H_kv=1, H_q=7, G=2), dict(n=37, lens=[515], H_kv=4, H_q=28, d=64),
    # no rows but the drafts, an order that is none, tokens that attend to nothing
    dict(n=40, lens=[0], tree="any"), dict(n=40, lens=[130], tree="any"), dict(n=9, lens=[0], tree="none"), dict(n=9, lens=[3], tree="none"),
    # more than 128 and more than 256 query rows a head
    dict(n=64, lens=[700], H_kv=2, H_q=8), dict(n=130, lens=[64], H_kv=1, H_q=2), dict(n=256, lens=[200], H_kv=1, H_q=1, tree="any"),
    dict(n=100, lens=[333], H_kv=1, H_q=16, d=64), dict(n=256, lens=[40], H_kv=1, H_q=3), dict(n=256, lens=[3000], H_kv=1, H_q=2, d=64),
    # batches of different lengths, sequences without drafts, without rows, more sequences than lanes
    dict(batch=3, n=8, lens=[5, 700, 0], drafts=[8, 3, 1]), dict(batch=4, n=70, lens=[129, 1, 300, 64], drafts=[70, 0, 33, 64], G=2, tree="any"),
    dict(batch=5, n=6, lens=[10, 20, 30, 40, 50], drafts=[0, 0, 6, 0, 0], d=64), dict(batch=67, n=2, lens=[3 * i for i in range(67)], H_kv=1, H_q=2),
    dict(batch=2, n=4, lens=[5, 6], drafts=[0, 0]),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_tree_attend(xkv, i):
    s = make(**CASES[i], seed=i)
    out, lse, flags = call(xkv, s)
    torch.cuda.synchronize()
    assert flags.item() == 0
    check(s, out, lse)


def test_many_tiles_per_cta_and_a_growing_maximum(xkv):
    """A sequence longer than the tiles of all CTAs together; later rows draw far larger logits, so that O is rescaled."""
    s = make(n=3, lens=[128 * 148 * 2 + 50], H_kv=1, H_q=4, seed=77)
    ramp = torch.linspace(0.1, 6.0, s["c"]["cap"], device="cuda")[:, None]
    s["K"] = (s["K"].float() * ramp).to(torch.bfloat16)
    out, lse, _ = call(xkv, s)
    check(s, out, lse)


def test_rows_with_one_huge_logit(xkv):
    s = make(n=8, lens=[1500], H_kv=1, H_q=8, seed=5)
    s["K"][0, 0, 0, 1200] = (8 * s["q"][0, 0, 3, 2].float()).to(torch.bfloat16)
    s["K"][0, 0, 0, 10] = (-8 * s["q"][0, 0, 3, 2].float()).to(torch.bfloat16)
    out, lse, _ = call(xkv, s)
    check(s, out, lse)


def test_softmax_scale(xkv):
    s = make(n=6, lens=[400], seed=6)
    out, lse, _ = call(xkv, s, scale=0.3)
    check(s, out, lse, scale=0.3)


def test_a_range_of_layers(xkv):
    s = make(G=4, n=6, lens=[400], seed=7)
    out, lse, _ = call(xkv, s, layers=(1, 3))
    check(s, out, lse, layers=(1, 3))


def test_no_lse_and_default_lengths(xkv):
    s = make(n=4, lens=[197], spare=0, seed=8, tree="chain")
    cfg = xkv.make_cache_config(**s["c"])
    out = torch.zeros_like(s["q"])
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, 4), dtype=torch.uint8, device="cuda")
    xkv.xkv_tree_attend(cfg, 0, 1, s["q"], 4, None, None, s["K"], s["V"], None, ws, out)
    full, _, _ = call(xkv, s)
    assert torch.equal(out, full)


@pytest.mark.parametrize("n,rep", [(20, 2), (150, 2)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_token_does_not_see_does_not_reach_it(xkv, n, rep, value):
    """A draft whose keys and values are not finite reaches the tokens that attend to it, and no others."""
    s = make(n=n, lens=[240], H_kv=2, H_q=2 * rep, seed=9, tree="tree")
    bad = [3, n - 1]
    clean, clean_lse, _ = call(xkv, s)
    for j in bad:
        s["V"][0, 0, 1, 240 + j, 5::7] = value
    s["K"][0, 0, 0, 240 + 3] = value
    out, lse, _ = call(xkv, s)
    hit = s["sees"][0][:, bad].any(1).cuda()
    rest = ~hit
    assert torch.equal(out[0, 0, rest], clean[0, 0, rest]) and torch.equal(lse[0, 0, rest], clean_lse[0, 0, rest])
    v = out[0, 0, hit, rep:]
    assert not torch.isfinite(v[..., 5::7]).any()
    if math.isinf(value):
        assert (v[..., 5::7] == value).all()
    keep = torch.ones(128, dtype=torch.bool)
    keep[5::7] = False
    assert torch.equal(v[..., keep], clean[0, 0, hit, rep:][..., keep])


def test_lengths_out_of_range_are_clamped_and_reported(xkv):
    s = make(batch=3, n=4, lens=[50, 60, 70], seed=10, fill=0.5)
    good = call(xkv, s)
    assert good[2].item() == 0
    for lens, drafts in (([10 ** 6, 60, 70], [4, 4, 4]), ([50, -5, 70], [4, 4, 4]), ([50, 60, 70], [4, 9, 4]), ([50, 60, 70], [4, -1, 4])):
        t = dict(s, lens=lens, drafts=drafts)
        out, lse, flags = call(xkv, t)
        assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE
        cap = s["c"]["cap"]
        t["drafts"] = [min(max(d, 0), 4) for d in drafts]
        t["lens"] = [min(max(x, 0), cap - d) for x, d in zip(lens, t["drafts"])]
        check(t, out, lse)


def test_the_same_call_twice_gives_the_same_bits(xkv):
    s = make(batch=2, n=48, lens=[5000, 3111], H_kv=2, H_q=14, seed=11)
    a, b = call(xkv, s), call(xkv, s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_on_another_stream_and_in_a_graph_as_lengths_grow(xkv):
    s = make(batch=2, n=5, lens=[200, 90], spare=300, seed=12, fill=0.25)
    c = s["c"]
    cfg = xkv.make_cache_config(**c)
    ln = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
    dl = torch.tensor(s["drafts"], dtype=torch.int32, device="cuda")
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, 5), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(s["q"], 7.0), torch.full((1, 2, 5, c["H_q"]), 7.0, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    run = lambda: xkv.xkv_tree_attend(cfg, 0, 1, s["q"], 5, s["mask"], dl, s["K"], s["V"], ln, ws, out, lse)
    with torch.cuda.stream(st):
        run()
    st.synchronize()
    check(s, out, lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for lens in ([0, 1], [417, 300], [128, 500]):
        ln.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        check(dict(s, lens=lens), out, lse)


def test_beside_dense_attention(xkv):
    """One token without a mask is the decode step that xkv_dense_attend does, to both kernels' rounding."""
    from paper_2503_18893_b200 import synth
    from tests import _cases as C
    sh = synth.config(1, T=256, k=64, d_h=128, r_k=64, r_v=64)
    g = C.GpuCase(sh, C.case_from_factors(sh))
    s = make(G=sh.G, batch=1, H_kv=sh.H_kv, H_q=sh.H_q, n=1, lens=[1234], spare=0, tree="chain", seed=13)
    out, lse, _ = call(xkv, s)
    cap = 1235
    ws = torch.empty(xkv.xkv_dense_workspace_bytes(g.grp, cap), dtype=torch.uint8, device="cuda")
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    xkv.xkv_dense_attend(g.grp, 0, sh.G, s["q"], s["K"], s["V"], None, cap, ws, o2, l2)
    # the dense kernel sums the rounded weights: its denominator and so its lse are off by up to half a bf16 step
    torch.testing.assert_close(lse, l2, rtol=0, atol=2 * R.BF16)
    torch.testing.assert_close(out.float(), o2.float(), rtol=4 * R.BF16, atol=4 * R.BF16)
    g.close()
