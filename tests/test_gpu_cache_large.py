"""The operators over an uncompressed cache where element offsets pass 32 bits, at many heads, on several streams at once, and
with tensors that are not aligned."""
import math

import pytest
import torch

from tests import _cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def test_offsets_beyond_32_bits(xkv):
    """Eight sequences of 4 M rows: 2^32 elements, 8.6 GB a tensor.  Zero rows have a logit of 0 and a value of 0, so that a row
    among n of them is known without touching them."""
    cap, d, n = xkv.XKV_CACHE_MAX_ROWS, 128, 3
    g = torch.Generator().manual_seed(1)
    K, V = (torch.zeros((1, 8, 1, cap, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ln = cap - n
    lens = [0, 5, 0, 0, 0, 0, 0, ln]
    at = list(range(ln - 40, cap))                       # the rows that are not zero, in the last sequence: its end, and its drafts
    K[0, 7, 0, at], V[0, 7, 0, at] = (torch.randn((len(at), d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((1, 8, n, 2, d), generator=g).to(torch.bfloat16).cuda()
    cfg = xkv.make_cache_config(G=1, batch=8, H_kv=1, H_q=2, d_h=d, cap=cap)
    out, lse = torch.zeros_like(q), torch.zeros((1, 8, n, 2), device="cuda")
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    flags = i32([0])
    xkv.xkv_tree_attend(cfg, 0, 1, q, n, None, i32([0] * 7 + [n]), K, V, i32(lens), ws, out, lse, flags)
    k, v = K[0, 7, 0, at].double(), V[0, 7, 0, at].double()
    zeros = ln - 40
    for i in range(n):
        for h in range(2):
            z = k[:40 + i + 1] @ q[0, 7, i, h].double() / math.sqrt(d)
            total = torch.logsumexp(torch.cat([z, torch.tensor([math.log(zeros)], dtype=torch.float64, device="cuda")]), 0)
            p = torch.exp(z - total)
            want, mag = p @ v[:40 + i + 1], p @ v[:40 + i + 1].abs()
            # sums of four million equal weights: fp32 partial sums of a CTA's tiles, off by 2^-24 of themselves an addition,
            # 64 additions a tile and thread, 222 tiles at most in a row
            slack = 2.0 ** -24 * 64 * 222
            assert ((out[0, 7, i, h].double() - want).abs() <= R.BF16 * want.abs() + (2 * R.BF16 + slack) * mag + 1e-12).all()
            assert abs(lse[0, 7, i, h].item() - total.item()) <= slack + 1e-4
    assert (out[0, :7] == 0).all()
    weights = torch.zeros((1, 8, 1, cap), device="cuda")
    vis = torch.zeros((8, n), dtype=torch.int32)
    vis[7] = torch.tensor([ln + 1, ln + 2, ln + 3])
    xkv.xkv_cache_weigh(cfg, 0, 1, q, n, lse, K, i32([0] * 7 + [cap]), vis.cuda(), i32([0] * 8), 1.0, weights, flags)
    want = torch.zeros(len(at), dtype=torch.float64, device="cuda")
    for i in range(n):
        for h in range(2):
            want[:40 + i + 1] += torch.exp(k[:40 + i + 1] @ q[0, 7, i, h].double() / math.sqrt(d) - lse[0, 7, i, h].double())
    torch.testing.assert_close(weights[0, 7, 0, at].double(), want, rtol=1e-4, atol=0)
    torch.testing.assert_close(weights[0, 7, 0, :100].double(), torch.exp(-lse[0, 7].double()).sum().expand(100), rtol=1e-4, atol=0)
    assert (weights[0, :7] == 0).all()
    # the last drafts move: the third and the first
    rows = K[0, 7, 0, ln:].clone()
    xkv.xkv_tree_commit(cfg, 0, 1, K, V, i32(lens), i32([[0, 0]] * 7 + [[2, 0]]), i32([0] * 7 + [2]), 2, None, None, flags)
    assert torch.equal(K[0, 7, 0, ln:ln + 2], rows[[2, 0]]) and torch.equal(K[0, 7, 0, ln + 2], rows[2])
    src = torch.arange(64, dtype=torch.int32, device="cuda").expand(1, 8, 1, 64).contiguous()
    src[0, 7, 0, 10] = cap - 1
    xkv.xkv_evict_compact(cfg, 0, 1, K, V, src, 64, weights, None, flags)
    assert torch.equal(K[0, 7, 0, 10], K[0, 7, 0, cap - 1]) and torch.equal(weights[0, 7, 0, 10], weights[0, 7, 0, cap - 1])
    assert not K[0, 7, 0, :10].any() and not K[0, :7].any()
    assert flags.item() == 0


@pytest.mark.parametrize("batch,H,cap", [(15, 2, 70000), (24, 2, 66000), (33, 2, 66000), (64, 2, 66000), (64, 2, 33000), (37, 4, 5000), (150, 2, 1500)])
def test_select_over_many_heads(xkv, batch, H, cap):
    """The number of CTAs per head goes by how many heads there are: clusters of every size."""
    g = torch.Generator(device="cuda").manual_seed(batch)
    w = (torch.rand((1, batch, H, cap), generator=g, device="cuda") * 1000).floor()
    lens = [max(cap - 17 * b, cap // 2) for b in range(batch)]
    keep = cap // 3
    src = torch.zeros((1, batch, H, keep), dtype=torch.int32, device="cuda")
    cfg = xkv.make_cache_config(G=1, batch=batch, H_kv=H, H_q=H, d_h=64, cap=cap)
    flags = i32([0])
    since = [x - 100 for x in lens]
    xkv.xkv_evict_select(cfg, 0, 1, w, None, i32(since), i32(lens), keep, src, flags)
    assert flags.item() == 0
    for b, h in ((0, 0), (batch // 2, 1), (batch - 1, H - 1)):
        assert src[0, b, h].tolist() == R.select_ref(w[0, b, h].cpu(), None, since[b], lens[b], keep), (b, h)
    # every head: a map's rows are all different, and its weights are the largest
    got = torch.gather(w, 3, src.long()).sort(-1, descending=True).values
    for b in range(batch):
        row = w[0, b, :, :lens[b] - 100].sort(-1, descending=True).values[:, :keep - 100]
        recent = w[0, b, :, lens[b] - 100:lens[b]]
        assert torch.equal(got[0, b], torch.cat([row, recent], 1).sort(-1, descending=True).values)
        assert all(src[0, b, h].unique().numel() == keep for h in range(H))


def test_several_streams_at_once(xkv):
    """Calls that share no output run at the same time: the same bits as one after the other."""
    g = torch.Generator().manual_seed(3)
    cap, n = 2500, 4
    cfg = xkv.make_cache_config(G=2, batch=2, H_kv=2, H_q=8, d_h=64, cap=cap)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    jobs = []
    for _ in range(4):
        K, V, q = bf(2, 2, 2, cap, 64), bf(2, 2, 2, cap, 64), bf(2, 2, n, 8, 64)
        w = torch.rand((2, 2, 2, cap), generator=g).cuda()
        jobs.append(dict(K=K, V=V, q=q, w=w, len=i32([cap - n, 1700]), out=torch.zeros_like(q), lse=torch.zeros((2, 2, n, 8), device="cuda"),
                         src=torch.zeros((2, 2, 2, 1000), dtype=torch.int32, device="cuda"),
                         ws=torch.empty(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")))

    def run(j, stream=None):
        xkv.xkv_tree_attend(cfg, 0, 2, j["q"], n, None, None, j["K"], j["V"], j["len"], j["ws"], j["out"], j["lse"], None, stream)
        xkv.xkv_cache_weigh(cfg, 0, 2, j["q"], n, j["lse"], j["K"], j["len"], None, None, 0.5, j["w"], None, stream)
        xkv.xkv_evict_select(cfg, 0, 2, j["w"], None, None, j["len"], 1000, j["src"], None, stream)
        xkv.xkv_evict_compact(cfg, 0, 2, j["K"], j["V"], j["src"], 1000, j["w"], None, None, stream)
    keys = ("K", "V", "w", "out", "lse", "src")
    start = [{k: j[k].clone() for k in keys} for j in jobs]
    for j in jobs:
        run(j)
    torch.cuda.synchronize()
    want = [{k: j[k].clone() for k in keys} for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for j, s in zip(jobs, start):
            for k in keys:
                j[k].copy_(s[k])
        torch.cuda.synchronize()
        for j, st in zip(jobs, streams):
            run(j, st)                                   # the stream is an argument, not torch's current one
        torch.cuda.synchronize()
        for j, s in zip(jobs, want):
            assert all(torch.equal(j[k], s[k]) for k in keys)


def test_unaligned_tensors_are_refused(xkv):
    cfg = xkv.make_cache_config(G=1, batch=1, H_kv=1, H_q=1, d_h=64, cap=20)
    K = torch.zeros(20 * 64 + 1, dtype=torch.bfloat16, device="cuda")
    good, odd = K[:-1].reshape(1, 1, 1, 20, 64), K[1:].reshape(1, 1, 1, 20, 64)
    src = torch.zeros((1, 1, 1, 4), dtype=torch.int32, device="cuda")
    xkv.xkv_evict_compact(cfg, 0, 1, good, good.clone(), src - 1, 4)
    with pytest.raises(xkv.XKVError) as e:
        xkv.xkv_evict_compact(cfg, 0, 1, odd, good, src, 4)
    assert e.value.status == xkv.XKV_ERR_INVALID_ARG


def test_a_batch_of_many_sequences(xkv):
    """More sequences than a warp has lanes, most of them short, through every operator."""
    g = torch.Generator().manual_seed(5)
    batch, cap, n = 300, 40, 2
    lens = [(7 * b) % (cap - n + 1) for b in range(batch)]
    cfg = xkv.make_cache_config(G=1, batch=batch, H_kv=1, H_q=2, d_h=64, cap=cap)
    K, V = (torch.randn((1, batch, 1, cap, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((1, batch, n, 2, 64), generator=g).to(torch.bfloat16).cuda()
    out, lse = torch.zeros_like(q), torch.zeros((1, batch, n, 2), device="cuda")
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    flags = i32([0])
    xkv.xkv_tree_attend(cfg, 0, 1, q, n, None, None, K, V, i32(lens), ws, out, lse, flags)
    for b in range(batch):
        at = torch.cat([torch.ones((n, lens[b]), dtype=torch.bool), torch.ones((n, n), dtype=torch.bool).tril()], 1).repeat_interleave(2, 0).cuda()
        want, wl, mag, top = R.head_attend(q[0, b].reshape(4, 64), K[0, b, 0, :lens[b] + n], V[0, b, 0, :lens[b] + n], at, 0.125)
        tol, tl = R.attend_bounds(want, wl, mag, top, 64)
        assert ((out[0, b].reshape(4, 64).double() - want).abs() <= tol).all() and ((lse[0, b].reshape(4).double() - wl).abs() <= tl).all()
    w = torch.rand((1, batch, 1, cap), generator=g).cuda()
    old = w.clone()
    vis = torch.tensor([[x + 1, x + 2] for x in lens])
    xkv.xkv_cache_weigh(cfg, 0, 1, q, n, lse, K, i32([x + n for x in lens]), vis.to(torch.int32).cuda(), i32(lens), 1.0, w, flags)
    want, err = R.weigh_ref(q, lse.cpu(), K, [x + n for x in lens], vis, lens, 1.0, old, 0.125)
    assert ((w.double() - want).abs() <= err + 1e-30).all()
    src = torch.zeros((1, batch, 1, 20), dtype=torch.int32, device="cuda")
    xkv.xkv_evict_select(cfg, 0, 1, w, None, None, i32(lens), 20, src, flags)
    for b in range(batch):
        assert src[0, b, 0].tolist() == R.select_ref(w[0, b, 0].cpu(), None, None, lens[b], 20)
    assert flags.item() == 0
