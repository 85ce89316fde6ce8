"""Attention over a paged cache of 8-bit codes against its definition in 64 bits."""
import math

import pytest
import torch

from tests import _cache8_ref as R

pytestmark = pytest.mark.gpu
NAN_CODE = 0x7F


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Sequences of `lens` rows, the last `news` of them new, in pages in no order; what no sequence holds are NaN codes."""

    def __init__(self, xkv, lens, news, H_kv=2, n_rep=4, d=128, page=16, G=1, seed=0, gap=0, scale=0.0, extra=0, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.x, self.lens, self.news, self.page, self.n_rep, self.d, self.G = xkv, lens, news, page, n_rep, d, G
        counts = [-(-n // page) for n in lens]
        self.n_pages = sum(counts) + 2
        ids = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        most = max(counts + [1]) + extra
        self.table = [[ids.pop() for _ in range(n)] + [-1] * (most - n) for n in counts]
        self.cfg = xkv.make_cache8_config(G=G, batch=len(lens), H_kv=H_kv, H_q=H_kv * n_rep, d_h=d, page=page, n_pages=self.n_pages,
                                          max_pages=most, softmax_scale=scale)
        self.scale = scale or 1 / math.sqrt(d)
        shape = (G, self.n_pages, H_kv, page, d)
        self.K, self.V = (torch.full(shape, NAN_CODE, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.ks, self.vs = (2.0 ** torch.randint(-9, -6, shape[:3], generator=g, device="cuda").float() for _ in range(2))
        for b, n in enumerate(lens):
            for j in range(counts[b]):
                m = min(page, n - j * page)
                for t in (self.K, self.V):
                    x = (spread * 100 * torch.randn((G, H_kv, m, d), generator=g, device="cuda")).clamp(-448, 448)
                    t[:, self.table[b][j], :, :m] = x.to(torch.float8_e4m3fn).view(torch.uint8)
        self.n_tok = sum(news) + 2 * gap
        self.first = [gap]
        for n in news:
            self.first.append(self.first[-1] + n)
        self.q = torch.randn((G, self.n_tok, H_kv * n_rep, d), generator=g, device="cuda").to(torch.bfloat16)
        self.max_new = max(news + [1])
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, layers=None, lse=True, decode=False, **kw):
        ws = torch.empty(self.x.xkv_cache8_workspace_bytes(self.cfg, self.max_new), dtype=torch.uint8, device="cuda")
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        l = torch.full(self.q.shape[:3], 7.0, device="cuda")
        self.flags.zero_()
        e = torch.float8_e4m3fn
        self.x.xkv_cache8_attend(self.cfg, *(layers or (0, self.G)), self.q, None if decode else dev(self.first), self.max_new, dev(self.table),
                                 dev(self.lens), self.K.view(e), self.V.view(e), self.ks, self.vs, ws, out, l if lse else None, self.flags, **kw)
        return out, l

    def check(self, out, lse, layer=0):
        want, wl, bo, bl = R.attend_ref(self.q[layer].cpu(), self.first, self.max_new, self.table, self.lens,
                                        self.K[layer].view(torch.float8_e4m3fn).cpu().double(), self.V[layer].view(torch.float8_e4m3fn).cpu().double(),
                                        self.ks[layer].cpu().double(), self.vs[layer].cpu().double(), self.page, self.n_rep, self.scale, self.n_tok)
        got, gl = out[layer].cpu().double(), lse[layer].cpu().double()
        seen = {t for b in range(len(self.lens)) for t in range(max(self.first[b], 0), min(self.first[b + 1], self.n_tok))[:self.max_new]}
        for t in range(self.n_tok):
            if t not in seen:
                assert bool((got[t] == 7.0).all()) and bool((gl[t] == 7.0).all()), t
                continue
            assert torch.equal(got[t].isnan(), want[t].isnan()), t
            ok = want[t].isnan() | ((got[t] - want[t]).abs() <= bo[t])
            assert bool(ok.all()), (t, float((got[t] - want[t]).abs().nan_to_num().max()), float(bo[t].nan_to_num().max()))
            inf = wl[t] == -math.inf
            assert torch.equal(gl[t] == -math.inf, inf), t
            assert bool((inf | wl[t].isnan() | ((gl[t] - wl[t]).abs() <= bl[t])).all()), t


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_rep", [1, 4, 7, 16])
def test_one_token_each(xkv, page, d, n_rep):
    c = Case(xkv, [1, 2, 127, 128, 129, 255, 257, 0, 390], [1] * 9, n_rep=n_rep, d=d, page=page, seed=n_rep)
    out, lse = c.run()
    c.check(out, lse)
    assert int(c.flags) == 0
    same, _ = c.run(decode=True)
    assert torch.equal(same, out)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_rep,news", [(1, [5, 70, 1]), (4, [33, 2, 16]), (7, [9, 10, 40]), (16, [3, 5, 17])])
def test_several_tokens(xkv, d, n_rep, news):
    c = Case(xkv, [140, 200, 300], news, H_kv=1, n_rep=n_rep, d=d, page=32, seed=n_rep + d)
    out, lse = c.run()
    c.check(out, lse)


@pytest.mark.parametrize("lens,news", [([5, 130, 64], [5, 130, 64]), ([128, 256, 127], [1, 128, 127]), ([3, 0, 90], [7, 4, 0]), ([40, 41, 42], [0, 0, 3])])
def test_prompts_from_their_start_and_tokens_that_see_nothing(xkv, lens, news):
    """A whole prompt at once; more new tokens than rows (the first see nothing); sequences without tokens; tokens of nobody."""
    c = Case(xkv, lens, news, H_kv=1, n_rep=2, d=64, page=16, seed=sum(news), gap=3)
    out, lse = c.run()
    c.check(out, lse)


def test_no_tokens_at_all(xkv):
    c = Case(xkv, [100, 40], [0, 0], H_kv=1, n_rep=4, seed=1, gap=2)
    for c.max_new in (1, 4):
        out, lse = c.run()
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()) and int(c.flags) == 0


def test_many_sequences(xkv):
    lens = [(37 * b) % 150 for b in range(150)]
    c = Case(xkv, lens, [1 + (b % 5 == 0) for b in range(150)], H_kv=1, n_rep=2, d=64, page=16, seed=5)
    out, lse = c.run()
    c.check(out, lse)


def test_layers_and_no_lse(xkv):
    c = Case(xkv, [200, 77], [2, 1], G=3, seed=9)
    out, lse = c.run(layers=(1, 3))
    assert bool((out[0] == 7.0).all()) and bool((lse[0] == 7.0).all())
    for l in (1, 2):
        c.check(out, lse, l)
    out2, lse2 = c.run(layers=(1, 3), lse=False)
    assert torch.equal(out2, out) and bool((lse2 == 7.0).all())


def test_rows_that_a_token_does_not_see_do_not_touch_it(xkv):
    """NaN codes in new rows: the tokens before them are as without, the tokens that see them get NaN in those elements."""
    for d in (64, 128):
        c = Case(xkv, [150, 300], [20, 6], H_kv=1, n_rep=4, d=d, page=16, seed=d)
        clean, clean_lse = c.run()
        row, p = 140 % 16, c.table[0][140 // 16]
        c.V[0, p, 0, row, 3] = NAN_CODE          # row 140 is new token 10's
        c.V[0, p, 0, row, 17] = 0xFF
        out, lse = c.run()
        c.check(out, lse)
        assert torch.equal(out[0, :10], clean[0, :10]) and torch.equal(out[0, 20:], clean[0, 20:])
        assert bool(out[0, 10:20, :, [3, 17]].isnan().all()) and not bool(out[0, 10:20, :, 4].isnan().any())
        c.V[0, p, 0, row, 3] = c.V[0, p, 0, row, 17] = 0
        c.K[0, p, 0, row, 5] = NAN_CODE
        out, lse = c.run()
        assert torch.equal(out[0, :10], clean[0, :10]) and torch.equal(lse[0, :10], clean_lse[0, :10])
        assert bool(out[0, 10:20].isnan().all())
        assert torch.equal(out[0, 20:], clean[0, 20:])


def test_a_value_that_is_nan_in_a_row_all_see(xkv):
    c = Case(xkv, [400], [3], H_kv=1, n_rep=2, page=32, seed=2)
    c.V[0, c.table[0][3], 0, 7, 90] = NAN_CODE
    out, lse = c.run()
    assert bool(out[0, :, :, 90].isnan().all()) and not bool(out[0, :, :, 89].isnan().any())


def test_queries_that_are_not_finite(xkv):
    c = Case(xkv, [200, 201], [2, 2], H_kv=1, n_rep=4, seed=3)
    clean, _ = c.run()
    c.q[0, 1, 2, 9] = math.nan
    c.q[0, 2, 0, 100] = math.inf
    out, _ = c.run()
    hit = torch.zeros((4, 4), dtype=torch.bool)
    hit[1, 2] = hit[2, 0] = True
    assert bool(out[0][hit.cuda()].isnan().all()) and torch.equal(out[0][~hit.cuda()], clean[0][~hit.cuda()])


def test_queries_of_zero_large_and_small(xkv):
    c = Case(xkv, [300], [6], H_kv=1, n_rep=4, seed=4)
    for i, f in enumerate((0.0, 1e-20, 1e-3, 30.0, 1.0, 1.0)):
        c.q[0, i] *= f
    c.q[0, 4, :, 0] = 1000.0                    # one element far above the others
    c.q[0, 5, :, 5:] *= 1e-4
    out, lse = c.run()
    c.check(out, lse)


def test_pages_out_of_range_are_left_out(xkv):
    for bad in (-1, 10 ** 6, -(1 << 31), None):
        c = Case(xkv, [200, 100], [2, 1], H_kv=1, page=16, seed=6)
        c.table[0][4] = c.n_pages if bad is None else bad
        c.table[1][6] = c.n_pages if bad is None else bad          # the last page, with the token's own row
        out, lse = c.run()
        c.check(out, lse)
        assert int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE
    c = Case(xkv, [50, 100], [1, 1], H_kv=1, page=16, seed=6)
    c.table[0] = [-1] * len(c.table[0])          # nothing is left
    out, lse = c.run()
    c.check(out, lse)
    assert bool((out[0, 0] == 0).all())


def test_a_scale_of_zero_marks_a_page_that_holds_nothing(xkv):
    c = Case(xkv, [200], [2], H_kv=1, page=32, seed=7)
    c.ks[0, c.table[0][1], 0] = 0.0
    c.vs[0, c.table[0][2], 0] = 0.0
    out, lse = c.run()
    c.check(out, lse)


def test_lengths_and_places_out_of_range(xkv):
    c = Case(xkv, [64, 64, 64], [2, 2, 2], H_kv=1, page=16, seed=8)
    good, _ = c.run()
    c.lens = [64, 4000, 64]                      # cut to the table's room
    out, lse = c.run()
    assert torch.equal(out, good) and int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE
    c.lens = [64, 64, -3]
    out, lse = c.run()
    c.check(out, lse)
    assert bool((out[0, 4:] == 0).all()) and int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE
    c.lens, c.first = [64, 64, 64], [0, 2, 4, 100]
    out, lse = c.run()
    assert torch.equal(out, good) and int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE
    c.first, c.max_new = [0, 2, 4, 6], 1         # more tokens than were announced: those behind are left out
    out, lse = c.run()
    c.check(out, lse)
    assert int(c.flags) == xkv.XKV_FLAG_INDEX_RANGE


def test_scales_far_apart(xkv):
    """Pages whose values differ by 2^40, keys' scales at the ends of their range; the loud page draws no weight, little, or all of it."""
    for k_loud in (-6, -8, -30):
        c = Case(xkv, [300], [1], H_kv=1, n_rep=4, page=64, seed=11)
        c.vs[0, c.table[0][0], 0], c.vs[0, c.table[0][3], 0] = 2.0 ** 20, 2.0 ** -20
        c.ks[0, c.table[0][0], 0] = 2.0 ** k_loud
        out, lse = c.run()
        c.check(out, lse)
    c = Case(xkv, [100], [1], H_kv=1, n_rep=1, page=16, seed=12)
    c.vs[:] = 2.0 ** -60
    c.ks[:] = 2.0 ** -60
    out, lse = c.run()
    c.check(out, lse)


def test_a_sink_and_a_long_even_rest(xkv):
    """One row draws most of the weight, thousands share the rest: weights of 2^-13 of the largest each, all of one sign."""
    c = Case(xkv, [6000], [1], H_kv=1, n_rep=2, page=128, seed=13, spread=0.01)
    first, one = c.table[0][0], torch.tensor([300.0]).to(torch.float8_e4m3fn).view(torch.uint8).item()
    c.q[0, 0, :] = 1.0
    c.ks[:], c.vs[:] = 2.0 ** -8, 2.0 ** -8
    for p in c.table[0]:
        c.K[0, p] = 0
        c.V[0, p] = one
    c.K[0, first, 0, 0] = torch.tensor([200.0]).to(torch.float8_e4m3fn).view(torch.uint8).item()     # logit 8.8
    c.V[0, first, 0, 0] = 0
    out, lse = c.run()
    c.check(out, lse)


def test_logits_that_climb_from_tile_to_tile(xkv):
    c = Case(xkv, [3000], [2], H_kv=2, n_rep=4, page=64, seed=14)
    for i, p in enumerate(c.table[0]):
        c.ks[0, p] = 2.0 ** (i // 6 - 11)
    out, lse = c.run()
    c.check(out, lse)


def reference(c, layer=0):
    """All tokens of a large case at once, on the device in 64 bits; bounds as in the small ones."""
    K, V = (t[layer].view(torch.float8_e4m3fn).double() for t in (c.K, c.V))
    at = c.first[0]
    for b, (rows, n) in enumerate(zip(c.lens, c.news)):
        pages = torch.tensor(c.table[b][:-(-rows // c.page)], device="cuda")
        for g in range(K.shape[1]):
            k = (K[pages, g] * c.ks[layer][pages, g].double()[:, None, None]).reshape(-1, c.d)[:rows]
            vsc = c.vs[layer][pages, g].double().repeat_interleave(c.page)[:rows]
            code = V[pages, g].reshape(-1, c.d)[:rows]
            for i0 in range(0, n, 64):
                m = min(64, n - i0)
                q = c.q[layer, at + i0:at + i0 + m, g * c.n_rep:(g + 1) * c.n_rep].double()
                z = torch.einsum("ihd,jd->ihj", q, k) * c.scale
                hidden = torch.arange(rows, device="cuda") > torch.arange(rows - n + i0, rows - n + i0 + m, device="cuda")[:, None]
                z.masked_fill_(hidden[:, None], -math.inf)
                total = torch.logsumexp(z, -1)
                p = torch.exp(z - total[..., None])
                ze = c.scale * (c.d * 2.0 ** -23 * (q.abs() @ k.abs().T).amax(-1) + 2.0 ** -18 * q.abs().amax(-1) * k.abs().sum(1).amax()) + 2.0 ** -20 * (1 + total.abs())
                o, mag = p @ (code * vsc[:, None]), p @ (code.abs() * vsc[:, None])
                bound = R.BF16 * o.abs() * (1 + R.BF16) + (2.0 ** -11 + 2 * ze[..., None] + 2.0 ** -16) * mag + 2.0 ** -21 * (p * vsc).amax(-1)[..., None] * code.abs().sum(0) + 1e-30
                yield slice(at + i0, at + i0 + m), slice(g * c.n_rep, (g + 1) * c.n_rep), o, total, bound, ze
        at += n


def check_large(c, out, lse, layer=0):
    for t, h, o, total, bound, ze in reference(c, layer):
        assert bool(((out[layer, t, h].double() - o).abs() <= bound).all())
        assert bool(((lse[layer, t, h].double() - total).abs() <= ze).all())


@pytest.mark.parametrize("lens,news,kw", [
    ([40000], [1], dict(H_kv=2, n_rep=4, page=64)), ([9000, 4100, 1], [1, 1, 1], dict(H_kv=4, n_rep=7, page=16)),
    ([7000, 50], [16, 3], dict(H_kv=2, n_rep=4, page=32)), ([5000, 3001], [600, 77], dict(H_kv=1, n_rep=7, page=128)),
    ([2500], [2500], dict(H_kv=1, n_rep=2, page=64, d=64)), ([20000, 10], [2, 1], dict(H_kv=2, n_rep=16, page=16, d=64)),
    ([1000] * 40, [1] * 40, dict(H_kv=8, n_rep=4, page=16))])
def test_large(xkv, lens, news, kw):
    c = Case(xkv, lens, news, seed=len(lens), **kw)
    out, lse = c.run()
    check_large(c, out, lse)
    again, lse2 = c.run()
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_a_pool_beyond_32_bit_offsets(xkv):
    """Pages behind 2^31 bytes of codes."""
    page, d, n_pages = 128, 128, 140000
    K = torch.zeros((1, n_pages, 1, page, d), dtype=torch.uint8, device="cuda")
    c = Case(xkv, [500, 300], [2, 1], H_kv=1, n_rep=4, page=page, seed=21)
    cfg = xkv.make_cache8_config(G=1, batch=2, H_kv=1, H_q=4, d_h=d, page=page, n_pages=n_pages, max_pages=c.cfg.max_pages)
    out, lse = c.run()
    shift = n_pages - c.n_pages
    V = torch.zeros_like(K)
    K[:, shift:], V[:, shift:] = c.K, c.V
    ks, vs = torch.zeros((1, n_pages, 1), device="cuda"), torch.zeros((1, n_pages, 1), device="cuda")
    ks[:, shift:], vs[:, shift:] = c.ks, c.vs
    c.table = [[p + shift if p >= 0 else p for p in r] for r in c.table]
    c.K, c.V, c.ks, c.vs, c.cfg = K, V, ks, vs, cfg
    far, far_lse = c.run()
    assert torch.equal(far, out) and torch.equal(far_lse, lse)


def test_streams_and_graphs(xkv):
    c = Case(xkv, [700, 90], [1, 1], H_kv=2, n_rep=4, page=16, seed=22, extra=9)
    e = torch.float8_e4m3fn
    want, _ = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    got, _ = c.run(stream=s)
    s.synchronize()
    # (the buffers that `run` fills on the current stream are ready: it waited for nothing, so compare once more on one stream)
    with torch.cuda.stream(s):
        got, _ = c.run()
    s.synchronize()
    assert torch.equal(got, want)
    bufs = []
    for _ in range(2):                           # two graphs with a workspace each, replayed at once
        ws = torch.empty(xkv.xkv_cache8_workspace_bytes(c.cfg, 1), dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros_like(c.q), torch.zeros(c.q.shape[:3], device="cuda")
        args = (c.q, dev(c.first), 1, dev(c.table), dev(c.lens), c.K.view(e), c.V.view(e), c.ks, c.vs, ws, out, lse)
        graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            xkv.xkv_cache8_attend(c.cfg, 0, 1, *args)
        bufs.append((graph, st, out, args))
    for i in range(20):
        for graph, st, out, _ in bufs:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, out, _ in bufs:
        assert torch.equal(out, want)
    bufs[0][3][4].copy_(dev([650, 33]))          # lengths are read on the device: shorter sequences, the same graph
    bufs[0][0].replay()
    torch.cuda.synchronize()
    c.lens = [650, 33]
    short, lse = c.run()
    assert torch.equal(bufs[0][2], short)
    c.check(short, lse)
