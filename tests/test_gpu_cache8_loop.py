"""A serving loop over a paged cache of 8-bit codes: pages, rotation, append and attention together, as a program calls them, against
attention over the uncompressed rows that the codes stand for; and its rows handed on to the uncompressed cache's operators."""
import math

import pytest
import torch

from tests import _cache8_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


class Server:
    def __init__(self, xkv, batch=3, G=2, H_kv=2, n_rep=4, d=128, page=16, rows=400, most_new=40):
        self.x, self.G, self.H_kv, self.H_q, self.d, self.batch, self.page = xkv, G, H_kv, H_kv * n_rep, d, batch, page
        max_pages = -(-rows // page)
        n_pages = batch * max_pages
        self.cfg = xkv.make_cache8_config(G=G, batch=batch, H_kv=H_kv, H_q=self.H_q, d_h=d, page=page, n_pages=n_pages, max_pages=max_pages)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((batch, max_pages), -1, **i32)
        self.ring, self.state = torch.arange(n_pages, **i32), torch.tensor([0, n_pages], **i32)
        self.length, self.first = torch.zeros(batch, **i32), torch.zeros(batch + 1, **i32)
        shape = (G, n_pages, H_kv, page, d)
        self.K, self.V = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        self.ks, self.vs = torch.zeros(shape[:3], device="cuda"), torch.zeros(shape[:3], device="cuda")
        self.ws = torch.empty(xkv.xkv_cache8_workspace_bytes(self.cfg, most_new), dtype=torch.uint8, device="cuda")
        self.rope = xkv.make_rope(d_h=d, base=500000.0, scaling="llama3", factor=8.0, original=8192.0)
        self.flags = torch.zeros(1, **i32)

    def step(self, qkv, want, max_new):
        """qkv bf16 [G][n_tok][H_q + 2 H_kv][d]: a projection's output for the new tokens."""
        x, G, Hq, Hk, n_tok = self.x, self.G, self.H_q, self.H_kv, qkv.shape[1]
        i32 = dict(dtype=torch.int32, device="cuda")
        pos, slot = torch.empty(n_tok, **i32), torch.empty(n_tok, **i32)
        x.xkv_page_assign(self.cfg, self.length, want, self.table, self.ring, self.state, self.first, self.length, pos, slot, self.flags)
        q = torch.empty((G, n_tok, Hq, self.d), dtype=torch.bfloat16, device="cuda")
        k = torch.empty((G, n_tok, Hk, self.d), dtype=torch.bfloat16, device="cuda")
        x.xkv_rope(self.rope, qkv[:, :, :Hq], pos, q, qkv[:, :, Hq:Hq + Hk], k)
        v = qkv[:, :, Hq + Hk:].contiguous()
        x.xkv_cache8_append(self.cfg, 0, G, k, v, slot, self.K, self.V, self.ks, self.vs, self.flags)
        out, lse = torch.zeros_like(q), torch.zeros((G, n_tok, Hq), device="cuda")
        x.xkv_cache8_attend(self.cfg, 0, G, q, self.first, max_new, self.table, self.length, self.K, self.V, self.ks, self.vs, self.ws, out, lse,
                            self.flags)
        return q, k, v, pos, slot, out, lse

    def check(self, q, out, lse):
        first, table, lens = self.first.tolist(), self.table.tolist(), self.length.tolist()
        for l in range(self.G):
            want, wl, bo, bl = R.attend_ref(q[l].cpu(), first, q.shape[1], table, lens, self.K[l].cpu().double(), self.V[l].cpu().double(),
                                            self.ks[l].cpu().double(), self.vs[l].cpu().double(), self.page, self.H_q // self.H_kv,
                                            1 / math.sqrt(self.d), q.shape[1])
            assert bool(((out[l].cpu().double() - want).abs() <= bo).all()) and bool(((lse[l].cpu().double() - wl).abs() <= bl).all())


def projection(s, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((s.G, n, s.H_q + 2 * s.H_kv, s.d), generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("d,page,n_rep", [(128, 16, 4), (64, 32, 7)])
def test_prompts_steps_and_turned_down_drafts(xkv, d, page, n_rep):
    s = Server(xkv, d=d, page=page, n_rep=n_rep)
    lens = [37, 21, 0]
    f, gain = R.frequencies(d, base=500000.0, scaling="llama3", factor=8.0, original=8192.0)
    kept = [[], [], []]                          # (key, value) rows of every sequence as 16-bit values, by the definition
    for step in range(9):
        if step:                                 # single tokens, drafts of which some are turned down, a third prompt
            lens = [lens[0] + 1, lens[1] + (4 if step % 3 == 1 else 1), lens[2] + (30 if step == 3 else 1 if step > 3 else 0)]
        news = [a - b for a, b in zip(lens, s.length.tolist())]
        qkv = projection(s, sum(news), step)
        q, k, v, pos, slot, out, lse = s.step(qkv, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(news))
        assert s.length.tolist() == lens and int(s.flags) == 0
        s.check(q, out, lse)
        rot, mag = R.rotate(qkv[:, :, s.H_q:s.H_q + s.H_kv].reshape(-1, s.H_kv, s.d), pos.repeat(s.G), f, gain, "half")
        assert bool(((k.reshape(rot.shape).double() - rot).abs() <= R.BF16 * rot.abs() + 2.0 ** -20 * mag).all())
        t = 0
        for b, n in enumerate(news):
            kept[b] += [(k[:, t + i], v[:, t + i]) for i in range(n)]
            t += n
        if step % 3 == 1:                        # two of the four drafts are turned down: their rows and pages go
            lens[1] -= 2
            kept[1] = kept[1][:-2]
            xkv.xkv_page_assign(s.cfg, s.length, torch.tensor(lens, dtype=torch.int32, device="cuda"), s.table, s.ring, s.state, None, s.length)
    # the rows as an uncompressed cache: within half a step of 4 bits of what went in (steps of the page's scale at its growth), and
    # the attention over it is that over the codes
    cap = 96
    K, V = (torch.zeros((s.G, s.batch, s.H_kv, cap, s.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xkv.xkv_cache8_read(s.cfg, 0, s.G, s.table, s.length, s.K, s.V, s.ks, s.vs, K, V, s.flags)
    for b in range(s.batch):
        for out16, which in ((K, 0), (V, 1)):
            x = torch.stack([r[which] for r in kept[b]], 2).double()                    # [G][H_kv][rows][d]
            y = out16[:, b, :, :lens[b]].double()
            page_top = torch.nn.functional.pad(x.abs().amax(-1), (0, -lens[b] % page)).reshape(s.G, s.H_kv, -1, page).amax(-1)
            floor = page_top.repeat_interleave(page, -1)[..., :lens[b], None] * 2.0 ** -16
            # a turned-down draft may have been louder than all that stayed, by a factor of four at most here
            assert bool(((y - x).abs() <= x.abs() * 2.0 ** -4 + 4 * floor).all())
    c = xkv.make_cache_config(G=s.G, batch=s.batch, H_kv=s.H_kv, H_q=s.H_q, d_h=s.d, cap=cap)
    q = projection(s, s.batch, 99)[:, :, :s.H_q].reshape(s.G, s.batch, 1, s.H_q, s.d).contiguous()
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(c, 1), dtype=torch.uint8, device="cuda")
    out16, out8 = torch.zeros_like(q), torch.zeros_like(q)
    xkv.xkv_tree_attend(c, 0, s.G, q, 1, None, None, K, V, s.length - 1, ws, out16)
    xkv.xkv_cache8_attend(s.cfg, 0, s.G, q.view(s.G, s.batch, s.H_q, s.d), None, 1, s.table, s.length, s.K, s.V, s.ks, s.vs, s.ws,
                          out8.view(s.G, s.batch, s.H_q, s.d))
    # two roundings of the output, one of the weights to 16 bits there
    size = V.abs().amax(dim=3).repeat_interleave(s.H_q // s.H_kv, 2)[:, :, None].double()
    assert bool(((out16.double() - out8.double()).abs() <= 4 * R.BF16 * size).all())


def test_keys_turned_back_are_what_the_factorisation_wants(xkv):
    """Rows of the cache, turned back by their positions: the keys before rotation, to the codes' rounding."""
    s = Server(xkv, batch=1, rows=200)
    qkv = projection(s, 180, 3)
    q, k, v, pos, slot, out, lse = s.step(qkv, torch.tensor([180], dtype=torch.int32, device="cuda"), 180)
    K = torch.zeros((s.G, 1, s.H_kv, 180, s.d), dtype=torch.bfloat16, device="cuda")
    xkv.xkv_cache8_read(s.cfg, 0, s.G, s.table, s.length, s.K, s.V, s.ks, s.vs, K, None)
    rows = K[:, 0].transpose(1, 2).contiguous()                      # [G][rows][H_kv][d]
    xkv.xkv_rope(s.rope, rows, pos, direction="inverse")
    raw = qkv[:, :, s.H_q:s.H_q + s.H_kv]
    pair = torch.cat([raw[..., s.d // 2:], raw[..., :s.d // 2]], -1)
    size = raw.double().abs() + pair.double().abs()
    # keys rounded to 16 bits, to 4, and to 16 again, each element of a pair counted
    assert bool(((rows.double() - raw.double()).abs() <= size * (2.0 ** -4 + 3 * R.BF16) + 2.0 ** -15 * float(raw.abs().max()) * 2).all())


def test_a_captured_step_serves_sequences_as_they_grow(xkv):
    s, t = Server(xkv, batch=2), Server(xkv, batch=2)
    start = torch.tensor([30, 47], dtype=torch.int32, device="cuda")
    prompt = projection(s, 77, 1)
    for w in (s, t):
        w.step(prompt, start, 47)
    qkv = projection(s, 2, 2)
    i32 = dict(dtype=torch.int32, device="cuda")
    want, pos, slot = start + 1, torch.empty(2, **i32), torch.empty(2, **i32)
    Hq, Hk = s.H_q, s.H_kv
    q, k = torch.empty((s.G, 2, Hq, s.d), dtype=torch.bfloat16, device="cuda"), torch.empty((s.G, 2, Hk, s.d), dtype=torch.bfloat16, device="cuda")
    v, out = torch.empty_like(k), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.xkv_page_assign(s.cfg, s.length, want, s.table, s.ring, s.state, s.first, s.length, pos, slot)
        xkv.xkv_rope(s.rope, qkv[:, :, :Hq], pos, q, qkv[:, :, Hq:Hq + Hk], k)
        v.copy_(qkv[:, :, Hq + Hk:])
        xkv.xkv_cache8_append(s.cfg, 0, s.G, k, v, slot, s.K, s.V, s.ks, s.vs)
        xkv.xkv_cache8_attend(s.cfg, 0, s.G, q, s.first, 1, s.table, s.length, s.K, s.V, s.ks, s.vs, s.ws, out)
    for i in range(40):
        qkv.copy_(projection(s, 2, 10 + i))
        graph.replay()
        eager = t.step(projection(s, 2, 10 + i), t.length + 1, 1)
        assert torch.equal(out, eager[5]) and s.length.tolist() == t.length.tolist() == [31 + i, 48 + i]
        want += 1
