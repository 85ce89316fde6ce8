"""A sequence handed from the paged cache of codes to the compressed window: its rows read back, keys turned back into the matrix that the
factorisation takes, landmarks, values; and to dense attention over the uncompressed rows."""
import math

import numpy as np
import pytest
import torch

from paper_2503_18893_b200 import synth
from tests import _cache8_ref as R
from tests import _cases as C
from tests.test_gpu_clf import _factorize_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


class Handed:
    def __init__(self, xkv, over, page):
        s = self.s = synth.config(1, **over)
        G, H, d, T = s.G, s.H_kv, s.d_h, s.T
        raw_k, raw_v = (t.cuda().view(G, T, H, d) for t in synth.make_kv(s))
        self.plan = xkv.make_rope(d_h=d, base=s.rope_base)
        self.pos = torch.arange(T, dtype=torch.int32, device="cuda")
        rotated = torch.empty_like(raw_k)
        xkv.xkv_rope(self.plan, raw_k, self.pos, rotated)
        n = -(-T // page)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.cfg = xkv.make_cache8_config(G=G, batch=1, H_kv=H, H_q=s.H_q, d_h=d, page=page, n_pages=n + 3, max_pages=n)
        self.table = torch.randperm(n + 3, generator=torch.Generator().manual_seed(1))[:n].to(torch.int32).cuda()[None].contiguous()
        slot = self.table[0].repeat_interleave(page)[:T] * page + self.pos % page
        self.K8, self.V8 = (torch.zeros((G, n + 3, H, page, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        self.ks, self.vs = (torch.zeros((G, n + 3, H), device="cuda") for _ in range(2))
        for a, b in ((0, T // 3 + 5), (T // 3 + 5, T)):             # a prompt in two chunks
            xkv.xkv_cache8_append(self.cfg, 0, G, rotated[:, a:b].contiguous(), raw_v[:, a:b].contiguous(), slot[a:b].to(torch.int32).contiguous(), self.K8,
                                  self.V8, self.ks, self.vs)
        self.length = torch.tensor([T], **i32)
        self.K, self.V = (torch.zeros((G, 1, H, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        xkv.xkv_cache8_read(self.cfg, 0, G, self.table, self.length, self.K8, self.V8, self.ks, self.vs, self.K, self.V)
        self.raw_k, self.raw_v, self.rotated = raw_k, raw_v, rotated

    def matrices(self, xkv):
        """X [T][G*H_kv*d_h] of keys before rotation, in one call, and of values."""
        s = self.s
        X = torch.empty((s.T, s.G * s.H_kv, s.d_h), dtype=torch.bfloat16, device="cuda")
        xkv.xkv_rope(self.plan, self.K.view(s.G * s.H_kv, s.T, s.d_h).transpose(0, 1), self.pos, X, direction="inverse")
        Xv = self.V.view(s.G * s.H_kv, s.T, s.d_h).transpose(0, 1).contiguous()
        return X.view(s.T, -1), Xv.view(s.T, -1)


CASES = [(dict(T=2048), 64, 16), (dict(T=1501, G=4, H_kv=2, d_h=128, rho=48), 96, 64)]


@pytest.mark.parametrize("over,r,page", CASES)
def test_factorisation(xkv, over, r, page):
    h = Handed(xkv, over, page)
    s = h.s
    for X, raw, turned in zip(h.matrices(xkv), (h.raw_k, h.raw_v), (True, False)):
        x, want = X.double(), raw.transpose(0, 1).reshape(s.T, -1).double()
        # codes are half a step of four bits off (of the page's largest, 2^-14 of it below), keys are rounded to 16 bits twice more and turned
        size = want.view(s.T, -1, s.d_h).abs()
        size = size + torch.cat([size[..., s.d_h // 2:], size[..., :s.d_h // 2]], -1) if turned else size
        assert bool(((x - want).abs() <= size.view(s.T, -1) * (2.0 ** -4 + 3 * R.BF16) + 2.0 ** -13 * float(size.max())).all())
        noise = float((x - want).norm())
        A, B, sig, _ = _factorize_gpu(X, s.G, s.d, r, 32, 2, seed=5)
        back = torch.cat([A.double() @ B[l].double() for l in range(s.G)], 1)
        tail = lambda m: float((torch.linalg.svdvals(m)[r:] ** 2).sum().sqrt())
        res = float((x - back).norm())
        assert res ** 2 <= 1.15 * tail(x) ** 2   # as for any matrix of this kind
        # and against the rows that went in: the optimum of theirs, and what the codes added, at most
        assert float((want - back).norm()) <= math.sqrt(1.15) * (tail(want) + noise) + noise
        assert noise <= 0.04 * float(want.norm())


@pytest.mark.parametrize("over,r,page", CASES)
def test_landmarks(xkv, over, r, page):
    h = Handed(xkv, over, page)
    s = h.s
    marks = [torch.empty((1, s.G, s.H_kv, s.n_c, s.d_h), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows = h.K[:, 0].transpose(1, 2).reshape(1, s.G, s.T, s.d)      # rotated as they are: no base
    for keys, m, base in ((rows.contiguous(), marks[0], 0.0), (h.raw_k.reshape(1, s.G, s.T, s.d).contiguous(), marks[1], s.rope_base)):
        xkv.xkv_build_landmarks(keys, m, G=s.G, batch=1, T=s.T, H_kv=s.H_kv, d_h=s.d_h, chunk=s.c, rope_base=base)
    size = torch.nn.functional.pad(h.rotated.double().abs(), (0, 0, 0, 0, 0, -s.T % s.c)).view(s.G, s.n_c, s.c, s.H_kv, s.d_h).mean(2).transpose(1, 2)[None]
    size = size * (s.c / torch.tensor([min(s.c, s.T - j * s.c) for j in range(s.n_c)], device="cuda", dtype=torch.float64))[:, None]
    off = (marks[0].double() - marks[1].double()).abs()
    assert bool((off <= size * (2.0 ** -4 + 4 * R.BF16) + 2.0 ** -13 * float(h.rotated.abs().max())).all())


def test_dense_attention(xkv):
    h = Handed(xkv, dict(T=2048), 32)
    s = h.s
    g = C.GpuCase(s, C.case_from_factors(s))
    q = torch.randn((s.G, 1, s.H_q, s.d_h), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.bfloat16)
    out16, out8 = torch.zeros_like(q), torch.zeros_like(q)
    lse16, lse8 = (torch.zeros(q.shape[:3], device="cuda") for _ in range(2))
    ws16 = torch.empty(xkv.xkv_dense_workspace_bytes(g.grp, s.T), dtype=torch.uint8, device="cuda")
    ws8 = torch.empty(xkv.xkv_cache8_workspace_bytes(h.cfg, 1), dtype=torch.uint8, device="cuda")
    xkv.xkv_dense_attend(g.grp, 0, s.G, q, h.K, h.V, h.length, s.T, ws16, out16, lse16)
    xkv.xkv_cache8_attend(h.cfg, 0, s.G, q, None, 1, h.table, h.length, h.K8, h.V8, h.ks, h.vs, ws8, out8, lse8)
    # an output is a mean of values: weights to 2^-9 of themselves there, to 2^-11 here, each output rounded
    size = h.V.double().abs().amax(3).repeat_interleave(s.n_rep, 2)
    assert bool(((out16.double() - out8.double()).abs() <= 4 * R.BF16 * size).all())
    np.testing.assert_allclose(lse16.cpu().numpy(), lse8.cpu().numpy(), atol=1e-3)
    g.close()
