"""Rows into 8-bit codes and back: every code and scale is the definition's."""
import math

import pytest
import torch

from tests import _cache8_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    def __init__(self, xkv, G, H, d, page, n_pages, batch=1, max_pages=1, seed=0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.cfg = xkv.make_cache8_config(G=G, batch=batch, H_kv=H, H_q=H, d_h=d, page=page, n_pages=n_pages, max_pages=max_pages)
        self.x, self.G, self.H, self.d, self.page, self.n_pages = xkv, G, H, d, page, n_pages
        shape = (G, n_pages, H, page, d)
        # any byte may lie in a page that no call has written; scales likewise (append reads one only where rows lie before its run)
        self.K, self.V = (torch.randint(0, 256, shape, generator=self.g, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2))
        self.ks, self.vs = (2.0 ** torch.randint(-20, 5, shape[:3], generator=self.g, device="cuda").float() for _ in range(2))
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    def append(self, k, v, slot, layers=None):
        ref = []
        for codes, scale, x in ((self.K, self.ks, k), (self.V, self.vs, v)):
            val, s = codes.cpu().double(), scale.cpu().double()
            l0, l1 = layers or (0, self.G)
            R.append_ref(val[l0:l1], s[l0:l1], x.cpu()[l0:l1], slot, self.page)
            ref.append((val, s))
        self.flags.zero_()
        self.x.xkv_cache8_append(self.cfg, *(layers or (0, self.G)), k, v, dev(slot), self.K, self.V, self.ks, self.vs, self.flags)
        for (val, s), codes, scale in zip(ref, (self.K, self.V), (self.ks, self.vs)):
            assert torch.equal(scale.cpu().double(), s)
            got = codes.cpu().double()
            assert torch.equal(got.isnan(), val.isnan()) and torch.equal(got.nan_to_num(7.0), val.nan_to_num(7.0))


def rows(p, n, scale=1.0):
    return (scale * torch.randn((p.G, n, p.H, p.d), generator=p.g, device="cuda")).to(torch.bfloat16)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d,G,H", [(128, 1, 2), (64, 2, 3)])
def test_runs_of_every_kind(xkv, page, d, G, H):
    p = Pool(xkv, G, H, d, page, 7)
    p.append(rows(p, 1), rows(p, 1), [3 * page])                                       # a page's first row
    p.append(rows(p, 1, 30.0), rows(p, 1, 1e-3), [3 * page + 1])                       # a louder row, a fainter one
    p.append(rows(p, page - 2, 2.0), rows(p, page - 2), list(range(3 * page + 2, 4 * page)))       # up to the page's end
    p.append(rows(p, page), rows(p, page), list(range(5 * page, 6 * page)))             # a whole page
    long = list(range(page + 5, 2 * page)) + list(range(page * 6, page * 7)) + list(range(0, page // 2 + 1))
    p.append(rows(p, len(long)), rows(p, len(long), 100.0), long)                       # a sequence through pages in no order
    p.append(rows(p, 3, 1e4), rows(p, 3, 1e-4), [4 * page, 2 * page + 7, page // 2 + 1])            # three sequences' tokens
    assert int(p.flags) == 0


def test_slots_that_are_skipped(xkv):
    p = Pool(xkv, 1, 2, 64, 16, 4)
    p.append(rows(p, 6), rows(p, 6), [-1, 5, 6, -1, 17, 18])
    assert int(p.flags) == 0
    for bad in (64, 65, -2, 1 << 30, -(1 << 31)):
        p.append(rows(p, 3), rows(p, 3), [20, bad, 33])
        assert int(p.flags) == xkv.XKV_FLAG_INDEX_RANGE
    p.append(rows(p, 2), rows(p, 2), [-1, -1])
    p.append(rows(p, 0), rows(p, 0), [])


def test_only_the_layers_asked_for(xkv):
    p = Pool(xkv, 4, 1, 128, 16, 3)
    p.append(rows(p, 20), rows(p, 20), list(range(16, 36)), layers=(1, 3))


@pytest.mark.parametrize("d", [64, 128])
def test_values_at_borders(xkv, d):
    """Largest magnitudes on both sides of 448 * 2^e, ties between codes, zeros, the smallest scale, infinities and NaN."""
    p = Pool(xkv, 1, 1, d, 16, 20)
    at = 0
    for top in (448.0, 450.0, 446.0, 447.9, 1.75, 1.7578125, 7.0 * 2.0 ** -70, 2.0 ** -80, 0.0, 3.3e38, 1e-38, 2.0 ** -133):
        x = torch.zeros((1, 16, 1, d))
        x[0, :, 0] = torch.linspace(-1, 1, 16 * d).reshape(16, d) * min(top, 1e38)
        x[0, 3, 0, 5] = top
        x = x.to(torch.bfloat16).cuda()
        p.append(x, -x, list(range(at, at + 16)))
        at += 16
    ties = torch.tensor([(8 + i / 2) / 8 * 2.0 ** k for k in range(-12, 8) for i in range(16)][:d], dtype=torch.float32).to(torch.bfloat16)
    x = ties.reshape(1, 1, 1, d).cuda()
    p.append(x, x, [at])
    y = x.clone()
    y[..., 0], y[..., 1], y[..., 2], y[..., 3] = math.inf, -math.inf, math.nan, -0.0
    p.append(y, x, [at + 1])
    p.append(torch.full_like(x, math.inf), torch.full_like(x, math.nan), [at + 2])
    p.append(x * 64, x * 8, [at + 3])                                                  # codes move down, NaN stays
    p.append(torch.full_like(x, math.nan), torch.full_like(x, -math.inf), [at + 16])    # a page whose first row is not finite


def test_a_scale_grows_step_by_step_as_at_once_but_for_faint_values(xkv):
    p = Pool(xkv, 1, 1, 128, 32, 2, seed=3)
    for i in range(32):
        p.append(rows(p, 1, 2.0 ** (i / 3 - 3)), rows(p, 1, 2.0 ** (3 - i / 3)), [32 + i])


@pytest.mark.parametrize("page,cap,lens", [(16, 40, [37, 0, 1, 40]), (128, 300, [300, 129, 128, 5]), (64, 65, [64, 65, 63, 2])])
@pytest.mark.parametrize("d", [64, 128])
def test_read(xkv, page, cap, lens, d):
    batch, most = len(lens), -(-cap // page) + 1
    p = Pool(xkv, 2, 3, d, page, batch * most + 2, batch, most, seed=page)
    table = torch.randperm(batch * most + 2, generator=torch.Generator().manual_seed(1))[:batch * most].reshape(batch, most).to(torch.int32)
    K, V = (torch.full((2, batch, 3, cap, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table[2, 0] = -1 if lens[2] < 100 else int(table[2, 0])
    xkv.xkv_cache8_read(p.cfg, 0, 2, table.cuda(), dev(lens), p.K, p.V, p.ks, p.vs, K, V, p.flags)
    for codes, scale, out in ((p.K, p.ks, K), (p.V, p.vs, V)):
        want = torch.full(out.shape, 5.0, dtype=torch.float64)
        for b, n in enumerate(lens):
            for j in range(n):
                t = int(table[b, j // page])
                if t >= 0:
                    want[:, b, :, j] = codes.view(torch.uint8)[:, t, :, j % page].view(torch.float8_e4m3fn).cpu().double() * scale[:, t].cpu().double()[..., None]
        got = out.cpu().double()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(9.0), want.nan_to_num(9.0))
    assert int(p.flags) == (xkv.XKV_FLAG_INDEX_RANGE if -1 in table[2].tolist() else 0)
    p.flags.zero_()
    K2 = torch.full_like(K, 5.0)
    xkv.xkv_cache8_read(p.cfg, 1, 2, table.cuda(), dev([cap + 9] + lens[1:]), p.K, p.V, p.ks, p.vs, K2, None, p.flags)      # cut to cap
    assert int(p.flags) == xkv.XKV_FLAG_INDEX_RANGE and bool((K2[0] == 5.0).all())
    assert torch.equal(K2[1, 1:].view(torch.int16), K[1, 1:].view(torch.int16))


def test_a_captured_append_and_read(xkv):
    p = Pool(xkv, 1, 2, 128, 16, 3, batch=1, max_pages=3)
    k, v, slot = rows(p, 1), rows(p, 1), dev([0])
    out, length, table = torch.zeros((1, 1, 2, 48, 128), dtype=torch.bfloat16, device="cuda"), dev([1]), dev([[0, 1, 2]])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.xkv_cache8_append(p.cfg, 0, 1, k, v, slot, p.K, p.V, p.ks, p.vs)
        xkv.xkv_cache8_read(p.cfg, 0, 1, table, length, p.K, p.V, p.ks, p.vs, out, None)
    val, s = p.K.cpu().double(), p.ks.cpu().double()
    for i in range(40):
        k.normal_()
        slot.fill_(i)
        length.fill_(i + 1)
        R.append_ref(val, s, k.cpu(), [i], 16)
        graph.replay()
        torch.cuda.synchronize()
        want = (val * s[..., None, None]).transpose(1, 2).reshape(1, 2, 48, 128)[:, :, :i + 1]
        assert torch.equal(out[0, 0, :, :i + 1].cpu().double(), want[0])
