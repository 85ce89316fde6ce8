"""Attention over codes where one row draws most of the weight and its value is zero: the whole output is a long even rest, which has to
keep its weights however small they are beside the loud row's."""
import math

import pytest
import torch

from tests import _cache8_ref as R
from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu
# tokens of a sequence, query heads of a KV head: blocks of 8, 16 and 128 query rows
WIDTHS = [(1, 4), (3, 4), (8, 4), (40, 7)]


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


class Rest:
    """`batch` sequences of the same pages: one holds the loud row, all others are one page of rows with equal keys and values."""

    def __init__(self, xkv, tokens, n_rep, rows, apart, batch=1, d=128, page=128, loud_at=0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.x, self.tokens, self.n_rep, self.rows, self.batch, self.d, self.page = xkv, tokens, n_rep, rows, batch, d, page
        pages = -(-rows // page)
        self.scale = float(torch.tensor(apart * math.log(2.0), dtype=torch.float32))
        self.cfg = xkv.make_cache8_config(G=1, batch=batch, H_kv=1, H_q=n_rep, d_h=d, page=page, n_pages=2, max_pages=pages,
                                          softmax_scale=self.scale)
        e = torch.float8_e4m3fn
        self.value = torch.linspace(16, 30, d, device="cuda") * (1 - 2 * torch.randint(0, 2, (d,), generator=g, device="cuda"))
        self.value = self.value.to(e)
        K, V = torch.zeros((1, 2, 1, page, d), device="cuda").to(e), torch.zeros((1, 2, 1, page, d), device="cuda").to(e)
        V.view(torch.uint8)[:] = self.value.view(torch.uint8)
        K[0, 0, 0, 0, 0] = 1.0                   # the loud row: its logit is softmax_scale, the others' 0
        V.view(torch.uint8)[0, 0, 0, 0] = 0
        self.K, self.V = K, V
        self.table = torch.ones((batch, pages), dtype=torch.int32, device="cuda")
        self.table[:, loud_at * (pages - 1)] = 0
        self.table[:, 0 if not loud_at else pages // 2] = 0
        if loud_at:
            self.table[:, pages - 1] = 1
        self.q = torch.zeros((1, batch * tokens, n_rep, d), dtype=torch.bfloat16, device="cuda")
        self.q[..., 0] = 1.0

    def run(self):
        ones = torch.ones((1, 2, 1), device="cuda")
        ws = torch.empty(self.x.xkv_cache8_workspace_bytes(self.cfg, self.tokens), dtype=torch.uint8, device="cuda")
        first = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda") * self.tokens
        length = torch.full((self.batch,), self.rows, dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(self.q, 7.0), torch.full(self.q.shape[:3], 7.0, device="cuda")
        self.x.xkv_cache8_attend(self.cfg, 0, 1, self.q, first, self.tokens, self.table, length, self.K, self.V, ones, ones, ws, out, lse)
        return out, lse

    def check(self, out, lse):
        rest = torch.arange(self.rows - self.tokens, self.rows, dtype=torch.float64, device="cuda").repeat(self.batch)[:, None]      # rows of the rest that a token sees
        w = math.exp(-self.scale)
        want = (rest * w / (1 + rest * w))[..., None] * self.value.double()
        # The output's rounding; the weights' to 16 bits, 2^-11 of themselves or 2^-34 of the largest; sums in fp32 of what all has one sign:
        # products add at most eight times a tile of 128 rows, a step of 2^-23 each, the denominator's threads eight times, half a step each;
        # logits and exponentials.
        tiles = -(-self.rows // 128) if self.batch > 1 else -(-self.rows // 128) // 148 + 1
        rel = R.BF16 + max(2.0 ** -11, 2.0 ** -34 / w) + 8 * tiles * (2.0 ** -23 + 2.0 ** -24) + 2.0 ** -12
        off = ((out[0].double() - want).abs() / want.abs()).max().item()
        assert off <= rel, (off, rel)
        total = self.scale + torch.log1p(rest * w)
        off = (lse[0].double() - total).abs()
        assert bool((off <= 2.0 ** -19 * (1 + total) + 8 * tiles * 2.0 ** -24).all()), float(off.max())


@pytest.mark.parametrize("apart", [17.3, 20.4, 23.6, 25.2, 27.9])
@pytest.mark.parametrize("tokens,n_rep", WIDTHS)
def test_a_long_even_rest(xkv, tokens, n_rep, apart):
    """One sequence, whose problem all CTAs share, and many, each of which lies in one piece or two."""
    for batch in (1, 160):
        c = Rest(xkv, tokens, n_rep, 131077, apart, batch)
        c.check(*c.run())


@pytest.mark.parametrize("tokens,n_rep", WIDTHS)
def test_a_million_rows(xkv, tokens, n_rep):
    c = Rest(xkv, tokens, n_rep, (1 << 20) + 3, 27.0)
    c.check(*c.run())


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (64, 128)])
@pytest.mark.parametrize("tokens,n_rep", WIDTHS)
def test_the_loud_row_in_the_middle(xkv, tokens, n_rep, d, page):
    """What has been summed before it is taken down, what comes after it is small from the start."""
    for batch in (1, 150):
        c = Rest(xkv, tokens, n_rep, 20011, 22.7, batch, d, page, loud_at=1)
        c.check(*c.run())


@pytest.mark.parametrize("lens,news,kw", [([40000], [1], dict(H_kv=2, n_rep=4, page=64)), ([30000, 9000], [4, 2], dict(H_kv=2, n_rep=4, page=16)),
                                          ([20000], [16], dict(H_kv=2, n_rep=4, page=32)), ([9000, 4100], [70, 3], dict(H_kv=1, n_rep=7, page=128, d=64))])
def test_random_rows_beside_a_loud_one(xkv, lens, news, kw):
    """Logits of every size, one row of value zero far above them.  Bounds as A.reference's, but that each logit's own error counts, and
    that a weight may be off by 2^-34 of the largest (times its value's scale), not 2^-21."""
    c = A.Case(xkv, lens, news, seed=31, **kw)
    K, V = (t[0].view(torch.float8_e4m3fn) for t in (c.K, c.V))
    at = c.first[0]
    for b, n in enumerate(news):                 # queries lean towards their sequence's first key, by about 14 in its logit
        p = c.table[b][0]
        c.V[0, p, :, 0] = 0
        key = K[p, :, 0].float() * c.ks[0, p][:, None]
        lean = 14.0 / c.scale * key / (key * key).sum(-1, keepdim=True)
        c.q[0, at:at + n] = (c.q[0, at:at + n].float() + lean.repeat_interleave(c.n_rep, 0)).to(torch.bfloat16)
        at += n
    out, lse = c.run()
    at = c.first[0]
    for b, (rows, n) in enumerate(zip(lens, news)):
        pages = torch.tensor(c.table[b][:-(-rows // c.page)], device="cuda")
        for g in range(K.shape[1]):
            k = (K.double()[pages, g] * c.ks[0][pages, g].double()[:, None, None]).reshape(-1, c.d)[:rows]
            v = (V.double()[pages, g] * c.vs[0][pages, g].double()[:, None, None]).reshape(-1, c.d)[:rows].abs()
            sign = V.double()[pages, g].reshape(-1, c.d)[:rows].sign()
            vsc = c.vs[0][pages, g].double().repeat_interleave(c.page)[:rows]
            mine = (0, slice(at, at + n), slice(g * c.n_rep, (g + 1) * c.n_rep))
            q = c.q[mine].double()
            z = torch.einsum("ihd,jd->ihj", q, k) * c.scale
            hidden = torch.arange(rows, device="cuda") > torch.arange(rows - n, rows, device="cuda")[:, None]
            z.masked_fill_(hidden[:, None], -math.inf)
            total = torch.logsumexp(z, -1)
            p = torch.exp(z - total[..., None])
            # a logit: d additions in fp32, each a step of the sum of magnitudes; queries to 2^-20 of their largest element
            ze = c.scale * (c.d * 2.0 ** -23 * (q.abs() @ k.abs().T) + 2.0 ** -20 * q.abs().amax(-1)[..., None] * k.abs().sum(1)) + 2.0 ** -20 * (1 + total.abs())[..., None]
            mean = (p * ze).sum(-1)              # of the denominator
            o = p @ (v * sign)
            bound = R.BF16 * o.abs() * (1 + R.BF16) + (2.0 ** -11 + 2.0 ** -16 + mean[..., None]) * (p @ v) + (p * ze) @ v \
                + 2.0 ** -34 * (p * vsc).amax(-1)[..., None] * (v / vsc[:, None]).sum(0)
            assert bool(((out[mine].double() - o).abs() <= bound).all()), float(((out[mine].double() - o).abs() / bound).max())
            assert bool(((lse[mine].double() - total).abs() <= mean + 2.0 ** -20 * (1 + total.abs())).all())
        at += n
