"""Pages, positions and slots from lengths, against the definition sequence by sequence."""
import random

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


class World:
    """A ring and a table that calls change, beside their definition."""

    def __init__(self, xkv, page, n_pages, max_pages, batch, head=0):
        self.x, self.page, self.n_pages, self.max_pages, self.batch = xkv, page, n_pages, max_pages, batch
        self.cfg = xkv.make_cache8_config(G=1, batch=batch, H_kv=1, H_q=1, d_h=64, page=page, n_pages=n_pages, max_pages=max_pages)
        ids = list(range(n_pages))
        random.Random(n_pages).shuffle(ids)
        self.ring, self.state = ids, [head, n_pages]
        self.table = [[-7] * max_pages for _ in range(batch)]
        self.d = [dev(self.table), dev(self.ring), dev(self.state)]
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(self, held, want, n_tok=None, tokens=True, in_place=False):
        total = sum(max(min(max(w, 0), self.max_pages * self.page) - min(max(h, 0), self.max_pages * self.page), 0) for h, w in zip(held, want))
        n_tok = total if n_tok is None else n_tok
        h, w = dev(held), dev(want)
        first = torch.full((self.batch + 1,), 99, dtype=torch.int32, device="cuda")
        length = h if in_place else torch.full((self.batch,), 99, dtype=torch.int32, device="cuda")
        pos, slot = (torch.full((n_tok,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        self.flags.zero_()
        if tokens:
            self.x.xkv_page_assign(self.cfg, h, w, *self.d, first, length, pos, slot, self.flags)
        else:
            self.x.xkv_page_assign(self.cfg, h, w, *self.d, None, length, flags=self.flags)
        want_all = R.assign_ref(self.page, self.n_pages, self.max_pages, held, want, self.table, self.ring, self.state, n_tok if tokens else total)
        self.table, self.ring, self.state, first_r, length_r, pos_r, slot_r, flagged = want_all
        assert self.d[0].tolist() == self.table
        assert self.d[1].tolist() == self.ring and self.d[2].tolist() == self.state
        assert length.tolist() == length_r
        if tokens:
            assert first.tolist() == first_r and pos.tolist() == pos_r and slot.tolist() == slot_r
        assert bool(self.flags.item()) == flagged
        return length_r


@pytest.mark.parametrize("page,max_pages,batch", [(16, 9, 1), (16, 300, 33), (32, 5, 64), (64, 7, 1023), (128, 3, 1025), (16, 2, 2500)])
def test_a_life_of_calls(xkv, page, max_pages, batch):
    rng = random.Random(batch)
    most = max_pages * page
    w = World(xkv, page, batch * max_pages // 2 + 3, max_pages, batch, head=batch // 2 % 3)
    held = [0] * batch
    for step in range(6):
        want = [rng.choice([h, min(most, h + 1), min(most, h + rng.randrange(3 * page)), rng.randrange(h + 1), 0 if step % 2 else h]) for h in held]
        held = w.call(held, want, in_place=step % 3 == 2)
    assert w.call(held, [0] * batch, tokens=False) == [0] * batch
    assert w.state[1] == w.n_pages and sorted(w.ring) == list(range(w.n_pages))          # every page has come back


def test_pages_run_out(xkv):
    w = World(xkv, 16, 10, 8, 6)
    # 3 + 4 pages go; the third wants 4 of 3 and gets none, and so does the fourth, who comes behind it; the fifth needs none
    held = w.call([0, 0, 0, 0, 0, 0], [48, 64, 64, 16, 0, 0])
    assert held == [48, 64, 0, 0, 0, 0]
    held = w.call(held, [48, 10, 64, 16, 3, 128])     # what the second gives back is there from the next call on
    assert held == [48, 10, 0, 0, 0, 0]
    assert w.call(held, [49, 10, 64, 16, 3, 0]) == [49, 10, 64, 16, 0, 0]


def test_out_of_range(xkv):
    w = World(xkv, 16, 20, 4, 3)
    held = w.call([0, -5, 0], [70, 20, -3])           # more than a table's row has room for, negative lengths
    assert held == [64, 20, 0]
    w.call(held, [70, 33, 1000], n_tok=7)             # fewer places than tokens
    w = World(xkv, 16, 20, 4, 2)
    w.state = [25, 3]
    w.d[2].copy_(dev(w.state))
    w.call([0, 0], [16, 16])                          # a state out of range: no page is free
    w = World(xkv, 16, 4, 8, 2)
    w.call([0, 0], [64, 0])
    w.call([64, 40], [0, 0])                          # the second never had pages: six come back to a ring with room for four
    w = World(xkv, 16, 6, 8, 2)
    w.ring = [3, -1, 77, 2, 1, 0]
    w.d[1].copy_(dev(w.ring))
    w.call([0, 0], [40, 17])                          # page numbers out of range: their tokens get no slot


def test_more_places_than_tokens(xkv):
    w = World(xkv, 32, 30, 6, 4)
    w.call([0, 0, 0, 0], [100, 0, 33, 1], n_tok=200)
    w.call([100, 0, 33, 1], [100, 0, 33, 1], n_tok=3)
    w.call([100, 0, 33, 1], [100, 0, 33, 1], n_tok=0)


def test_a_long_prompt_and_a_captured_step(xkv):
    w = World(xkv, 16, 3000, 2000, 3)
    held = w.call([0, 0, 0], [31000, 5, 9000])
    batch = 3
    h, want = dev(held), dev([x + 1 for x in held])
    first, pos, slot = dev([0] * 4), dev([0] * 3), dev([0] * 3)
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        xkv.xkv_page_assign(w.cfg, h, want, *w.d, first, h, pos, slot)
    for _ in range(20):
        graph.replay()
        torch.cuda.synchronize()
        r = R.assign_ref(16, 3000, 2000, held, want.tolist(), w.table, w.ring, w.state, batch)
        w.table, w.ring, w.state, _, held, pos_r, slot_r, _ = r
        assert pos.tolist() == pos_r and slot.tolist() == slot_r and h.tolist() == held
        assert w.d[0].tolist() == w.table and w.d[2].tolist() == w.state
        want += 1
