"""Attention over codes at sizes drawn from the whole range, against the definition in 64 bits."""
import random

import pytest
import torch

from tests import test_gpu_cache8_attend as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.mark.parametrize("seed", range(60))
def test_drawn(xkv, seed):
    rng = random.Random(seed)
    batch = rng.choice([1, 1, 2, 3, 7, 40])
    n_rep = rng.choice([1, 2, 3, 4, 5, 7, 8, 11, 16])
    H_kv = rng.choice([1, 2, 4, 8])
    top_new = rng.choice([1, 1, 2, 5, 17, 60, 300])
    top_rows = rng.choice([60, 300, 2000, 9000]) // (4 if batch == 40 else 1)
    news = [rng.randint(0 if batch > 1 else 1, top_new) for _ in range(batch)]
    if not sum(news):
        news[0] = 1
    lens = [max(n, rng.randint(0, top_rows)) for n in news]
    c = A.Case(xkv, lens, news, H_kv=H_kv, n_rep=n_rep, d=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]), seed=seed,
               gap=rng.choice([0, 2]), scale=rng.choice([0.0, 0.02]), extra=rng.choice([0, 3]), spread=rng.choice([0.3, 1.0, 2.0]))
    out, lse = c.run()
    for t, h, o, total, bound, ze in A.reference(c):
        assert bool(((out[0, t, h].double() - o).abs() <= bound).all())
        assert bool(((lse[0, t, h].double() - total).abs() <= ze).all())
    assert int(c.flags) == 0
    for t in list(range(c.first[0])) + list(range(c.first[-1], c.n_tok)):
        assert bool((out[0, t] == 7.0).all())


def test_other_work_on_the_device_does_not_change_results(xkv):
    """Calls on two streams at once, with a workspace each, beside products that fill the device; problems that lie in many pieces."""
    cases = [A.Case(xkv, [20000], [1], H_kv=1, page=16, seed=1), A.Case(xkv, [300] * 50, [1] * 50, H_kv=4, page=32, seed=2),
             A.Case(xkv, [4000, 700], [40, 7], H_kv=2, page=64, seed=3)]
    want = [c.run()[0] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    x = torch.randn((4096, 4096), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    got = [[] for _ in cases]
    for _ in range(8):
        x @ x
        for c, s, g in zip(cases, streams, got):
            with torch.cuda.stream(s):
                g.append(c.run()[0])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w, y) for y in g)
