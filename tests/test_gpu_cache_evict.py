"""xkv_evict_select, xkv_evict_compact and xkv_tree_commit against their definitions: exact."""
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


def select(xkv, w, pos, since, lens, keep, layers=None):
    G, batch, H, cap = w.shape
    cfg = xkv.make_cache_config(G=G, batch=batch, H_kv=H, H_q=H, d_h=64, cap=cap)
    src = torch.full((G, batch, H, keep), -7, dtype=torch.int32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    l0, l1 = layers or (0, G)
    xkv.xkv_evict_select(cfg, l0, l1, w.cuda(), None if pos is None else i32(pos), None if since is None else i32(since),
                         None if lens is None else i32(lens), keep, src, flags)
    return src.cpu(), flags.item()


def check_select(w, pos, since, lens, keep, src, layers=None):
    G, batch, H, cap = w.shape
    for l in range(*(layers or (0, G))):
        for b in range(batch):
            for h in range(H):
                want = R.select_ref(w[l, b, h], None if pos is None else pos[l, b, h], None if since is None else since[b],
                                    cap if lens is None else lens[b], keep)
                assert src[l, b, h].tolist() == want, (l, b, h)


def weights(kind, shape, g):
    w = torch.rand(shape, generator=g)
    if kind == "ties":
        w = (w * 5).floor()
    elif kind == "equal":
        w = torch.full(shape, 0.25)
    elif kind == "special":
        pick = (w * 12).floor()
        for i, x in enumerate((math.inf, -math.inf, math.nan, 0.0, -0.0, 1e-45, -1e-45, -3.0, 3.4e38)):
            w = torch.where(pick == i, torch.tensor(x), w)
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "special"])
@pytest.mark.parametrize("cap,keep", [(1, 1), (2, 1), (33, 7), (1024, 1000), (1025, 1024), (4097, 4000), (5000, 100), (9001, 4500), (20000, 19999),
                                      (40001, 20000)])
def test_select(xkv, kind, cap, keep):
    g = torch.Generator().manual_seed(cap)
    w = weights(kind, (1, 2, 2, cap), g)
    pos = torch.stack([torch.randperm(2 * cap, generator=g)[:cap] for _ in range(4)]).reshape(1, 2, 2, cap)
    for since in (None, [2 * cap - cap // 3, cap // 4]):             # recent rows that all stay; more than there is room for
        src, flags = select(xkv, w, pos, since, [cap, max(1, cap - 3)], keep)
        assert flags == 0
        check_select(w, pos, since, [cap, max(1, cap - 3)], keep, src)


def test_select_lengths(xkv):
    g = torch.Generator().manual_seed(1)
    lens = [0, 1, 99, 100, 101, 6000]
    w = weights("ties", (2, 6, 1, 6000), g)
    src, _ = select(xkv, w, None, [0, 0, 50, 50, 50, 5990], lens, 100, layers=(1, 2))
    assert (src[0] == -7).all()
    check_select(w, None, [0, 0, 50, 50, 50, 5990], lens, 100, src, layers=(1, 2))
    src, flags = select(xkv, w, None, None, None, 100)
    check_select(w, None, None, None, 100, src)
    assert flags == 0
    src, flags = select(xkv, w, None, None, [0, -4, 99, 100, 101, 7000], 100)
    assert flags == xkv.XKV_FLAG_INDEX_RANGE
    check_select(w, None, None, [0, 0, 99, 100, 101, 6000], 100, src)


def test_select_at_the_largest_cache(xkv):
    g = torch.Generator().manual_seed(2)
    cap = xkv.XKV_EVICT_MAX_ROWS
    w = weights("ties", (1, 1, 1, cap), g) + torch.rand((1, 1, 1, cap), generator=g).round()
    src, _ = select(xkv, w, None, [cap - 1000], [cap], 65536)
    check_select(w, None, [cap - 1000], [cap], 65536, src)


def cache(G, batch, H, cap, d, g):
    K, V = (torch.randn((G, batch, H, cap, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    return K, V, torch.rand((G, batch, H, cap), generator=g).cuda(), torch.randint(0, 10 ** 6, (G, batch, H, cap), generator=g, dtype=torch.int32).cuda()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,keep", [(2, 1), (300, 150), (1000, 970), (5003, 257)])
def test_compact(xkv, d, cap, keep):
    g = torch.Generator().manual_seed(cap + d)
    G, batch, H = 2, 2, 3
    K, V, w, pos = cache(G, batch, H, cap, d, g)
    src, _ = select(xkv, w.cpu(), None, None, [cap, cap], keep)
    old = [t.clone() for t in (K, V, w, pos)]
    cfg = xkv.make_cache_config(G=G, batch=batch, H_kv=H, H_q=H, d_h=d, cap=cap)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    xkv.xkv_evict_compact(cfg, 1, 2, K, V, src.cuda(), keep, w, pos, flags)
    assert flags.item() == 0
    for got, was in zip((K, V, w, pos), old):
        assert torch.equal(got[0], was[0]) and torch.equal(got[1][:, :, keep:], was[1][:, :, keep:])
        for b in range(batch):
            for h in range(H):
                assert torch.equal(got[1, b, h, :keep], was[1, b, h][src[1, b, h].long().cuda()])


def test_compact_skips_and_reports_what_is_no_row_behind(xkv):
    g = torch.Generator().manual_seed(4)
    K, V, w, pos = cache(1, 1, 1, 50, 64, g)
    old = [t.clone() for t in (K, V, w, pos)]
    cfg = xkv.make_cache_config(G=1, batch=1, H_kv=1, H_q=1, d_h=64, cap=50)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in (5, 50, 2 ** 31 - 1):
        flags.zero_()
        src = torch.arange(10, dtype=torch.int32)
        src[2], src[3], src[4] = bad, 49, -1
        xkv.xkv_evict_compact(cfg, 0, 1, K, V, i32(src).reshape(1, 1, 1, 10), 10, w, pos, flags)
        assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE
        for got, was in zip((K, V, w, pos), old):
            want = was.clone()
            want[0, 0, 0, 3] = was[0, 0, 0, 49]
            assert torch.equal(got, want)
    xkv.xkv_evict_compact(cfg, 0, 1, K, V, i32([20] * 10).reshape(1, 1, 1, 10), 10)    # the same row to all, neither weights nor positions
    assert all(torch.equal(K[0, 0, 0, j], old[0][0, 0, 0, 20]) for j in range(10)) and torch.equal(w[..., 4:], old[2][..., 4:])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_path", [1, 5, 64, 65, 256])
def test_commit(xkv, d, n_path):
    g = torch.Generator().manual_seed(n_path + d)
    G, batch, H, cap = 2, 3, 2, 700
    K, V, _, pos = cache(G, batch, H, cap, d, g)
    old = [t.clone() for t in (K, V, pos)]
    lens = [0, 100, cap - 300]
    for shuffled in (False, True):
        K, V, pos = (t.clone() for t in old)
        path = torch.stack([torch.randperm(300, generator=g)[:n_path] for _ in range(batch)]).to(torch.int32)
        if not shuffled:
            path = path.sort(1).values
        m = [n_path, n_path // 2, 0 if shuffled else max(1, n_path - 1)]
        cfg = xkv.make_cache_config(G=G, batch=batch, H_kv=H, H_q=H, d_h=d, cap=cap)
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        xkv.xkv_tree_commit(cfg, 0, 1, K, V, i32(lens), path.cuda(), i32(m), n_path, pos, i32([1000, 2000, 3000]), flags)
        assert flags.item() == 0
        for b in range(batch):
            for got, was in ((K, old[0]), (V, old[1])):
                want = was.clone()
                want[0, b, :, lens[b]:lens[b] + m[b]] = was[0, b][:, lens[b] + path[b, :m[b]].long().cuda()]
                assert torch.equal(got[:, b], want[:, b])
            want = old[2][:, b].clone()
            want[0, :, lens[b]:lens[b] + m[b]] = 1000 * (b + 1) + torch.arange(m[b], dtype=torch.int32, device="cuda")
            assert torch.equal(pos[:, b], want)


def test_commit_skips_and_reports_rows_that_are_none(xkv):
    g = torch.Generator().manual_seed(5)
    K, V, _, pos = cache(1, 1, 1, 20, 64, g)
    cfg = xkv.make_cache_config(G=1, batch=1, H_kv=1, H_q=1, d_h=64, cap=20)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    old = K.clone()
    xkv.xkv_tree_commit(cfg, 0, 1, K, V, i32([10]), i32([[3, -1, 10, 2 ** 31 - 1, 9]]), None, 5, flags=flags)
    assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE
    want = old.clone()
    want[0, 0, 0, 10], want[0, 0, 0, 14] = old[0, 0, 0, 13], old[0, 0, 0, 19]
    assert torch.equal(K, want)
    for lens, path_len in (([-1], None), ([20], None), ([2 ** 31 - 1], None)):
        flags.zero_()
        xkv.xkv_tree_commit(cfg, 0, 1, K, V, i32(lens), i32([[0, 1, 2, 3, 4]]), path_len, 5, flags=flags)
        assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE and torch.equal(K, want)
    flags.zero_()
    xkv.xkv_tree_commit(cfg, 0, 1, K, V, i32([10]), i32([[0, 1, 2, 3, 4]]), i32([9]), 5, flags=flags)
    assert flags.item() == xkv.XKV_FLAG_INDEX_RANGE and torch.equal(K, want)
