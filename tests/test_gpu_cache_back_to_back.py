"""The operators over an uncompressed cache one behind the other in a stream, each reading what the one before has just written,
give the same bits as with the device idle in between."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


@pytest.mark.parametrize("d,H,rows,keep", [(64, 2, 700, 600), (128, 8, 4000, 3000), (128, 3, 30000, 9000)])
def test_a_chain_without_a_pause(xkv, d, H, rows, keep):
    n, path_n, steps = 6, 4, 12
    cap = rows + n
    cfg = xkv.make_cache_config(G=1, batch=2, H_kv=H, H_q=2 * H, d_h=d, cap=cap)
    g = torch.Generator().manual_seed(rows)
    start = [torch.randn((1, 2, H, cap, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    q = torch.randn((steps, 1, 2, n, 2 * H, d), generator=g).to(torch.bfloat16).cuda()
    path = torch.stack([torch.randperm(n, generator=g)[:path_n].sort().values for _ in range(2)]).to(torch.int32).cuda()
    lens = [rows, rows - 50]
    visible = i32([[x + path[b].tolist().index(i) + 1 if i in path[b].tolist() else 0 for i in range(n)] for b, x in enumerate(lens)])
    length, after, flags = i32(lens), i32([x + path_n for x in lens]), i32([0])
    positions = [i32([cap + 10 * t, cap + 10 * t]) for t in range(steps)]
    since = [i32([rows // 2 + 40 * t] * 2) for t in range(steps)]

    def run(pause):
        K, V = (t.clone() for t in start)
        w = torch.ones((1, 2, H, cap), device="cuda")
        pos = torch.arange(cap, dtype=torch.int32, device="cuda").expand(1, 2, H, cap).contiguous()
        out, lse = torch.zeros_like(q[0]), torch.zeros(q[0].shape[:-1], device="cuda")
        ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
        src = torch.zeros((steps, 1, 2, H, keep), dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        for t in range(steps):                   # nothing of torch's lies between the calls
            for call in (lambda: xkv.xkv_tree_attend(cfg, 0, 1, q[t], n, None, None, K, V, length, ws, out, lse, flags),
                         lambda: xkv.xkv_tree_commit(cfg, 0, 1, K, V, length, path, None, path_n, pos, positions[t], flags),
                         lambda: xkv.xkv_cache_weigh(cfg, 0, 1, q[t], n, lse, K, after, visible, length, 0.75, w, flags),
                         lambda: xkv.xkv_evict_select(cfg, 0, 1, w, pos, since[t], after, keep, src[t], flags),
                         lambda: xkv.xkv_evict_compact(cfg, 0, 1, K, V, src[t], keep, w, pos, flags)):
                call()
                if pause:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return K, V, w, pos, out, lse, src

    want = run(True)
    for _ in range(5):
        for got, right in zip(run(False), want):
            assert torch.equal(got, right)
    assert flags.item() == 0
