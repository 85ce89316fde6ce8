"""The operators over an uncompressed cache as a serving program runs them: verify drafts, commit the accepted path, weigh the
rows, evict and go on -- eagerly and as one captured graph, beside a plain program over lists of tokens."""
import math

import pytest
import torch

from tests import _cache_ref as R

pytestmark = pytest.mark.gpu

G, BATCH, H_KV, REP, D, N = 2, 2, 2, 3, 128, 12
KEEP, RECENT, HIGH = 150, 20, 170


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def bf16(*shape, g):
    return torch.randn(shape, generator=g).to(torch.bfloat16)


class Plain:
    """Per layer, sequence and head: a list of rows (key, value, weight, position), in 64 bits."""

    def __init__(self, K, V, lens):
        self.rows = {(l, b, h): [[K[l, b, h, j].double(), V[l, b, h, j].double(), 0.0, j] for j in range(lens[b])]
                     for l in range(G) for b in range(BATCH) for h in range(H_KV)}

    def step(self, q, k, v, sees, paths, new):
        """Verifies drafts, takes the accepted ones in, adds their weights; returns the outputs."""
        out = torch.zeros((G, BATCH, N, H_KV * REP, D), dtype=torch.float64)
        for (l, b, h), rows in self.rows.items():
            K0 = torch.stack([r[0] for r in rows])
            V0 = torch.stack([r[1] for r in rows])
            K = torch.cat([K0, k[l, b, h].double()])
            V = torch.cat([V0, v[l, b, h].double()])
            at = torch.cat([torch.ones((N, len(rows)), dtype=torch.bool), sees[b]], 1)
            weights = torch.zeros(len(rows) + N, dtype=torch.float64)
            for i in range(N):
                for r in range(REP):
                    z = (K @ q[l, b, i, h * REP + r].double()) / math.sqrt(D)
                    z[~at[i]] = -math.inf
                    p = torch.softmax(z, 0)
                    out[l, b, i, h * REP + r] = p @ V
                    if i in paths[b]:
                        weights += p
            for j, row in enumerate(rows):
                row[2] += float(weights[j])
            for m, i in enumerate(paths[b]):
                rows.append([k[l, b, h, i].double(), v[l, b, h, i].double(), float(weights[len(rows) - m + i]), new[b] + m])
        return out


def test_the_loop(xkv):
    g = torch.Generator().manual_seed(3)
    cap = HIGH + 2 * N
    lens = [140, 95]
    K, V = bf16(G, BATCH, H_KV, cap, D, g=g), bf16(G, BATCH, H_KV, cap, D, g=g)
    plain = Plain(K, V, lens)
    K, V = K.cuda(), V.cuda()
    cfg = xkv.make_cache_config(G=G, batch=BATCH, H_kv=H_KV, H_q=H_KV * REP, d_h=D, cap=cap)
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, N), dtype=torch.uint8, device="cuda")
    weights = torch.zeros((G, BATCH, H_KV, cap), device="cuda")
    pos = torch.arange(cap, dtype=torch.int32, device="cuda").expand(G, BATCH, H_KV, cap).contiguous()
    length, next_pos = i32(lens), i32(lens)
    q, out = torch.zeros((G, BATCH, N, H_KV * REP, D), dtype=torch.bfloat16, device="cuda"), None
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
    mask, path, path_len = i32(torch.zeros((BATCH, N, 1))), i32(torch.zeros((BATCH, N))), i32([0] * BATCH)
    visible, flags = i32(torch.zeros((BATCH, N))), i32([0])
    src = torch.zeros((G, BATCH, H_KV, KEEP), dtype=torch.int32, device="cuda")

    def layers():                                # a model's own loop: every layer is a call of its own
        for l in range(G):
            xkv.xkv_tree_attend(cfg, l, l + 1, q, N, mask, None, K, V, length, ws, out, lse, flags)

    def take():                                  # after the verification, once the path is known; all on the device
        xkv.xkv_tree_commit(cfg, 0, G, K, V, length, path, path_len, N, pos, next_pos, flags)
        after = length + path_len
        xkv.xkv_cache_weigh(cfg, 0, G, q, N, lse, K, after, visible, length, 1.0, weights, flags)
        length.copy_(after)
        next_pos.add_(path_len)

    def evict():
        xkv.xkv_evict_select(cfg, 0, G, weights, pos, next_pos - RECENT, length, KEEP, src, flags)
        xkv.xkv_evict_compact(cfg, 0, G, K, V, src, KEEP, weights, pos, flags)
        length.clamp_(max=KEEP)

    graphs = {}
    for step in range(9):
        kd, vd, qd = bf16(G, BATCH, H_KV, N, D, g=g), bf16(G, BATCH, H_KV, N, D, g=g), bf16(G, BATCH, N, H_KV * REP, D, g=g)
        sees = torch.stack([R.random_tree(N, g) for _ in range(BATCH)])
        deepest = [int(sees[b].sum(1).argmax()) for b in range(BATCH)]
        paths = [sees[b, deepest[b]].nonzero().flatten().tolist() for b in range(BATCH)]
        if step % 4 == 3:
            paths[1] = []                        # nothing accepted
        new = next_pos.tolist()
        now = length.tolist()
        for b in range(BATCH):                   # the model writes its drafts' rows behind the committed ones
            K[:, b, :, now[b]:now[b] + N], V[:, b, :, now[b]:now[b] + N] = kd[:, b].cuda(), vd[:, b].cuda()
        q.copy_(qd)
        mask.copy_(R.words(sees))
        path.copy_(torch.tensor([p + [-1] * (N - len(p)) for p in paths]))
        path_len.copy_(torch.tensor([len(p) for p in paths]))
        # a token of the path saw the committed rows and the path up to itself, which lie in this order now
        visible.copy_(torch.tensor([[now[b] + paths[b].index(i) + 1 if i in paths[b] else 0 for i in range(N)] for b in range(BATCH)]))
        for name, part in (("layers", layers), ("take", take), ("evict", evict)):
            if name == "evict" and max(len(r) for r in plain.rows.values()) <= HIGH - N:
                continue
            if step < 3:
                part()
            else:                                # the same calls, captured once and replayed from then on
                if name not in graphs:
                    saved = [t.clone() for t in (K, V, weights, pos, length, next_pos, src)]
                    torch.cuda.synchronize()
                    graphs[name] = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graphs[name]):
                        part()
                    for t, was in zip((K, V, weights, pos, length, next_pos, src), saved):
                        assert torch.equal(t, was)               # a capture runs nothing
                graphs[name].replay()
            if name == "layers":
                want = plain.step(qd, kd, vd, sees, paths, new)
                torch.cuda.synchronize()
                # weights and outputs are rounded to bf16: half a step of the output and of sum p |v| (below 4 here)
                torch.testing.assert_close(out.double().cpu(), want, rtol=R.BF16, atol=4 * R.BF16)
            if name == "evict":
                torch.cuda.synchronize()
                src_now, n_now, new_now = src.cpu(), length.tolist(), next_pos.tolist()
                for (l, b, h), rows in plain.rows.items():
                    if len(rows) <= KEEP:
                        continue
                    order = sorted(range(len(rows)), key=lambda j: (rows[j][3] < new_now[b] - RECENT, -rows[j][2], j))
                    stays = set(order[:KEEP])
                    movers = iter([j for j in range(KEEP, len(rows)) if j in stays])
                    want = [j if j in stays else next(movers) for j in range(KEEP)]
                    assert src_now[l, b, h].tolist() == want
                    plain.rows[l, b, h] = [rows[j] for j in want]
        torch.cuda.synchronize()
        assert flags.item() == 0
        for (l, b, h), rows in plain.rows.items():
            n = length.tolist()[b]
            assert n == len(rows)
            assert torch.equal(K[l, b, h, :n].cpu().double(), torch.stack([r[0] for r in rows]))
            assert torch.equal(V[l, b, h, :n].cpu().double(), torch.stack([r[1] for r in rows]))
            assert pos[l, b, h, :n].tolist() == [r[3] for r in rows]
            # logits below 8, each off by less than 128 * 2^-23 of a sum of magnitudes below 128, as is the log-sum-exp
            torch.testing.assert_close(weights[l, b, h, :n].double().cpu(), torch.tensor([r[2] for r in rows], dtype=torch.float64), rtol=4e-4, atol=1e-7)


def test_two_graphs_with_their_own_workspaces_run_at_once(xkv):
    g = torch.Generator().manual_seed(4)
    cfg = xkv.make_cache_config(G=1, batch=1, H_kv=2, H_q=8, d_h=D, cap=3000)
    K, V = bf16(1, 1, 2, 3000, D, g=g).cuda(), bf16(1, 1, 2, 3000, D, g=g).cuda()
    qs = [bf16(1, 1, 6, 8, D, g=g).cuda() for _ in range(2)]
    outs, alone, graphs, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for q in qs:
        ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, 6), dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(q)
        xkv.xkv_tree_attend(cfg, 0, 1, q, 6, None, None, K, V, None, ws, out)
        alone.append(out.clone())
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            xkv.xkv_tree_attend(cfg, 0, 1, q, 6, None, None, K, V, None, ws, out)
        graphs.append((gr, ws))
        outs.append(out)
    for _ in range(20):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for (gr, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, alone))


def test_tensors_that_do_not_fit_are_refused(xkv):
    cfg = xkv.make_cache_config(G=1, batch=1, H_kv=2, H_q=8, d_h=64, cap=100)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    K, q = bf(1, 1, 2, 100, 64), bf(1, 1, 3, 8, 64)
    ws = torch.empty(xkv.xkv_tree_workspace_bytes(cfg, 3), dtype=torch.uint8, device="cuda")
    good = dict(q=q, n=3, mask=None, dl=None, K=K, V=K, ln=i32([9]), ws=ws, out=torch.zeros_like(q), lse=None)

    def run(**over):
        a = dict(good, **over)
        xkv.xkv_tree_attend(cfg, 0, 1, a["q"], a["n"], a["mask"], a["dl"], a["K"], a["V"], a["ln"], a["ws"], a["out"], a["lse"])
    run()
    for over in (dict(q=q.float()), dict(q=bf(1, 1, 8, 3, 64).transpose(2, 3)), dict(q=bf(1, 1, 2, 8, 64)), dict(K=K.cpu()), dict(V=bf(1, 1, 2, 99, 64)),
                 dict(ln=i32([9]).long()), dict(ln=i32([9, 9])), dict(ws=ws[:-1]), dict(out=q.half()), dict(mask=i32([[1, 2]])),
                 dict(lse=torch.zeros(5, device="cuda")), dict(n=2)):
        with pytest.raises(ValueError):
            run(**over)
    with pytest.raises(TypeError):
        run(K=K.data_ptr())
    with pytest.raises(xkv.XKVError):
        xkv.xkv_tree_attend(cfg, 0, 2, q, 3, None, None, K, K, i32([9]), ws, torch.zeros_like(q))
