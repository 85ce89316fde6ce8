"""Operators over an uncompressed KV cache that speculative decoding and a bounded cache need, as cases that can be timed and
compared.

A cache is K, V bf16 [G][batch][H_kv][cap][d_h]; sequence b holds `length[b]` rows in every head.

  attend    attention of n drafted tokens per sequence over the rows of the cache and, by a mask, over one another (a tree)
  commit    the accepted path of such a tree becomes the next rows of the cache, with their positions
  weigh     every row's accumulated attention weight, from the queries and the log-sum-exp of their attention
  select    which `keep` rows of every head stay: the recent ones, then those of the largest weight; as a map that fills holes
  compact   the rows that stay move into the holes, with their weights and positions

A case is a dict of plain values; `prepare` makes what a program has in hand, `run` is one pass: with `own` through the
library's calls, else in plain torch operations in 32 bits.  Sizes are those of the benchmark configurations' heads.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LLAMA = dict(H_kv=8, H_q=32, d_h=128)
QWEN = dict(H_kv=4, H_q=28, d_h=128)
TINY = dict(H_kv=2, H_q=8, d_h=64)


def _case(name, op, heads, **sizes):
    c = dict(op=op, **heads, **sizes)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the smallest model, a short prompt, five drafts: all latency
        _case("attend_tiny_300", "attend", TINY, G=2, batch=1, rows=300, n=5, tree=True, ragged=False),
        # one layer of an 8B model (a model calls layer after layer), a tree of 64 drafts: 256 query rows a head
        _case("attend_layer_8k_tree64", "attend", LLAMA, G=1, batch=1, rows=8192, n=64, tree=True, ragged=False),
        # eight sequences of different lengths with different numbers of drafts, seven query heads per KV head
        _case("attend_qwen_16k_batch8_tree33", "attend", QWEN, G=4, batch=8, rows=16411, n=33, tree=True, ragged=True),
        # a window at full context, a chain of 16 drafts: the whole cache is read once
        _case("attend_128k_chain16", "attend", LLAMA, G=4, batch=1, rows=131072, n=16, tree=False, ragged=False),
        # what one verification step of four sequences accepts: up to eight of 64 drafts
        _case("commit_batch4_8of64", "commit", LLAMA, G=4, batch=4, rows=1900, n=64, path=8),
        # a long accepted chain in a batch of eight
        _case("commit_qwen_batch8_200of256", "commit", QWEN, G=4, batch=8, rows=777, n=256, path=200),
        # the weights of one decode step over a cache of bounded size
        _case("weigh_8k_token", "weigh", LLAMA, G=4, batch=2, rows=8192, n=1, used=1, decay=1.0, ragged=True),
        # the last 32 tokens of a prompt weigh its rows
        _case("weigh_128k_window32", "weigh", LLAMA, G=4, batch=1, rows=131072, n=32, used=32, decay=1.0, ragged=False),
        # steady state: a cache of 4096 rows that has grown by 128
        _case("select_4224_to_4096", "select", LLAMA, G=4, batch=1, rows=4224, keep=4096, recent=256, ragged=False),
        # after a long prompt: a quarter stays, four sequences
        _case("select_64k_to_16k_batch4", "select", LLAMA, G=4, batch=4, rows=65536, keep=16384, recent=1024, ragged=True),
        _case("compact_4224_to_4096", "compact", LLAMA, G=4, batch=1, rows=4224, keep=4096),
        _case("compact_64k_to_16k", "compact", LLAMA, G=4, batch=1, rows=65531, keep=16384),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_ROWS = 4 * 8 * 131072          # rows of all heads of one cache


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "weigh", "weigh", "select", "select", "compact", "compact", "commit"])
    heads = rng.choice([LLAMA, QWEN, TINY])
    G = rng.choice([1, 2, 4])
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    n_rep = heads["H_q"] // heads["H_kv"]
    ragged = batch > 1 and rng.random() < 0.7
    if op == "commit":
        n = _logint(rng, 2, 256)
        return _case(None, op, heads, G=G, batch=batch, rows=_logint(rng, 16, 2048), n=n, path=_logint(rng, 1, min(n, 200)))
    most = min(131072, MOST_ROWS // (G * batch * heads["H_kv"]))
    if op in ("attend", "weigh"):
        n = _logint(rng, 1, 128)
        # no more multiplications than 64 query rows a head over the largest cache
        most = min(most, MOST_ROWS * 64 // (G * batch * heads["H_kv"] * n * n_rep))
        rows = _logint(rng, 16, most) if op == "attend" else max(n, _logint(rng, 64, most))
        if op == "attend":
            return _case(None, op, heads, G=G, batch=batch, rows=rows, n=n, tree=rng.random() < 0.7, ragged=ragged)
        return _case(None, op, heads, G=G, batch=batch, rows=rows, n=n, used=rng.choice([n, max(1, n // 3)]),
                     decay=rng.choice([1.0, 1.0, 0.97]), ragged=ragged)
    rows = _logint(rng, 256, most // (2 if op == "compact" else 1))
    keep = max(16, int(rows * rng.choice([0.97, 0.75, 0.5, 0.25, 0.1])))
    if op == "select":
        return _case(None, op, heads, G=G, batch=batch, rows=rows, keep=keep, recent=rng.choice([0, keep // 16, keep // 4]),
                     ragged=ragged)
    return _case(None, op, heads, G=G, batch=batch, rows=rows, keep=keep)


def _lens(c):
    """Rows of every sequence."""
    return [max(1, c["rows"] - (b * c["rows"] // (2 * c["batch"]) if c.get("ragged") else 0)) for b in range(c["batch"])]


def _drafts(c):
    """Drafted tokens of every sequence."""
    return [max(1, c["n"] - (b * c["n"] // (2 * c["batch"]) if c.get("ragged") else 0)) for b in range(c["batch"])]


def _paths(c):
    """Accepted tokens of every sequence."""
    return [max(1, c["path"] - b * c["path"] // (2 * c["batch"])) for b in range(c["batch"])]


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _randn(shape, g, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out:                # a layer at a time: the 32-bit numbers of a large cache are not all held at once
        part.copy_(torch.randn(shape[1:], generator=g, device="cuda"))
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _queries(c, K, g):
    """Queries of n tokens, bf16 [G][batch][n][H_q][d_h]: noise, and a share of one of the sequence's keys, so that some rows
    draw far more weight than others (logits of 9 against a standard deviation of 1)."""
    G, batch, n, H_kv, H_q, d_h = (c[k] for k in ("G", "batch", "n", "H_kv", "H_q", "d_h"))
    q = torch.randn((G, batch, n, H_kv, H_q // H_kv, d_h), generator=g, device="cuda")
    for b, rows in enumerate(_lens(c)):
        pick = torch.randint(0, rows, (n,), generator=g, device="cuda")
        q[:, b] += 0.8 * K[:, b][:, :, pick].float().transpose(1, 2).unsqueeze(3)
    return q.reshape(G, batch, n, H_q, d_h).to(torch.bfloat16)


def _tree(n, rng):
    """bool [n][n]: token i attends to itself and its ancestors."""
    sees = np.eye(n, dtype=bool)
    for i in range(1, n):
        parent = rng.integers(-1, i)
        if parent >= 0:
            sees[i] |= sees[parent]
    return sees


def _words(sees):
    """uint32 words of a bool [batch][n][n], bit j % 32 of word j / 32: what token i sees of draft j; int32 on the device."""
    batch, n, _ = sees.shape
    bits = np.zeros((batch, n, -(-n // 32) * 32), dtype=np.uint64)
    bits[:, :, :n] = sees
    words = (bits.reshape(batch, n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return torch.from_numpy(words.astype(np.uint32).view(np.int32)).cuda()


def _prepare_attend(c, g, seed):
    G, batch, n, H_kv, H_q, d_h = (c[k] for k in ("G", "batch", "n", "H_kv", "H_q", "d_h"))
    cap = c["rows"] + n + 17                     # a cache has room left behind its rows
    s = dict(K=_randn((G, batch, H_kv, cap, d_h), g), V=_randn((G, batch, H_kv, cap, d_h), g), cap=cap)
    s["q"] = _queries(c, s["K"], g)
    rng = np.random.default_rng(seed)
    sees = np.stack([_tree(n, rng) for _ in range(batch)]) if c["tree"] else np.tril(np.ones((batch, n, n), dtype=bool))
    s["sees"] = torch.from_numpy(sees).cuda()
    s["mask"] = _words(sees) if c["tree"] else None              # no mask: a chain
    s["length"], s["drafts"] = _int32(_lens(c)), _int32(_drafts(c))
    s["out"] = torch.zeros((G, batch, n, H_q, d_h), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((G, batch, n, H_q), dtype=torch.float32, device="cuda")
    return s


def _prepare_commit(c, g, seed):
    G, batch, H_kv, d_h = (c[k] for k in ("G", "batch", "H_kv", "d_h"))
    cap = c["rows"] + c["n"] + 9
    s = dict(K=_randn((G, batch, H_kv, cap, d_h), g), V=_randn((G, batch, H_kv, cap, d_h), g), cap=cap)
    s["pos"] = torch.arange(cap, dtype=torch.int32, device="cuda").expand(G, batch, H_kv, cap).contiguous()
    rng = np.random.default_rng(seed)
    path = np.full((batch, c["path"]), -1, dtype=np.int32)
    for b, m in enumerate(_paths(c)):
        path[b, :m] = np.sort(rng.choice(c["n"], m, replace=False))
    s["path"], s["path_len"] = torch.from_numpy(path).cuda(), _int32(_paths(c))
    s["length"] = _int32([max(0, c["rows"] - 3 * b) for b in range(batch)])
    s["first_pos"] = s["length"] + 100_000
    return s


def _prepare_weigh(c, g, seed):
    G, batch, n, H_kv, H_q, d_h = (c[k] for k in ("G", "batch", "n", "H_kv", "H_q", "d_h"))
    n_rep, cap = H_q // H_kv, c["rows"] + 5
    s = dict(K=_randn((G, batch, H_kv, cap, d_h), g), cap=cap)
    s["q"] = _queries(c, s["K"], g)
    s["lse"] = torch.zeros((G, batch, n, H_q), dtype=torch.float32, device="cuda")
    visible = []
    for b, rows in enumerate(_lens(c)):
        # the tokens are the last `used` rows of the sequence; what a verification step turned down weighs nothing
        m = min(c["used"], rows)
        vis = torch.tensor([rows - m + i + 1 if i < m else 0 for i in range(n)], device="cuda")
        visible.append(vis)
        at = torch.arange(rows, device="cuda") < vis[:, None]
        for l in range(G):
            q = s["q"][l, b].float().reshape(n, H_kv, n_rep, d_h).permute(1, 0, 2, 3).reshape(H_kv, n * n_rep, d_h)
            z = (q @ s["K"][l, b, :, :rows].float().transpose(1, 2) / math.sqrt(d_h)).reshape(H_kv, n, n_rep, rows)
            z.masked_fill_(~at[None, :, None], -math.inf)
            s["lse"][l, b] = torch.nan_to_num(torch.logsumexp(z, -1), neginf=0.0).permute(1, 0, 2).reshape(n, H_q)
    s["visible"] = torch.stack(visible).to(torch.int32)
    s["length"] = _int32(_lens(c))
    s["seen"] = _int32([max(0, r - c["used"]) for r in _lens(c)])
    s["weights"] = torch.rand((G, batch, H_kv, cap), generator=g, device="cuda") ** 4
    return s


def _prepare_select(c, g, seed):
    G, batch, H_kv = (c[k] for k in ("G", "batch", "H_kv"))
    cap, keep = c["rows"] + 3, c["keep"]
    # accumulated weights: heavy-tailed, and one row in ten drew none at all
    w = torch.exp(2.0 * torch.randn((G, batch, H_kv, cap), generator=g, device="cuda") - 4.0)
    w[torch.rand(w.shape, generator=g, device="cuda") < 0.1] = 0.0
    # an earlier eviction filled holes: the positions of the first rows are in no order, those behind ascend
    first = min(keep, c["rows"])
    old = torch.rand((G, batch, H_kv, first), generator=g, device="cuda").argsort(-1) * 3
    new = torch.arange(cap - first, device="cuda").expand(G, batch, H_kv, -1) + 3 * first
    s = dict(weights=w, pos=torch.cat([old, new], -1).to(torch.int32).contiguous(), cap=cap, keep=keep)
    s["length"] = _int32(_lens(c))
    s["since"] = _int32([(3 * first + r - first if r > first else 3 * r) - c["recent"] for r in _lens(c)])
    s["src"] = torch.zeros((G, batch, H_kv, keep), dtype=torch.int32, device="cuda")
    return s


def _moved(c):
    """Rows that move in every head."""
    return c["keep"] * (c["rows"] - c["keep"]) // c["rows"]


def _prepare_compact(c, g, seed):
    G, batch, H_kv, d_h, rows, keep = (c[k] for k in ("G", "batch", "H_kv", "d_h", "rows", "keep"))
    cap = rows + 3
    s = dict(K=_randn((G, batch, H_kv, cap, d_h), g), V=_randn((G, batch, H_kv, cap, d_h), g), cap=cap, keep=keep)
    s["weights"] = torch.rand((G, batch, H_kv, cap), generator=g, device="cuda")
    s["pos"] = torch.arange(cap, dtype=torch.int32, device="cuda").expand(G, batch, H_kv, cap).contiguous()
    m = _moved(c)
    src = torch.arange(keep, device="cuda").expand(G, batch, H_kv, keep).clone()
    holes = torch.rand(src.shape, generator=g, device="cuda").argsort(-1)[..., :m].sort(-1).values
    movers = keep + torch.rand((G, batch, H_kv, rows - keep), generator=g, device="cuda").argsort(-1)[..., :m].sort(-1).values
    s["src"] = src.scatter(3, holes, movers).to(torch.int32)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, g, seed)
    s["case"] = case
    if own:                                      # what a program keeps for its calls: the cache's sizes and a workspace
        from paper_2503_18893_b200 import xkv
        s["xkv"] = xkv
        s["cfg"] = xkv.make_cache_config(G=case["G"], batch=case["batch"], H_kv=case["H_kv"], H_q=case["H_q"],
                                         d_h=case["d_h"], cap=s["cap"])
        if case["op"] == "attend":
            s["workspace"] = torch.empty(xkv.xkv_tree_workspace_bytes(s["cfg"], case["n"]), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the library's calls


def _own_attend(s):
    c = s["case"]
    s["xkv"].xkv_tree_attend(s["cfg"], 0, c["G"], s["q"], c["n"], s["mask"], s["drafts"], s["K"], s["V"], s["length"],
                             s["workspace"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_commit(s):
    c = s["case"]
    s["xkv"].xkv_tree_commit(s["cfg"], 0, c["G"], s["K"], s["V"], s["length"], s["path"], s["path_len"], c["path"], s["pos"],
                             s["first_pos"])
    return {"K": s["K"], "V": s["V"], "pos": s["pos"]}


def _own_weigh(s):
    c = s["case"]
    s["xkv"].xkv_cache_weigh(s["cfg"], 0, c["G"], s["q"], c["n"], s["lse"], s["K"], s["length"], s["visible"], s["seen"],
                             c["decay"], s["weights"])
    return {"weights": s["weights"]}


def _own_select(s):
    c = s["case"]
    s["xkv"].xkv_evict_select(s["cfg"], 0, c["G"], s["weights"], s["pos"], s["since"], s["length"], s["keep"], s["src"])
    return {"src": s["src"]}


def _own_compact(s):
    c = s["case"]
    s["xkv"].xkv_evict_compact(s["cfg"], 0, c["G"], s["K"], s["V"], s["src"], s["keep"], s["weights"], s["pos"])
    return {"K": s["K"], "V": s["V"], "weights": s["weights"], "pos": s["pos"]}


# ---------------------------------------------------------------------------------------------------------------------
# plain forms


def _by_head(q, H_kv):
    """[G][batch][n][H_q][d] -> fp32 [G][batch][H_kv][n * n_rep][d]"""
    G, batch, n, H_q, d = q.shape
    return q.float().reshape(G, batch, n, H_kv, H_q // H_kv, d).permute(0, 1, 3, 2, 4, 5).reshape(G, batch, H_kv, -1, d)


def _plain_attend(s):
    c = s["case"]
    G, batch, n, H_kv, H_q, d_h = (c[k] for k in ("G", "batch", "n", "H_kv", "H_q", "d_h"))
    n_rep, cap = H_q // H_kv, s["cap"]
    row = torch.arange(cap, device="cuda")
    draft = row - s["length"][:, None]                                               # [batch][cap]
    seen = s["sees"].gather(2, draft.clamp(0, n - 1)[:, None].expand(batch, n, cap))
    live = (draft >= 0) & (draft < s["drafts"][:, None])
    at = (draft < 0)[:, None] | (live[:, None] & seen)                               # [batch][n][cap]
    z = _by_head(s["q"], H_kv) @ s["K"].float().transpose(3, 4) * (1.0 / math.sqrt(d_h))
    z = z.reshape(G, batch, H_kv, n, n_rep, cap).masked_fill_(~at[None, :, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = (z - top.clamp_min(-3e38)).exp_().reshape(G, batch, H_kv, n * n_rep, cap)
    total = p.sum(-1, keepdim=True)
    held = (row < (s["length"] + s["drafts"])[:, None])[None, :, None, :, None]      # rows behind the last hold anything
    o = p @ torch.where(held, s["V"], 0).float() / total.clamp_min(1e-38)
    lse = top[..., 0] + total.log().reshape(G, batch, H_kv, n, n_rep)
    out, out_lse = s["out"].clone(), s["lse"].clone()
    there = torch.arange(n, device="cuda") < s["drafts"][:, None]
    o = o.reshape(G, batch, H_kv, n, n_rep, d_h).permute(0, 1, 3, 2, 4, 5).reshape(G, batch, n, H_q, d_h).to(torch.bfloat16)
    out = torch.where(there[None, :, :, None, None], o, out)
    out_lse = torch.where(there[None, :, :, None], lse.permute(0, 1, 3, 2, 4).reshape(G, batch, n, H_q), out_lse)
    return {"out": out, "lse": out_lse}


def _plain_commit(s):
    c = s["case"]
    G, batch, H_kv, d_h = (c[k] for k in ("G", "batch", "H_kv", "d_h"))
    j = torch.arange(c["path"], device="cuda")
    to = (s["length"][:, None] + j).long()
    fro = torch.where(j < s["path_len"][:, None], s["length"][:, None] + s["path"], to).long()  # behind the path: itself
    at = fro[None, :, None, :, None].expand(G, batch, H_kv, c["path"], d_h)
    onto = to[None, :, None, :, None].expand(G, batch, H_kv, c["path"], d_h)
    s["K"].scatter_(3, onto, s["K"].gather(3, at))
    s["V"].scatter_(3, onto, s["V"].gather(3, at))
    one = to[None, :, None].expand(G, batch, H_kv, c["path"])
    new = (s["first_pos"][:, None] + j).to(torch.int32)[None, :, None].expand(G, batch, H_kv, c["path"])
    s["pos"].scatter_(3, one, torch.where((j < s["path_len"][:, None])[None, :, None], new, s["pos"].gather(3, one)))
    return {"K": s["K"], "V": s["V"], "pos": s["pos"]}


def _plain_weigh(s):
    c = s["case"]
    G, batch, n, H_kv, H_q, d_h = (c[k] for k in ("G", "batch", "n", "H_kv", "H_q", "d_h"))
    n_rep, cap = H_q // H_kv, s["cap"]
    row = torch.arange(cap, device="cuda")
    z = _by_head(s["q"], H_kv) @ s["K"].float().transpose(3, 4) * (1.0 / math.sqrt(d_h))
    z = z.reshape(G, batch, H_kv, n, n_rep, cap)
    z -= s["lse"].reshape(G, batch, n, H_kv, n_rep).permute(0, 1, 3, 2, 4).unsqueeze(-1)
    at = row < torch.minimum(s["visible"], s["length"][:, None])[..., None]          # [batch][n][cap]
    p = z.exp_().masked_fill_(~at[None, :, None, :, None], 0.0).sum((3, 4))
    old = torch.where((row < s["seen"][:, None])[None, :, None], s["weights"] * c["decay"], 0.0)
    s["weights"] = torch.where((row < s["length"][:, None])[None, :, None], old + p, s["weights"])
    return {"weights": s["weights"]}


def _plain_select(s):
    keep = s["keep"]
    row = torch.arange(s["cap"], device="cuda")
    held = (row < s["length"][:, None])[None, :, None].expand(s["weights"].shape)
    recent = held & (s["pos"] >= s["since"][None, :, None, None])
    w = torch.nan_to_num(s["weights"], nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    order = w.sort(dim=-1, descending=True, stable=True).indices                         # by weight, ties by row,
    rank = recent.int() + held.int()                                                 # the recent rows before the others
    order = order.gather(-1, rank.gather(-1, order).sort(dim=-1, descending=True, stable=True).indices)
    stays = torch.zeros_like(held).scatter(-1, order[..., :keep], True) & held
    # the i-th hole among the first `keep` rows takes the i-th row that stays behind them
    hole = (held & ~stays)[..., :keep]
    nth = hole.cumsum(-1) - 1
    behind = stays[..., keep:]
    count = behind.cumsum(-1)
    movers = torch.full_like(order[..., :keep + 1], -1)
    movers = movers.scatter(-1, torch.where(behind, count - 1, keep), (row[keep:]).expand(behind.shape))
    src = torch.where(hole, movers.gather(-1, nth.clamp_min(0)), row[:keep])
    return {"src": torch.where(held[..., :keep], src, -1).to(torch.int32)}


def _plain_compact(s):
    keep, d_h = s["keep"], s["case"]["d_h"]
    at = torch.where(s["src"] < 0, torch.arange(keep, device="cuda"), s["src"]).long()
    rows = at.unsqueeze(-1).expand(*at.shape, d_h)
    s["K"][:, :, :, :keep] = s["K"].gather(3, rows)
    s["V"][:, :, :, :keep] = s["V"].gather(3, rows)
    s["weights"][..., :keep] = s["weights"].gather(3, at)
    s["pos"][..., :keep] = s["pos"].gather(3, at)
    return {"K": s["K"], "V": s["V"], "weights": s["weights"], "pos": s["pos"]}


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    heads, d_h = c["G"] * c["H_kv"], c["d_h"]
    if c["op"] == "attend":
        rows, pairs, tokens = 0, 0, 0
        for r, n in zip(_lens(c), _drafts(c)):
            rows += heads * (r + n)
            pairs += c["G"] * c["H_q"] * n * (r + n)
            tokens += c["G"] * c["H_q"] * n
        return {"bytes": rows * 4 * d_h + tokens * (4 * d_h + 4), "flops": pairs * 4 * d_h}
    if c["op"] == "commit":
        return {"bytes": sum(heads * m * (8 * d_h + 4) + 4 * m for m in _paths(c)), "flops": 0}
    if c["op"] == "weigh":
        rows = heads * sum(_lens(c))
        used = sum(min(c["used"], r) * r for r in _lens(c))
        return {"bytes": rows * (2 * d_h + 8) + sum(min(c["used"], r) for r in _lens(c)) * c["G"] * c["H_q"] * (2 * d_h + 4),
                "flops": c["G"] * c["H_q"] * used * 2 * d_h}
    if c["op"] == "select":
        return {"bytes": heads * (8 * sum(_lens(c)) + 4 * c["keep"] * c["batch"]), "flops": 0}
    return {"bytes": heads * c["batch"] * (_moved(c) * (8 * d_h + 16) + 4 * c["keep"]), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits, head by head


def _exact_attend(s):
    c = s["case"]
    G, batch, H_kv, H_q = (c[k] for k in ("G", "batch", "H_kv", "H_q"))
    n_rep = H_q // H_kv
    out, lse = s["out"].double(), s["lse"].double()
    for b, (rows, n) in enumerate(zip(_lens(c), _drafts(c))):
        at = torch.cat([torch.ones((n, rows), dtype=torch.bool, device="cuda"), s["sees"][b, :n, :n]], 1)
        hidden = ~at.repeat_interleave(n_rep, 0)
        for l in range(G):
            for h in range(H_kv):
                heads = slice(h * n_rep, (h + 1) * n_rep)
                q = s["q"][l, b, :n, heads].double().reshape(n * n_rep, -1)
                z = q @ s["K"][l, b, h, :rows + n].double().T / math.sqrt(c["d_h"])
                z[hidden] = -math.inf
                total = torch.logsumexp(z, 1)
                o = torch.exp(z - total[:, None]) @ s["V"][l, b, h, :rows + n].double()
                out[l, b, :n, heads] = o.reshape(n, n_rep, -1)
                lse[l, b, :n, heads] = total.reshape(n, n_rep)
    return {"out": out, "lse": lse}


def _exact_commit(s):
    K, V = s["K"].clone(), s["V"].clone()
    for b, m in enumerate(_paths(s["case"])):
        first = int(s["length"][b])
        for j, i in enumerate(s["path"][b, :m].tolist()):
            K[:, b, :, first + j], V[:, b, :, first + j] = s["K"][:, b, :, first + i], s["V"][:, b, :, first + i]
    return {"K": K, "V": V, "pos": None}


def _exact_weigh(s):
    c = s["case"]
    G, batch, H_kv, H_q = (c[k] for k in ("G", "batch", "H_kv", "H_q"))
    n_rep = H_q // H_kv
    w = s["weights"].double()
    for b, rows in enumerate(_lens(c)):
        w[:, b, :, int(s["seen"][b]):rows] = 0.0
        w[:, b, :, :int(s["seen"][b])] *= c["decay"]
        for i, sees in enumerate(s["visible"][b].tolist()):
            if not sees:
                continue
            for l in range(G):
                q = s["q"][l, b, i].double().reshape(H_kv, n_rep, -1)
                z = torch.einsum("hrd,hjd->hrj", q, s["K"][l, b, :, :sees].double()) / math.sqrt(c["d_h"])
                w[l, b, :, :sees] += torch.exp(z - s["lse"][l, b, i].double().reshape(H_kv, n_rep, 1)).sum(1)
    return {"weights": w}


def _exact_compact(s):
    K, V, w = s["K"].clone(), s["V"].clone(), s["weights"].double()
    m = s["src"] != torch.arange(s["keep"], device="cuda")
    l, b, h, j = m.nonzero(as_tuple=True)
    i = s["src"][m].long()
    K[l, b, h, j], V[l, b, h, j], w[l, b, h, j] = s["K"][l, b, h, i], s["V"][l, b, h, i], s["weights"][l, b, h, i].double()
    return {"K": K, "V": V, "weights": w, "pos": None}


def exact(case, seed):
    if case["op"] == "select":
        return None                              # whole numbers: the plain form's own
    s = globals()["_prepare_" + case["op"]](case, torch.Generator(device="cuda").manual_seed(seed), seed)
    s["case"] = case
    return globals()["_exact_" + case["op"]](s)
