"""Operators over a paged KV cache of 8-bit codes, from the rotation of a step's queries and keys to the attention over the cache,
as cases that can be timed and compared.

The cache is K, V e4m3 [G][n_pages][H_kv][page][d_h] with a scale, a power of two, for each page and head: fp32 [G][n_pages][H_kv].
Row j of sequence b lies in row j % page of page table[b][j // page].  A step's new tokens lie behind one another, sequence by
sequence: token t of all n_tok, with `first` int32 [batch + 1] the places where sequences begin.

  rope     queries and keys rotated by their positions: interleaved or half layout, part of the head, scaled for long contexts
  assign   lengths -> pages taken from and given back to a ring of free ones, table, positions and slots of the new tokens
  append   new keys and values into their slots as codes; a page's scale grows with what it holds
  read     rows of a sequence back from codes, as an uncompressed cache
  attend   attention of each sequence's last tokens over its rows of the cache, each up to its own row

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
LOWEST = -60                    # exponent of the smallest scale


def _case(name, op, heads, **sizes):
    c = dict(op=op, **heads, **sizes)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one decode step of 64 sequences in one layer, frequencies scaled in three bands: all latency
        _case("rope_token_batch64", "rope", LLAMA, n_tok=64, rot=128, layout="half", scaling="llama3", dtype="bf16", direction="forward"),
        # a prompt in one layer, neighbouring pairs of the first half of the head, NTK-by-parts; its gradient in the other direction
        _case("rope_gradient_prompt_8k", "rope", QWEN, n_tok=8189, rot=64, layout="interleaved", scaling="yarn", dtype="fp32",
              direction="adjoint"),
        # a verification step of 48 sequences: eight drafts each get places, and give them back when they are turned down
        _case("assign_drafts_batch48", "assign", LLAMA, batch=48, rows=4000, new=8, page=16, ragged=False),
        # 300 requests of which some begin with a prompt's chunk, and all end
        _case("assign_chunks_batch300", "assign", LLAMA, batch=300, rows=700, new=128, page=64, ragged=True),
        # a decode step of 32 sequences in a window of four layers, into caches of a few pages; the cache is then read back
        _case("append_token_batch32", "append", LLAMA, G=4, batch=32, rows=29, new=1, page=16, ragged=True),
        # a prompt's chunk of odd length behind another, in long pages
        _case("append_chunk_4k", "append", QWEN, G=4, batch=1, rows=517, new=4099, page=128, ragged=False),
        # a sequence handed from the 8-bit cache to the factorisation, which takes 16-bit rows
        _case("read_32k", "read", LLAMA, G=4, batch=1, rows=32768, page=64),
        # short sequences of different lengths in the smallest pages
        _case("read_batch5_333", "read", TINY, G=2, batch=5, rows=333, page=16),
        # the smallest model, a short prompt, one token: all latency
        _case("attend_tiny_300", "attend", TINY, G=2, batch=1, rows=300, new=1, page=16, ragged=False),
        # a decode step of eight sequences of different lengths in a window of four layers
        _case("attend_token_8k_batch8", "attend", LLAMA, G=4, batch=8, rows=8191, new=1, page=16, ragged=True),
        # a decode step at full context
        _case("attend_token_128k", "attend", LLAMA, G=4, batch=1, rows=131072, new=1, page=64, ragged=False),
        # a prompt's chunk of 512 tokens behind 12k rows, seven query heads per KV head, one layer
        _case("attend_chunk_12k", "attend", QWEN, G=1, batch=2, rows=12301, new=512, page=32, ragged=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_ROWS = 4 * 8 * 131072          # rows of all heads of one cache
MOST_PAIRS = 28 * 512 * 20000       # products of a query row with a key


def draw(rng):
    op = rng.choice(["rope", "assign", "append", "read", "attend", "attend", "attend"])
    heads = rng.choice([LLAMA, QWEN, TINY])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope":
        d_h = heads["d_h"]
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        return _case(None, op, heads, n_tok=_logint(rng, 1, 8192), rot=rng.choice([d_h, d_h, d_h // 2, d_h // 4]),
                     layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "llama3", "yarn"]), dtype=dtype,
                     direction=rng.choice(["forward", "forward", "inverse", "adjoint"]))
    if op == "assign":
        batch = _logint(rng, 1, 300)
        return _case(None, op, heads, batch=batch, rows=_logint(rng, 16, 4000), new=_logint(rng, 1, 128), page=page, ragged=rng.random() < 0.6)
    G, batch = rng.choice([1, 2, 4]), rng.choice([1, 1, 2, 3, 5, 8])
    ragged = batch > 1 and rng.random() < 0.7
    if op == "append":
        new = _logint(rng, 1, 4096 // batch)
        return _case(None, op, heads, G=G, batch=batch, rows=_logint(rng, 1, 600), new=new, page=page, ragged=ragged)
    if op == "read":
        return _case(None, op, heads, G=G, batch=batch, rows=_logint(rng, 16, 131072 // (G * batch)), page=page)
    new = rng.choice([1, 1, 1, _logint(rng, 2, 16), _logint(rng, 16, 512)])
    most = min(131072, MOST_ROWS // (G * batch * heads["H_kv"]), MOST_PAIRS // (G * batch * heads["H_q"] * new))
    return _case(None, op, heads, G=G, batch=batch, rows=_logint(rng, 16, max(17, most)), new=new, page=page, ragged=ragged)


def _lens(c):
    """Rows of every sequence before the new ones."""
    return [max(1, c["rows"] - (b * c["rows"] // (2 * c["batch"]) if c.get("ragged", True) else 0)) for b in range(c["batch"])]


def _news(c):
    """New tokens of every sequence."""
    return [max(1, c["new"] - (b * c["new"] // (2 * c["batch"]) if c.get("ragged") else 0)) for b in range(c["batch"])]


# ---------------------------------------------------------------------------------------------------------------------
# inputs

TYPES = dict(bf16=torch.bfloat16, fp16=torch.float16, fp32=torch.float32)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages_of(rows, page):
    return -(-rows // page)


def _table(lens, page, spare, rng):
    """Pages in no order: int32 [batch][most], -1 behind a sequence's last; how many pages there are."""
    counts = [_pages_of(n, page) for n in lens]
    n_pages = sum(counts) + spare
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max(counts)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, n_pages


def _exponent(top):
    """The smallest e >= LOWEST with top <= 448 * 2^e, element by element (top finite, fp32): frexp gives top = m 2^x, 0.5 <= m < 1."""
    m, x = torch.frexp(top)
    e = x.to(torch.int32) - 9 + (m > 0.875).to(torch.int32)
    return torch.where(top > 0, e.clamp_min(LOWEST), LOWEST)


def _two(e):
    """2^e in fp32 for -126 <= e <= 127 (int32)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x, e):
    """x 2^-e as e4m3 (x fp32, e int32 of a shape that broadcasts)."""
    return (x * _two(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _at(codes, *index):
    """fp32 values of the codes at an index."""
    return codes.view(torch.uint8)[index].view(torch.float8_e4m3fn).float()


def _cache(c, g, lens, spare, rng):
    """Codes and scales of a cache whose sequences hold `lens` rows.  Keys: some channels are several times the others; values: pages
    differ in magnitude.  What no sequence holds is what memory may hold: any finite code and scale."""
    G, H_kv, d_h, page = (c[k] for k in ("G", "H_kv", "d_h", "page"))
    table, n_pages = _table(lens, page, spare, rng)
    s = dict(table=torch.from_numpy(table).cuda(), n_pages=n_pages, page=page)
    loud = 1.0 + 4.0 * (torch.rand((H_kv, 1, d_h), generator=g, device="cuda") < 0.04)
    for name in ("K", "V"):
        codes = torch.empty((G, n_pages, H_kv, page, d_h), dtype=torch.float8_e4m3fn, device="cuda")
        scale = torch.empty((G, n_pages, H_kv), device="cuda")
        for l in range(G):
            x = torch.randn((n_pages, H_kv, page, d_h), generator=g, device="cuda")
            x *= loud if name == "K" else torch.exp(0.5 * torch.randn((n_pages, H_kv, 1, 1), generator=g, device="cuda"))
            e = _exponent(x.abs().amax((2, 3)))
            codes[l] = _encode(x, e[..., None, None])
            scale[l] = _two(e)
        s[name], s[name.lower() + "_scale"] = codes, scale
    return s


def _prepare_rope(c, g, seed):
    n, d_h, H = c["n_tok"], c["d_h"], c["H_q"] + 2 * c["H_kv"]
    # what a projection has made: queries, keys and values of a token side by side
    qkv = torch.randn((n, H, d_h), generator=g, device="cuda").to(TYPES[c["dtype"]])
    s = dict(qkv=qkv, q=qkv[:, :c["H_q"]], k=qkv[:, c["H_q"]:c["H_q"] + c["H_kv"]])
    first = int(torch.randint(0, 1 << 17, (1,), generator=g, device="cuda")) if n > 64 else 0
    s["pos"] = (first + torch.arange(n, device="cuda") if n > 64 else torch.randint(0, 1 << 17, (n,), generator=g, device="cuda")).to(torch.int32)
    s["q_out"], s["k_out"] = torch.empty(s["q"].shape, dtype=qkv.dtype, device="cuda"), torch.empty(s["k"].shape, dtype=qkv.dtype, device="cuda")
    return s


def _prepare_assign(c, g, seed):
    rng = np.random.default_rng(seed)
    held = _lens(c)
    new = [int(x) for x in (rng.integers(1, c["new"] + 1, c["batch"]) if c["ragged"] else np.full(c["batch"], c["new"]))]
    if c["ragged"]:                              # a third has not begun yet
        held = [0 if rng.random() < 0.33 else h for h in held]
    want = [h + n for h, n in zip(held, new)]
    page = c["page"]
    most = _pages_of(c["rows"] + c["new"], page) + 1
    n_pages = c["batch"] * most + 5              # more than can be wanted
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((c["batch"], most), -1, dtype=np.int32)
    at = 0
    for b, h in enumerate(held):
        n = _pages_of(h, page)
        table[b, :n] = ids[at:at + n]
        at += n
    ring = np.full(n_pages, -1, dtype=np.int32)  # the free pages lie behind a head that has gone round
    head = int(rng.integers(0, n_pages))
    ring[(head + np.arange(n_pages - at)) % n_pages] = ids[at:]
    s = dict(held=_int32(held), want=_int32(want), table=torch.from_numpy(table).cuda(), ring=torch.from_numpy(ring).cuda(),
             state=_int32([head, n_pages - at]), n_pages=n_pages, page=page, n_tok=c["batch"] * c["new"])
    for key, size in (("first", c["batch"] + 1), ("length", c["batch"]), ("pos", s["n_tok"]), ("slot", s["n_tok"])):
        s[key] = torch.zeros(size, dtype=torch.int32, device="cuda")
    s["length2"] = torch.zeros_like(s["length"])
    return s


def _prepare_append(c, g, seed):
    rng = np.random.default_rng(seed)
    lens, news, G = _lens(c), _news(c), c["G"]
    s = _cache(c, g, [a + n for a, n in zip(lens, news)], 1, rng)
    n_tok, page = sum(news), c["page"]
    table = s["table"].cpu().numpy()
    s["slot"] = _int32([int(table[b, j // page]) * page + j % page for b, (a, n) in enumerate(zip(lens, news)) for j in range(a, a + n)])
    shape = (G, n_tok, c["H_kv"], c["d_h"])
    # some tokens are louder than what their pages hold so far: those pages' scales grow
    loud = torch.exp(1.5 * torch.randn((1, n_tok, 1, 1), generator=g, device="cuda"))
    s["k"] = (loud * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
    s["v"] = (loud * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
    s["length"] = _int32([a + n for a, n in zip(lens, news)])
    s["cap"] = max(a + n for a, n in zip(lens, news))
    for name in ("K_out", "V_out"):
        s[name] = torch.zeros((G, c["batch"], c["H_kv"], s["cap"], c["d_h"]), dtype=torch.bfloat16, device="cuda")
    return s


def _prepare_read(c, g, seed):
    lens = _lens(c)
    s = _cache(c, g, lens, 2, np.random.default_rng(seed))
    s["length"], s["cap"] = _int32(lens), max(lens) + 3
    for name in ("K_out", "V_out"):
        s[name] = torch.zeros((c["G"], c["batch"], c["H_kv"], s["cap"], c["d_h"]), dtype=torch.bfloat16, device="cuda")
    return s


def _rows_of(codes, scale, table_row, rows, page):
    """fp32 [H_kv][rows][d_h]: what one layer's codes of one sequence stand for."""
    pages = table_row[:_pages_of(rows, page)].long()
    x = _at(codes, pages) * scale[pages][..., None, None]
    n, H, _, d = x.shape
    return x.transpose(0, 1).reshape(H, n * page, d)[:, :rows]


def _prepare_attend(c, g, seed):
    G, batch, H_kv, H_q, d_h, page = (c[k] for k in ("G", "batch", "H_kv", "H_q", "d_h", "page"))
    rng = np.random.default_rng(seed)
    news = _news(c)
    lens = [a + n for a, n in zip(_lens(c), news)]       # with the new rows
    s = _cache(c, g, lens, 3, rng)
    n_tok = sum(news)
    q = torch.randn((G, n_tok, H_kv, H_q // H_kv, d_h), generator=g, device="cuda")
    at = 0
    for b, (rows, n) in enumerate(zip(lens, news)):      # a share of one of the rows' keys: some rows draw far more weight than others
        row = torch.randint(0, rows - n + 1, (n,), generator=g, device="cuda")
        pages, off = s["table"][b].long()[row // page], row % page
        for l in range(G):
            key = _at(s["K"][l], pages, slice(None), off) * s["k_scale"][l][pages][..., None]
            q[l, at:at + n] += 0.5 * key.unsqueeze(2)
        at += n
    s["q"] = q.reshape(G, n_tok, H_q, d_h).to(torch.bfloat16)
    s["first"] = _int32(np.concatenate([[0], np.cumsum(news)]).tolist())
    s["length"], s["lens"], s["news"] = _int32(lens), lens, news
    s["out"] = torch.zeros((G, n_tok, H_q, d_h), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((G, n_tok, H_q), dtype=torch.float32, device="cuda")
    return s


# Settings of the rotation as a model's configuration has them.
ROPE = dict(base=500000.0, factor=8.0, original=8192, low=1.0, high=4.0, beta_fast=32.0, beta_slow=1.0)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, g, seed)
    s["case"] = case
    if own:                                      # what a program keeps for its calls: sizes, frequencies and a workspace
        from paper_2503_18893_b200 import xkv
        s["xkv"] = xkv
        if case["op"] == "rope":
            s["rope"] = xkv.make_rope(d_h=case["d_h"], rot=case["rot"], layout=case["layout"], scaling=case["scaling"], **ROPE)
        else:
            batch, most = s["table"].shape
            s["cfg"] = xkv.make_cache8_config(G=case.get("G", 1), batch=batch, H_kv=case["H_kv"], H_q=case["H_q"], d_h=case["d_h"],
                                              page=case["page"], n_pages=s["n_pages"], max_pages=most)
        if case["op"] == "attend":
            s["workspace"] = torch.empty(xkv.xkv_cache8_workspace_bytes(s["cfg"], max(s["news"])), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the library's calls


def _own_rope(s):
    s["xkv"].xkv_rope(s["rope"], s["q"], s["pos"], s["q_out"], s["k"], s["k_out"], direction=s["case"]["direction"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_assign(s):
    x = s["xkv"]
    x.xkv_page_assign(s["cfg"], s["held"], s["want"], s["table"], s["ring"], s["state"], s["first"], s["length"], s["pos"], s["slot"])
    x.xkv_page_assign(s["cfg"], s["length"], s["held"], s["table"], s["ring"], s["state"], None, s["length2"])
    return {k: s[k] for k in ("table", "ring", "state", "first", "length", "pos", "slot", "length2")}


def _own_append(s):
    G = s["case"]["G"]
    s["xkv"].xkv_cache8_append(s["cfg"], 0, G, s["k"], s["v"], s["slot"], s["K"], s["V"], s["k_scale"], s["v_scale"])
    return _own_read(s)


def _own_read(s):
    s["xkv"].xkv_cache8_read(s["cfg"], 0, s["case"]["G"], s["table"], s["length"], s["K"], s["V"], s["k_scale"], s["v_scale"],
                             s["K_out"], s["V_out"])
    return {"K": s["K_out"], "V": s["V_out"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _own_attend(s):
    s["xkv"].xkv_cache8_attend(s["cfg"], 0, s["case"]["G"], s["q"], s["first"], max(s["news"]), s["table"], s["length"], s["K"], s["V"],
                               s["k_scale"], s["v_scale"], s["workspace"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------------------------------------------------------------
# plain forms


def _frequencies(c):
    """Radians per position of every pair, and the factor on cosine and sine: float64 on the host."""
    r, n = ROPE, c["rot"]
    base = r["base"]
    if c["scaling"] == "ntk":
        base *= r["factor"] ** (n / max(n - 2, 1))
    f = base ** (-np.arange(0, n, 2, dtype=np.float64) / n)
    if c["scaling"] == "linear":
        return f / r["factor"], 1.0
    if c["scaling"] == "llama3":
        turns = r["original"] * f / (2 * math.pi)                    # in the original context
        share = np.clip((turns - r["low"]) / (r["high"] - r["low"]), 0.0, 1.0)
        return (1 - share) * f / r["factor"] + share * f, 1.0
    if c["scaling"] == "yarn":
        def pair(beta):
            return n * math.log(r["original"] / (beta * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(r["beta_fast"])), 0), min(math.ceil(pair(r["beta_slow"])), n - 1)
        keep = 1 - np.clip((np.arange(n // 2) - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return (1 - keep) * f / r["factor"] + keep * f, 0.1 * math.log(r["factor"]) + 1.0
    return f, 1.0


def _plain_rope(s):
    c = s["case"]
    f, m = _frequencies(c)
    angle = s["pos"].double()[:, None] * torch.from_numpy(f).cuda()  # far positions: 32 bits have too few for the angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["direction"] == "inverse":
        cos, sin = cos / m, -sin / m
    else:
        cos, sin = cos * m, (sin if c["direction"] == "forward" else -sin) * m
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        y = x.clone()
        half = c["rot"] // 2
        one, two = (slice(0, half), slice(half, c["rot"])) if c["layout"] == "half" else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
        y[..., one] = x[..., one] * cos - x[..., two] * sin
        y[..., two] = x[..., two] * cos + x[..., one] * sin
        out[name] = y.to(s[name].dtype)
    return out


def _plain_give_and_take(s, held, want, length, first=None):
    """The pages' way for lengths that grow and shrink, in whole numbers."""
    page, table, ring, state, n_pages = s["page"], s["table"], s["ring"], s["state"], s["n_pages"]
    have, need = (held + page - 1) // page, (want + page - 1) // page
    take, give = (need - have).clamp_min(0), (have - need).clamp_min(0)
    upto, back = take.cumsum(0), give.cumsum(0)
    head, count = state[0].clone(), state[1].clone()
    ok = (take == 0) | (upto <= count)
    take = torch.where(ok, take, 0)
    col = torch.arange(table.shape[1], device="cuda")
    entry = (col >= have[:, None]) & (col < (have + take)[:, None])
    got = ring[((head + (upto - take)[:, None] + col - have[:, None]) % n_pages).long()]
    gone = (col >= need[:, None]) & (col < have[:, None])
    to = ((head + count + (back - give)[:, None] + col - need[:, None]) % n_pages).long()
    ring[to[gone]] = table[gone]
    table.copy_(torch.where(entry, got, torch.where(gone, -1, table)))
    length.copy_(torch.where(ok, want, held))
    taken = torch.where(ok, upto, 0).amax()
    state.copy_(torch.stack([(head + taken) % n_pages, count - taken + back[-1]]))
    if first is None:
        return
    new = (want - held).clamp_min(0)
    first[0] = 0
    first[1:] = new.cumsum(0)
    t = torch.arange(s["n_tok"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(first[1:].contiguous(), t, right=True).clamp_max(len(held) - 1)
    there = t < first[-1]
    pos = held[b] + t - first[b]
    slot = table[b, (pos // page).clamp(0, table.shape[1] - 1).long()] * page + pos % page
    s["pos"].copy_(torch.where(there, pos, 0))
    s["slot"].copy_(torch.where(there & ok[b], slot, -1))


def _plain_assign(s):
    _plain_give_and_take(s, s["held"], s["want"], s["length"], s["first"])
    _plain_give_and_take(s, s["length"], s["held"], s["length2"])
    return {k: s[k] for k in ("table", "ring", "state", "first", "length", "pos", "slot", "length2")}


def _plain_append(s):
    page, slot = s["page"], s["slot"].long()
    at, off = slot // page, slot % page
    pages, place = torch.unique(at, return_inverse=True)
    begin = torch.full((len(pages),), page, device="cuda").scatter_reduce(0, place, off, "amin")      # rows that a page holds already
    fresh = torch.zeros((len(pages), page), dtype=torch.bool, device="cuda")
    fresh[place, off] = True
    for name, x in (("K", s["k"]), ("V", s["v"])):
        codes, scale = s[name], s[name.lower() + "_scale"]
        for l in range(s["case"]["G"]):
            rows = torch.zeros((len(pages), page, *x.shape[2:]), device="cuda")
            rows[place, off] = x[l].float()
            rows = rows.transpose(1, 2)                                                               # [pages][H_kv][page][d_h]
            e = _exponent(rows.abs().amax((2, 3)))
            m, before = torch.frexp(scale[l][pages])
            before = before.to(torch.int32) - 1
            e = torch.where((begin > 0)[:, None], torch.maximum(e, before), e)
            old = _at(codes[l], pages)
            held = torch.arange(page, device="cuda") < begin[:, None]
            # a held row's code moves down by the steps that the scale has moved up
            old = torch.where(held[:, None, :, None], old * _two((before - e).clamp_min(-126))[..., None, None], old)
            new = (rows * _two(-e)[..., None, None]).clamp(-448.0, 448.0)
            codes[l].view(torch.uint8)[pages] = torch.where(fresh[:, None, :, None], new, old).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[l][pages] = _two(e)
    return _plain_read(s)


def _plain_read(s):
    c = s["case"]
    for name, out in (("K", s["K_out"]), ("V", s["V_out"])):
        row = torch.arange(s["cap"], device="cuda")
        there = row < s["length"][:, None]
        pages = s["table"].long().gather(1, (row // s["page"]).clamp_max(s["table"].shape[1] - 1).expand(c["batch"], -1)).clamp_min(0)
        off = (row % s["page"]).expand(c["batch"], -1)
        for l in range(c["G"]):
            x = _at(s[name][l], pages, slice(None), off)                                                # [batch][cap][H_kv][d_h]
            x *= s[name.lower() + "_scale"][l][pages].unsqueeze(-1)
            out[l] = torch.where(there[:, None, :, None], x.transpose(1, 2).to(torch.bfloat16), out[l])
    return {"K": s["K_out"], "V": s["V_out"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attend(s):
    c = s["case"]
    G, H_kv, H_q, d_h, page = (c[k] for k in ("G", "H_kv", "H_q", "d_h", "page"))
    n_rep, at = H_q // H_kv, 0
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    for b, (rows, n) in enumerate(zip(s["lens"], s["news"])):
        sees = torch.arange(rows, device="cuda") < torch.arange(rows - n + 1, rows + 1, device="cuda")[:, None]
        for l in range(G):
            K = _rows_of(s["K"][l], s["k_scale"][l], s["table"][b], rows, page)
            q = s["q"][l, at:at + n].float().reshape(n, H_kv, n_rep, d_h).transpose(0, 1).reshape(H_kv, n * n_rep, d_h)
            z = (q @ K.transpose(1, 2) * (1.0 / math.sqrt(d_h))).reshape(H_kv, n, n_rep, rows)
            z.masked_fill_(~sees[None, :, None], -math.inf)
            top = z.amax(-1, keepdim=True)
            p = (z - top).exp_().reshape(H_kv, n * n_rep, rows)
            total = p.sum(-1, keepdim=True)
            V = _rows_of(s["V"][l], s["v_scale"][l], s["table"][b], rows, page)
            o = (p @ V / total).reshape(H_kv, n, n_rep, d_h).transpose(0, 1)
            out[l, at:at + n] = o.reshape(n, H_q, d_h).to(torch.bfloat16)
            lse[l, at:at + n] = (top[..., 0] + total.log().reshape(H_kv, n, n_rep)).transpose(0, 1).reshape(n, H_q)
        at += n
    return {"out": out, "lse": lse}


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    d_h, width = c["d_h"], dict(bf16=2, fp16=2, fp32=4).get(c.get("dtype"), 2)
    if c["op"] == "rope":
        heads = c["n_tok"] * (c["H_q"] + c["H_kv"])
        return {"bytes": heads * 2 * d_h * width + 4 * c["n_tok"], "flops": heads * c["rot"] * 3}
    if c["op"] == "assign":
        new = c["batch"] * c["new"] // (2 if c["ragged"] else 1)
        # lengths in and out and the places where sequences begin, twice; new tokens' positions and slots; entries of the table
        return {"bytes": c["batch"] * 32 + new * 8 + 16 * c["batch"] * max(1, c["new"] // c["page"]), "flops": 0}
    heads = c["G"] * c["H_kv"]
    if c["op"] == "read":
        return {"bytes": heads * sum(_lens(c)) * 2 * d_h * 3, "flops": 0}
    lens, news = _lens(c), _news(c)
    if c["op"] == "append":
        return {"bytes": heads * (sum(news) * 2 * d_h * 3 + sum(a + n for a, n in zip(lens, news)) * 2 * d_h * 3), "flops": 0}
    rows, pairs, tokens = 0, 0, 0
    for a, n in zip(lens, news):
        rows += heads * (a + n)
        pairs += c["G"] * c["H_q"] * (n * a + n * (n + 1) // 2)
        tokens += c["G"] * c["H_q"] * n
    return {"bytes": rows * 2 * d_h + tokens * (4 * d_h + 4), "flops": pairs * 4 * d_h}


# ---------------------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits


def _exact_rope(s):
    c, r = s["case"], ROPE
    n = c["rot"]
    out = {"q": s["q"].double(), "k": s["k"].double()}
    gain = 1.0
    for i in range(n // 2):
        base = r["base"] * (r["factor"] ** (n / (n - 2)) if c["scaling"] == "ntk" and n > 2 else 1.0)
        f = math.exp(-2 * i / n * math.log(base))
        if c["scaling"] == "linear":
            f /= r["factor"]
        elif c["scaling"] == "llama3":
            wave = 2 * math.pi / f
            if wave > r["original"] / r["low"]:
                f /= r["factor"]
            elif wave > r["original"] / r["high"]:
                smooth = (r["original"] / wave - r["low"]) / (r["high"] - r["low"])
                f = (1 - smooth) * f / r["factor"] + smooth * f
        elif c["scaling"] == "yarn":
            low = max(math.floor(n * math.log(r["original"] / (r["beta_fast"] * 2 * math.pi)) / (2 * math.log(base))), 0)
            high = min(math.ceil(n * math.log(r["original"] / (r["beta_slow"] * 2 * math.pi)) / (2 * math.log(base))), n - 1)
            ramp = min(max((i - low) / max(high - low, 0.001), 0.0), 1.0)
            f = f / r["factor"] * ramp + f * (1 - ramp)
            gain = 0.1 * math.log(r["factor"]) + 1.0
        turn = torch.exp(1j * (s["pos"].double() * f))[:, None]
        if c["direction"] != "forward":
            turn = turn.conj()
        turn = turn / gain if c["direction"] == "inverse" else turn * gain
        a, b = (i, i + n // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        for name, y in out.items():
            z = torch.complex(s[name][..., a].double(), s[name][..., b].double()) * turn
            y[..., a], y[..., b] = z.real, z.imag
    return out


def _round_e4m3(x):
    """The nearest value of e4m3, ties to even: steps of 2^(e - 3) for 2^e <= |x| < 2^(e + 1), of 2^-9 below 2^-6 (float64)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _values(codes, scale):
    return codes.double() * scale.double()[..., None, None]


def _exact_append(s):
    c, page = s["case"], s["page"]
    slots = s["slot"].tolist()
    out = {}
    by_page = {}
    for t, slot in enumerate(slots):
        by_page.setdefault(slot // page, []).append((slot % page, t))
    for name, x in (("K", s["k"].double()), ("V", s["v"].double())):
        codes, scale = s[name].double(), s[name.lower() + "_scale"].double()
        for p, rows in by_page.items():
            begin = min(off for off, _ in rows)
            new = x[:, [t for _, t in rows]]                                        # [G][rows][H_kv][d_h]
            top = new.abs().amax((1, 3))
            e = torch.floor(torch.log2(top.clamp_min(2.0 ** -90))) - 9              # or one or two more, whatever the logarithm's last bit
            for _ in range(3):
                e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
            e = e.clamp_min(LOWEST)
            if begin:
                before = torch.log2(scale[:, p])
                e = torch.maximum(e, before)
                codes[:, p, :, :begin] = _round_e4m3(codes[:, p, :, :begin] * torch.exp2(before - e)[..., None, None])
            codes[:, p, :, [off for off, _ in rows]] = _round_e4m3(new.transpose(1, 2) * torch.exp2(-e)[..., None, None])
            scale[:, p] = torch.exp2(e)
        out[name], out[name.lower() + "_scale"] = codes, scale
    read = _exact_read(dict(s, **out))
    return dict(read, k_scale=out["k_scale"], v_scale=out["v_scale"])


def _exact_read(s):
    c, page = s["case"], s["page"]
    out = {"k_scale": None, "v_scale": None}
    for name in ("K", "V"):
        y = s[name + "_out"].double()
        value = _values(s[name], s[name.lower() + "_scale"])
        for b, rows in enumerate(s["length"].tolist()):
            for j in range(_pages_of(rows, page)):
                n = min(page, rows - j * page)
                y[:, b, :, j * page:j * page + n] = value[:, int(s["table"][b, j]), :, :n]
        out[name] = y
    return out


def _exact_attend(s):
    c = s["case"]
    G, H_kv, H_q, d_h, page = (c[k] for k in ("G", "H_kv", "H_q", "d_h", "page"))
    n_rep, at = H_q // H_kv, 0
    out, lse = s["out"].double(), s["lse"].double()
    for b, (rows, n) in enumerate(zip(s["lens"], s["news"])):
        pages = s["table"][b, :_pages_of(rows, page)].long()
        hidden = torch.ones((n, rows), dtype=torch.bool, device="cuda").triu(rows - n + 1).repeat_interleave(n_rep, 0)
        for l in range(G):
            for h in range(H_kv):
                K, V = (_values(s[x][l].view(torch.uint8)[pages, h].view(torch.float8_e4m3fn),
                                s[x.lower() + "_scale"][l][pages, h]).reshape(-1, d_h)[:rows] for x in ("K", "V"))
                mine = slice(h * n_rep, (h + 1) * n_rep)
                q = s["q"][l, at:at + n, mine].double().reshape(n * n_rep, d_h)
                z = (q @ K.T / math.sqrt(d_h)).masked_fill_(hidden, -math.inf)
                total = torch.logsumexp(z, 1)
                out[l, at:at + n, mine] = (torch.exp(z - total[:, None]) @ V).reshape(n, n_rep, d_h)
                lse[l, at:at + n, mine] = total.reshape(n, n_rep)
        at += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] == "assign":
        return None                              # whole numbers: the plain form's own
    s = globals()["_prepare_" + case["op"]](case, torch.Generator(device="cuda").manual_seed(seed), seed)
    s["case"] = case
    return globals()["_exact_" + case["op"]](s)
