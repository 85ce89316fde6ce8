"""Definitions of rotary positions and of the operators over a paged cache of 8-bit codes in 64 bits, and bounds of what kernels that
sum in fp32 may differ by."""
import math

import torch

BF16 = torch.finfo(torch.bfloat16).eps / 2           # 2^-8: half a step, relative
LOWEST = -60


def round_e4m3(x):
    """The nearest value of e4m3, ties to even, magnitudes above 448 cut (float64; NaN stays)."""
    a = x.abs().clamp(max=448.0)
    m, ex = torch.frexp(a.clamp_min(2.0 ** -6))
    step = torch.ldexp(torch.ones_like(a), (ex - 1 - 3).to(torch.float64))
    return torch.copysign(torch.round(a / step) * step, x)


def exponent(top):
    """The smallest e >= -60 with top <= 448 * 2^e (a float)."""
    e = LOWEST
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def append_ref(values, scale, rows, slot, page):
    """values float64 [G][n_pages][H][page][d] (codes, not times their scale), scale float64 [G][n_pages][H], rows [G][n_tok][H][d]: what
    they are after the call (in place), run by run."""
    n_pages = values.shape[1]
    t, n = 0, len(slot)
    while t < n:
        s = slot[t]
        if s < 0 or s >= n_pages * page:
            t += 1
            continue
        p, off, m = s // page, s % page, 1
        while t + m < n and off + m < page and slot[t + m] == s + m:
            m += 1
        for l in range(values.shape[0]):
            for h in range(values.shape[2]):
                x = rows[l, t:t + m, h].double()
                fin = x[torch.isfinite(x)].abs()
                e = exponent(float(fin.max()) if fin.numel() else 0.0)
                if off:
                    old = int(math.log2(float(scale[l, p, h])))
                    e = max(e, old)
                    values[l, p, h, :off] = round_e4m3(values[l, p, h, :off] * 2.0 ** (old - e))
                values[l, p, h, off:off + m] = round_e4m3(x * 2.0 ** -e)
                scale[l, p, h] = 2.0 ** e
        t += m


def assign_ref(page, n_pages, max_pages, held, want, table, ring, state, n_tok):
    """Lists in, lists out: (table, ring, state, first, length, pos, slot, flagged)."""
    most = max_pages * page
    table, ring, flagged = [list(r) for r in table], list(ring), False
    head, count = state
    if not (0 <= head < n_pages and 0 <= count <= n_pages):
        head = count = 0
        flagged = True
    room, wanted, taken, back = n_pages - count, 0, 0, 0
    first, length, pos, slot = [0], [], [], []
    old = list(ring)
    for b in range(len(held)):
        h, w = min(max(held[b], 0), most), min(max(want[b], 0), most)
        flagged |= h != held[b] or w != want[b]
        have, need = -(-h // page), -(-w // page)
        ok = True
        if need > have:
            wanted += need - have
            ok = wanted <= count
            if ok:
                for i in range(need - have):
                    table[b][have + i] = old[(head + wanted - (need - have) + i) % n_pages]
                taken = wanted
        for i in range(need, have):
            if back < room:
                ring[(head + count + back) % n_pages] = table[b][i]
            else:
                flagged = True
            back += 1
            table[b][i] = -1
        length.append(w if ok else h)
        first.append(first[-1] + max(w - h, 0))
        for j in range(h, w):
            p = table[b][j // page] if ok else -1
            good = 0 <= p < n_pages
            flagged |= ok and not good
            pos.append(j)
            slot.append(p * page + j % page if good else -1)
    flagged |= len(pos) > n_tok
    pos, slot = (pos + [0] * n_tok)[:n_tok], (slot + [-1] * n_tok)[:n_tok]
    return table, ring, [(head + taken) % n_pages, count - taken + min(back, room)], first, length, pos, slot, flagged


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0.0, low=1.0, high=4.0, beta_fast=32.0, beta_slow=1.0):
    """(radians per position of every pair, gain)."""
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f, gain = [base ** (-2 * i / rot) for i in range(rot // 2)], 1.0
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "llama3":
        def banded(x):
            wave = 2 * math.pi / x
            if wave < original / high:
                return x
            if wave > original / low:
                return x / factor
            s = (original / wave - low) / (high - low)
            return (1 - s) * x / factor + s * x
        f = [banded(x) for x in f]
    if scaling == "yarn":
        def at(beta):
            return rot * math.log(original / (2 * math.pi * beta)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(beta_fast)), 0), min(math.ceil(at(beta_slow)), rot - 1)
        ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(rot // 2)]
        f = [r * x / factor + (1 - r) * x for r, x in zip(ramp, f)]
        gain = 0.1 * math.log(factor) + 1.0
    return torch.tensor(f, dtype=torch.float64), gain


def rotate(x, pos, f, gain, layout, direction="forward"):
    """x [rows][heads][d] any type, pos [rows] -> (float64 result, sum of the magnitudes that each element is made of)."""
    x = x.double()
    n = 2 * len(f)
    a, b = (torch.arange(n // 2), torch.arange(n // 2) + n // 2) if layout == "half" else (torch.arange(0, n, 2), torch.arange(1, n, 2))
    angle = (pos.double()[:, None] * f.to(pos.device))[:, None]
    c, s = angle.cos(), angle.sin()
    if direction != "forward":
        s = -s
    g = 1 / gain if direction == "inverse" else gain
    y, mag = x.clone(), x.abs()
    y[..., a], y[..., b] = g * (x[..., a] * c - x[..., b] * s), g * (x[..., b] * c + x[..., a] * s)
    mag[..., a] = mag[..., b] = g * (x[..., a].abs() + x[..., b].abs())
    return y, mag


def attend_ref(q, first, max_new, table, length, K, V, ks, vs, page, n_rep, scale, n_tok):
    """q [n_tok][H_q][d]; K, V float64 codes [n_pages][H][page][d], ks, vs [n_pages][H] of one layer.  Returns float64 (out, lse, bound of
    out, bound of lse), NaN in rows of `out` that the call leaves alone."""
    d, H_q = q.shape[-1], q.shape[1]
    n_pages = K.shape[0]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(length)):
        f0, f1 = min(max(first[b], 0), n_tok), min(max(first[b + 1], 0), n_tok)
        n = f1 - f0
        rows_b = min(max(length[b], 0), len(table[b]) * page)
        for i in range(min(max(n, 0), max_new)):
            rows = max(0, min(rows_b, rows_b - n + i + 1))
            keep = [j for j in range(rows) if 0 <= table[b][j // page] < n_pages]
            pg = torch.tensor([table[b][j // page] for j in keep], dtype=torch.long)
            off = torch.tensor([j % page for j in keep], dtype=torch.long)
            for h in range(H_q):
                g = h // n_rep
                if len(keep):
                    sk, sv = ks[pg, g], vs[pg, g]
                    live = (sk > 0) & (sv > 0)
                    p2, o2, sk, sv = pg[live], off[live], sk[live], sv[live]
                if not len(keep) or not len(p2):
                    out[f0 + i, h], lse[f0 + i, h] = 0.0, -math.inf
                    continue
                k, c = K[p2, g, o2] * sk[:, None], V[p2, g, o2]
                x = q[f0 + i, h].double()
                z = k @ x * scale
                total = torch.logsumexp(z, 0)
                p = torch.exp(z - total)
                o = p @ (c * sv[:, None])
                mag = p @ (c.abs() * sv[:, None])
                # products in fp32: d additions, each by a step of the sum of magnitudes; queries to 2^-18 of their largest element
                ze = scale * float((d * 2.0 ** -23 * (k.abs() @ x.abs()) + 2.0 ** -18 * x.abs().max() * k.abs().sum(1)).max())
                ze += 2.0 ** -20 * (1 + abs(float(total)))
                out[f0 + i, h], lse[f0 + i, h] = o, total
                # weights to 2^-11 of themselves or 2^-21 of the largest (times its scale)
                bo[f0 + i, h] = BF16 * o.abs() * (1 + BF16) + (2.0 ** -11 + 2 * ze + 2.0 ** -16) * mag + 2.0 ** -21 * (p * sv).max() * c.abs().sum(0) + 1e-30
                bl[f0 + i, h] = ze
    return out, lse, bo, bl
