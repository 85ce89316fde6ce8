"""Definitions of the operators over an uncompressed cache in 64 bits (torch, head by head), and bounds for what a kernel that
sums in fp32 and rounds weights and outputs to bf16 may differ by."""
import math

import torch

BF16 = torch.finfo(torch.bfloat16).eps / 2           # 2^-8: half a step, relative


def words(sees):
    """int32 words [batch][n][ceil(n/32)] of a bool [batch][n][n] (CPU)."""
    batch, n, _ = sees.shape
    w = -(-n // 32)
    bits = torch.zeros((batch, n, w * 32), dtype=torch.int64)
    bits[:, :, :n] = sees.long()
    v = (bits.reshape(batch, n, w, 32) << torch.arange(32)).sum(-1)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).to(torch.int32)


def random_tree(n, g):
    """bool [n][n]: every token sees itself and its ancestors."""
    sees = torch.eye(n, dtype=torch.bool)
    for i in range(1, n):
        p = int(torch.randint(-1, i, (1,), generator=g))
        if p >= 0:
            sees[i] |= sees[p]
    return sees


def head_attend(q, K, V, at, scale):
    """q [m][d], K, V [rows][d], at bool [m][rows] -> (out, lse, sum p |v|, largest sum_i |q_i k_ji| scale) in 64 bits; rows that a
    query does not attend to are not touched."""
    q, K, V = q.double(), K.double(), V.double()
    d = V.shape[1]
    out = torch.zeros((q.shape[0], d), dtype=torch.float64, device=q.device)
    lse = torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    mag, top = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(q.shape[0]):
        k = K[at[i]]
        if not k.shape[0]:
            continue
        z = k @ q[i] * scale
        lse[i] = torch.logsumexp(z, 0)
        p = torch.exp(z - lse[i])
        out[i] = p @ V[at[i]]
        mag[i] = p @ V[at[i]].abs()
        top[i] = (k.abs() @ q[i].abs()).max() * scale
    return out, lse, mag, top


def attend_bounds(out, lse, mag, top, d):
    """A sum of d products in fp32 is off by at most d 2^-23 of the sum of their magnitudes (each of d additions by one step, a
    tensor core may truncate): that is the error of a logit, and so the relative error of a weight and the error of the
    log-sum-exp.  Weights and the output are rounded to bf16; exponentials, their sums and the value sums are fp32."""
    z = d * 2.0 ** -23 * top + 2.0 ** -20 * (1 + lse.abs().nan_to_num(posinf=0, neginf=0))
    return BF16 * out.abs() * (1 + BF16) + (BF16 + 2 * z[:, None] + 2.0 ** -16) * mag + 1e-30, z


def weigh_ref(q, lse, K, length, visible, seen, decay, weights, scale):
    """64-bit weights after the call; also the bound of their error."""
    G, batch, n, H_q, d = q.shape
    H_kv = K.shape[2]
    rep = H_q // H_kv
    w, err = weights.double(), torch.zeros_like(weights, dtype=torch.float64)
    for l in range(G):
        for b in range(batch):
            for h in range(H_kv):
                ln = int(length[b])
                old = w[l, b, h, :ln].clone()
                old[int(seen[b]):] = 0
                acc = decay * old if decay else torch.zeros_like(old)
                e = acc.abs() * 2.0 ** -22
                for i in range(n):
                    vis = int(visible[b, i])
                    for r in range(rep):
                        L = float(lse[l, b, i, h * rep + r])
                        if not vis or L == -math.inf:
                            continue
                        k, x = K[l, b, h, :vis].double(), q[l, b, i, h * rep + r].double()
                        p = torch.exp(k @ x * scale - L)
                        acc[:vis] += p
                        e[:vis] += p * (d * 2.0 ** -23 * (k.abs() @ x.abs()) * scale + 2.0 ** -21 * (4 + abs(L)))
                w[l, b, h, :ln] = acc
                err[l, b, h, :ln] = e + acc.abs() * n * rep * 2.0 ** -24 + 1e-35
    return w, err


def select_ref(weights, pos, since, length, keep):
    """The map of one head, row by row from the definition."""
    rows = list(range(length))
    w = [-math.inf if math.isnan(x) else float(x) for x in weights[:length].tolist()]
    p = pos.tolist() if pos is not None else list(range(len(weights)))
    order = sorted(rows, key=lambda j: (0 if since is not None and p[j] >= since else 1, -w[j], j))
    stays = set(order[:keep])
    movers = iter(sorted(j for j in stays if j >= keep))
    return [-1 if j >= length else j if j in stays else next(movers) for j in range(keep)]
