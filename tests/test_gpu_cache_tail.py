"""The operators over an uncompressed cache on the uncompressed tail of a compressed window: its rows are weighed with the log-sum-exp
of xkv_sr_reconstruct_attend_tail (the joint softmax of selected and tail rows), the tail is bounded, and the next step attends to
what is left of it."""
import math

import numpy as np
import pytest
import torch

from paper_2503_18893_b200 import synth
from tests import _cache_ref as R
from tests import _cases as C
from tests.test_gpu_tail import TOL, _fixed_selection, _key_rms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("over,cap,lens,keep", [
    (dict(T=1024, k=128, batch=2, d_h=128, r_k=64, r_v=64), 700, [650, 333], 300),
    (dict(T=1024, k=128, H_kv=2, H_q=14, d_h=128, r_k=96, r_v=160), 1500, [1400], 1000),
    (dict(T=1024, k=128, batch=3), 600, [600, 0, 129], 100)], ids=["d128_batch2", "d128_rep7", "d64_batch3"])
def test_a_bounded_tail(over, cap, lens, keep):
    s = synth.config(1, **over)
    inp = C.case_from_factors(s, n_steps=2)
    g = C.GpuCase(s, inp)
    x = g.xkv
    tk, tv = (t.cuda() for t in synth.make_tail(s, cap, key_rms=_key_rms(s, inp), value_rms=1.0))
    idx, cnt = _fixed_selection(s, 100)
    idx_d, cnt_d = torch.from_numpy(idx).cuda(), torch.from_numpy(cnt).cuda()
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.empty(x.xkv_tail_workspace_bytes(g.grp, cap), dtype=torch.uint8, device="cuda")
    out = torch.zeros((s.G, s.batch, s.H_q, s.d_h), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((s.G, s.batch, s.H_q), device="cuda")
    cfg = x.make_cache_config(G=s.G, batch=s.batch, H_kv=s.H_kv, H_q=s.H_q, d_h=s.d_h, cap=cap)
    weights = torch.full((s.G, s.batch, s.H_kv, cap), 7.0, device="cuda")
    before = weights.clone()
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    q0 = g.inp.q[0].reshape(s.G, s.batch, 1, s.H_q, s.d_h)
    x.xkv_sr_reconstruct_attend_tail(g.grp, 0, s.G, g.inp.q[0], idx_d, cnt_d, idx.shape[-1], tk, tv, ln, cap, ws, out, lse)
    x.xkv_cache_weigh(cfg, 0, s.G, q0, 1, lse.reshape(s.G, s.batch, 1, s.H_q), tk, ln, None, torch.zeros_like(ln), 1.0, weights, flags)
    want, err = R.weigh_ref(q0, lse.reshape(s.G, s.batch, 1, s.H_q).cpu(), tk, lens, torch.tensor(lens)[:, None], [0] * s.batch, 1.0, before,
                            1 / math.sqrt(s.d_h))
    for b, n in enumerate(lens):
        assert ((weights[:, b, :, :n].double() - want[:, b, :, :n]).abs() <= err[:, b, :, :n]).all() and (weights[:, b, :, n:] == 7).all()
    if max(lens) > 0:                            # a share of the joint softmax: together less than one a query head
        b = int(np.argmax(lens))
        total = weights[:, b, :, :lens[b]].double().sum(-1)
        assert (total > 0).all() and (total < s.H_q // s.H_kv).all()
    # the rows of the largest weight and the last 20 stay
    src = torch.zeros((s.G, s.batch, s.H_kv, keep), dtype=torch.int32, device="cuda")
    since = torch.tensor([max(0, n - 20) for n in lens], dtype=torch.int32, device="cuda")
    x.xkv_evict_select(cfg, 0, s.G, weights, None, since, ln, keep, src, flags)
    old_k, old_v, drawn = tk.clone(), tv.clone(), weights.cpu()
    x.xkv_evict_compact(cfg, 0, s.G, tk, tv, src, keep, weights, None, flags)
    ln.clamp_(max=keep)
    x.xkv_sr_reconstruct_attend_tail(g.grp, 0, s.G, g.inp.q[1], idx_d, cnt_d, idx.shape[-1], tk, tv, ln, cap, ws, out, lse)
    torch.cuda.synchronize()
    assert flags.item() == 0 and g.status() == (0, 0)
    left_k, left_v = torch.zeros_like(tk[:, :, :, :keep]), torch.zeros_like(tv[:, :, :, :keep])
    for l in range(s.G):
        for b in range(s.batch):
            for h in range(s.H_kv):
                rows = R.select_ref(drawn[l, b, h], None, int(since[b]), lens[b], keep)
                assert src[l, b, h].tolist() == rows, (l, b, h)
                at = [r for r in rows if r >= 0]
                left_k[l, b, h, :len(at)], left_v[l, b, h, :len(at)] = old_k[l, b, h, at], old_v[l, b, h, at]
                assert torch.equal(tk[l, b, h, :len(at)], left_k[l, b, h, :len(at)]) and torch.equal(tv[l, b, h, :len(at)], left_v[l, b, h, :len(at)])
    n_left = [min(n, keep) for n in lens]
    want_out, want_lse = C.oracle_step_with_tail(s, inp, idx, cnt, left_k.cpu(), left_v.cpu(), n_left, step=1)
    assert C.rel_err(C.f32(out), want_out) <= TOL
    np.testing.assert_allclose(lse.cpu().numpy(), want_lse, atol=2e-2)
    g.close()
