"""Kernels that hold tensor memory of an SM at the same time on two streams: weights of a cache (all of it) one behind the other, beside
the attention over an uncompressed cache and over a window (a part, or all of it).  Results as without the other stream."""
import pytest
import torch

from paper_2503_18893_b200 import synth
from tests import _cases as C
from tests import test_gpu_cache_weigh as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_two_streams(d):
    s = synth.config(1, T=4096, k=256, d_h=128, r_k=64, r_v=64)
    g = C.GpuCase(s, C.case_from_factors(s))
    x, cap = g.xkv, 20000
    K, V = synth.make_tail(s, cap, key_rms=1.0, value_rms=1.0, device="cuda")
    ws = torch.empty(x.xkv_dense_workspace_bytes(g.grp, cap), dtype=torch.uint8, device="cuda")
    out = torch.zeros((s.G, s.batch, s.H_q, s.d_h), dtype=torch.bfloat16, device="cuda")
    w = W.make(n=3, lens=[3000, 411], batch=2, H_kv=2, H_q=8, d=d, seed=d)
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    ln, vis, seen, cfg = i32(w["lens"]), i32(w["visible"]), i32(w["seen"]), x.make_cache_config(**w["c"])
    got = w["w"].clone()

    def weigh(stream):
        got.copy_(w["w"]) if stream is None else None
        for _ in range(4):
            x.xkv_cache_weigh(cfg, 0, 1, w["q"], 3, w["lse"], w["K"], ln, vis, seen, 0.5, got, None, stream)

    def dense(stream):
        x.xkv_dense_attend(g.grp, 0, s.G, g.inp.q[0], K, V, None, cap, ws, out, None, stream)
    weigh(None)
    dense(None)
    torch.cuda.synchronize()
    want, want_out = got.clone(), out.clone()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(30):
        got.copy_(w["w"])
        out.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            dense(b)
        weigh(a)
        dense(b)
        torch.cuda.synchronize()
        assert torch.equal(got.nan_to_num(9), want.nan_to_num(9)) and torch.equal(out, want_out)
    assert g.status() == (0, 0)
    g.close()
