"""Calls one behind the other in a stream, each reading what the one before has just written, give the same bits as with the device
idle in between: selection and attention, attention over an uncompressed cache and its merge, codes and their values."""
import pytest
import torch

from paper_2503_18893_b200 import synth
from tests import _cases as C

pytestmark = pytest.mark.gpu


def both(calls, results):
    """Runs `calls` with the device idle after each, then several times without a pause; `results()` has to be the same."""
    for call in calls:
        call()
        torch.cuda.synchronize()
    want = [t.clone() for t in results()]
    for _ in range(4):
        for t in results():
            t.zero_()
        torch.cuda.synchronize()
        for call in calls:
            call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(), want))


@pytest.mark.parametrize("d_h", [64, 128])
def test_selection_and_attention(d_h):
    s = synth.config(1, T=4096, k=256, d_h=d_h, r_k=64, r_v=64)
    g = C.GpuCase(s, C.case_from_factors(s, n_steps=6))
    x = g.xkv
    idx = torch.zeros((s.G, s.batch, s.H_kv, s.k), dtype=torch.int32, device="cuda")
    cnt = torch.zeros((s.G, s.batch, s.H_kv), dtype=torch.int32, device="cuda")
    out = torch.zeros((6, s.G, s.batch, s.H_q, s.d_h), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((6, s.G, s.batch, s.H_q), device="cuda")
    calls = []
    for t in range(6):                               # one pair of index arrays, written anew by every step
        calls.append(lambda t=t: x.xkv_sr_select(g.grp, 0, s.G, g.inp.q[t], s.k, idx, cnt))
        calls.append(lambda t=t: x.xkv_sr_reconstruct_attend(g.grp, 0, s.G, g.inp.q[t], idx, cnt, s.k, out[t], lse[t]))
    both(calls, lambda: (out, lse))
    assert g.status() == (0, 0)
    g.close()


def test_attention_over_an_uncompressed_cache():
    s = synth.config(1, T=256, k=64, d_h=128, r_k=64, r_v=64)
    g = C.GpuCase(s, C.case_from_factors(s, n_steps=6))
    x, cap = g.xkv, 5000
    K, V = synth.make_tail(s, cap, key_rms=1.0, value_rms=1.0, device="cuda")
    ws = torch.empty(x.xkv_dense_workspace_bytes(g.grp, cap), dtype=torch.uint8, device="cuda")
    out = torch.zeros((6, s.G, s.batch, s.H_q, s.d_h), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((6, s.G, s.batch, s.H_q), device="cuda")
    both([lambda t=t: x.xkv_dense_attend(g.grp, 0, s.G, g.inp.q[t], K, V, None, cap, ws, out[t], lse[t]) for t in range(6)], lambda: (out, lse))
    g.close()


@pytest.mark.parametrize("bits", [3, 4])
def test_codes_and_their_values(bits):
    from paper_2503_18893_b200 import xkv
    gen = torch.Generator().manual_seed(bits)
    x = torch.randn((5, 3000, 256), generator=gen).to(torch.bfloat16).cuda()

    def values(pause):
        back = []
        for t in range(5):
            codes, meta = xkv.xkv_quantize_rtn(x[t], bits)
            if pause:
                torch.cuda.synchronize()
            back.append(xkv.xkv_dequantize_rtn(codes, meta, bits))
            if pause:
                torch.cuda.synchronize()
        return torch.stack(back)
    want = values(True)
    for _ in range(4):
        assert torch.equal(values(False), want)
