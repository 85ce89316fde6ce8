"""A step without new tokens through the calls that take any number of them."""
import pytest
import torch

from tests.test_gpu_cache8_loop import Server, projection, xkv  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_a_step_without_tokens(xkv):  # noqa: F811
    s = Server(xkv, batch=2)
    want = torch.tensor([30, 17], dtype=torch.int32, device="cuda")
    s.step(projection(s, 47, 1), want, 30)
    state = [t.clone() for t in (s.table, s.ring, s.state, s.length, s.K.view(torch.uint8), s.V.view(torch.uint8), s.ks, s.vs)]
    i32 = dict(dtype=torch.int32, device="cuda")
    qkv, pos, slot = projection(s, 0, 2), torch.empty(0, **i32), torch.empty(0, **i32)
    q, k = torch.empty((s.G, 0, s.H_q, s.d), dtype=torch.bfloat16, device="cuda"), torch.empty((s.G, 0, s.H_kv, s.d), dtype=torch.bfloat16, device="cuda")
    xkv.xkv_page_assign(s.cfg, s.length, want, s.table, s.ring, s.state, s.first, s.length, pos, slot, s.flags)
    assert s.first.tolist() == [0, 0, 0]
    for direction in ("forward", "adjoint", "inverse"):
        xkv.xkv_rope(s.rope, qkv[:, :, :s.H_q], pos, q, qkv[:, :, s.H_q:s.H_q + s.H_kv], k, direction=direction)
        xkv.xkv_rope(s.rope, q, pos, direction=direction)
    xkv.xkv_cache8_append(s.cfg, 0, s.G, k, torch.empty_like(k), slot, s.K, s.V, s.ks, s.vs, s.flags)
    for was, t in zip(state, (s.table, s.ring, s.state, s.length, s.K.view(torch.uint8), s.V.view(torch.uint8), s.ks, s.vs)):
        assert torch.equal(was, t)
    assert int(s.flags) == 0
