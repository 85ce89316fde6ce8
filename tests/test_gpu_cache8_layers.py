"""More layers than a grid has room for in one dimension: rows of one head into codes, back, and attended to, in all of them."""
import pytest
import torch

from tests import test_gpu_cache8_codes as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def test_forty_thousand_layers(xkv):
    G, d, n = 40000, 64, 3
    p = C.Pool(xkv, G, 1, d, 16, 1, seed=4)
    k, v = C.rows(p, n), C.rows(p, n, 3.0)
    slot, table, length = C.dev([0, 1, 2]), C.dev([[0]]), C.dev([n])
    xkv.xkv_cache8_append(p.cfg, 0, G, k, v, slot, p.K, p.V, p.ks, p.vs, p.flags)
    K, V = (torch.zeros((G, 1, 1, 16, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xkv.xkv_cache8_read(p.cfg, 0, G, table, length, p.K, p.V, p.ks, p.vs, K, V, p.flags)
    assert int(p.flags) == 0
    for x, y, s in ((k, K, p.ks), (v, V, p.vs)):
        top = x.float().abs().amax((1, 2, 3))
        e = torch.frexp(top / 448.0)
        assert torch.equal(s.flatten(), 2.0 ** (e.exponent - (e.mantissa == 0.5).int()).float())
        want = ((x.float() / s[:, :, :, None]).to(torch.float8_e4m3fn).float() * s[:, :, :, None]).to(torch.bfloat16)
        assert torch.equal(y[:, 0, 0, :n], want[:, :, 0]) and not bool(y[:, 0, 0, n:].any())
    # a call over the last layers alone
    K2 = torch.zeros_like(K)
    xkv.xkv_cache8_read(p.cfg, G - 5, G, table, length, p.K, p.V, p.ks, p.vs, K2, None, p.flags)
    assert torch.equal(K2[-5:], K[-5:]) and not bool(K2[:-5].any())
    # one row of weight one: the value itself
    q = torch.zeros((G, 1, 1, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(xkv.xkv_cache8_workspace_bytes(p.cfg, 1), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    xkv.xkv_cache8_attend(p.cfg, 0, G, q, None, 1, table, C.dev([1]), p.K, p.V, p.ks, p.vs, ws, out)
    assert torch.equal(out[:, 0, 0], V[:, 0, 0, 0])
