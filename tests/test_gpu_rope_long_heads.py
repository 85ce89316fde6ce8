"""Heads of more places than a CTA has threads, and others at the ends of what is taken, at addresses that allow pieces of 16 bytes and not."""
import pytest
import torch

from tests import _cache8_ref as R
from tests.test_gpu_rope import check, xkv  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d_h,rot", [(1024, 256), (1024, 2), (1022, 254), (514, 130), (512, 256), (768, 64), (1000, 8)])
def test_long_heads(xkv, dtype, layout, d_h, rot):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(d_h + rot)
    plan = xkv.make_rope(d_h=d_h, rot=rot, layout=layout, base=500000.0)
    f, gain = R.frequencies(rot, base=500000.0)
    for rows, heads, heads2 in ((1, 1, 0), (5, 3, 2), (9, 1, 7), (4000, 1, 1)):
        for shift in (0, 1):                     # elements behind a 16-byte border
            def tensor(h):
                flat = torch.randn(rows * h * d_h + shift, generator=g, device="cuda").to(dtype)
                return flat[shift:].view(rows, h, d_h)
            x, y = tensor(heads), tensor(heads2)
            ox, oy = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
            pos = torch.randint(0, 1 << 18, (rows,), generator=g, device="cuda", dtype=torch.int32)
            for direction in ("forward", "adjoint"):
                xkv.xkv_rope(plan, x, pos, ox, y, oy, direction=direction)
                check(ox, x, pos, f, gain, layout, direction, dtype)
                check(oy, y, pos, f, gain, layout, direction, dtype)
            keep, want_y = x.clone(), oy.clone()
            xkv.xkv_rope(plan, x, pos, None, y, oy, direction="adjoint")             # one in place, one not
            assert torch.equal(x, ox) and torch.equal(oy, want_y)
            x.copy_(keep)
            xkv.xkv_rope(plan, x, pos, direction="adjoint")
            assert torch.equal(x, ox)
