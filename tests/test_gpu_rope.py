"""Rotary positions against their definition in 64 bits."""
import pytest
import torch

from tests import _cache8_ref as R

pytestmark = pytest.mark.gpu
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}
LONG = dict(base=500000.0, factor=8.0, original=8192.0, low=1.0, high=4.0, beta_fast=32.0, beta_slow=1.0)


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


def check(got, x, pos, f, gain, layout, direction, dtype):
    want, mag = R.rotate(x, pos, f, gain, layout, direction)
    # cosine, sine and the gain are off by 2^-22 of one, two products and a sum by 2^-22; then one rounding (of fp16's smallest: 2^-25)
    bound = HALF_STEP[dtype] * want.abs() + 2.0 ** -20 * mag + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert got.dtype == dtype and bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "llama3", "yarn"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("d_h,rot", [(128, 128), (64, 32), (128, 16), (80, 40), (256, 256), (6, 4), (2, 2)])
def test_sizes(xkv, scaling, layout, dtype, d_h, rot):
    if scaling == "ntk" and rot < 4:
        pytest.skip("refused")
    g = torch.Generator(device="cuda").manual_seed(d_h + rot)
    kw = LONG if scaling != "none" else dict(base=10000.0)
    plan = xkv.make_rope(d_h=d_h, rot=rot, layout=layout, scaling=scaling, **kw)
    f, gain = R.frequencies(rot, scaling=scaling, **kw)
    for rows, heads, heads2 in ((1, 1, 1), (7, 5, 3), (65, 28, 4)):
        x = torch.randn((rows, heads, d_h), generator=g, device="cuda").to(dtype)
        y = torch.randn((rows, heads2, d_h), generator=g, device="cuda").to(dtype)
        pos = torch.randint(0, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int32)
        ox, oy = torch.empty_like(x), torch.empty_like(y)
        for direction in ("forward", "adjoint", "inverse"):
            xkv.xkv_rope(plan, x, pos, ox, y, oy, direction=direction)
            check(ox, x, pos, f, gain, layout, direction, dtype)
            check(oy, y, pos, f, gain, layout, direction, dtype)


@pytest.mark.parametrize("pos", [0, 1, -1, 8191, 131071, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31)])
def test_far_positions(xkv, pos):
    plan = xkv.make_rope(d_h=128)
    f, gain = R.frequencies(128)
    x = torch.randn((3, 4, 128), device="cuda")
    p = torch.full((3,), pos, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    xkv.xkv_rope(plan, x, p, out)
    # (the definition's own angle is off by 2^-52 of itself at these positions)
    want, mag = R.rotate(x, p, f, gain, "half")
    assert bool(((out.double() - want).abs() <= (2.0 ** -20 + abs(pos) * 2.0 ** -51) * mag + 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_parts_of_a_projection_in_place_and_not(xkv, dtype, shift):
    """Queries and keys as slices of one tensor, at any element; what lies between stays as it was."""
    n, d = 37, 128
    flat = torch.randn(n * 13 * d + 16, device="cuda").to(dtype)
    qkv = flat[shift:shift + n * 13 * d].view(n, 13, d)
    before = flat.clone()
    plan = xkv.make_rope(d_h=d, rot=64)
    f, gain = R.frequencies(64)
    pos = torch.arange(n, device="cuda", dtype=torch.int32) + 1000
    q, k = qkv[:, :8], qkv[:, 8:10]
    q0, k0 = q.clone(), k.clone()
    out_q, out_k = torch.empty_like(q0), torch.empty((n, 2, d + 24), device="cuda", dtype=dtype)[..., :d]
    xkv.xkv_rope(plan, q, pos, out_q, k, out_k)
    assert torch.equal(flat, before)
    xkv.xkv_rope(plan, q, pos, None, k, None)
    assert torch.equal(q, out_q) and torch.equal(k, out_k)
    check(q, q0, pos, f, gain, "half", "forward", dtype)
    check(k, k0, pos, f, gain, "half", "forward", dtype)
    rest = flat.clone()
    rest[shift:shift + n * 13 * d].view(n, 13, d)[:, :10] = before[shift:shift + n * 13 * d].view(n, 13, d)[:, :10]
    assert torch.equal(rest, before)


def test_layers_share_positions(xkv):
    plan = xkv.make_rope(d_h=64)
    f, gain = R.frequencies(64)
    x = torch.randn((4, 11, 6, 64), device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 5000, (11,), device="cuda", dtype=torch.int32)
    out = torch.empty_like(x)
    xkv.xkv_rope(plan, x, pos, out)
    check(out.reshape(44, 6, 64), x.reshape(44, 6, 64), pos.repeat(4), f, gain, "half", "forward", torch.bfloat16)


def test_inverse_undoes_forward_and_adjoint_is_the_gradient(xkv):
    plan = xkv.make_rope(d_h=128, rot=96, layout="interleaved", scaling="yarn", **LONG)
    x, w = torch.randn((50, 3, 128), device="cuda"), torch.randn((50, 3, 128), device="cuda")
    pos = torch.randint(0, 100000, (50,), device="cuda", dtype=torch.int32)
    y, back, grad = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    xkv.xkv_rope(plan, x, pos, y)
    xkv.xkv_rope(plan, y, pos, back, direction="inverse")
    assert float((back - x).abs().max()) <= 2.0 ** -19 * 2 * float(x.abs().max()) * 2
    xkv.xkv_rope(plan, w, pos, grad, direction="adjoint")
    # <R x, w> = <x, R^T w>, and against differences: R is linear, so (R(x + h e) - R(x)) / h = R e
    one, two = (y.double() * w.double()).sum(-1), (x.double() * grad.double()).sum(-1)
    size = 2.0 ** -19 * 1.5 * 2 * (x.abs().double().sum(-1) * w.abs().double().amax(-1))
    assert bool(((one - two).abs() <= size).all())
    for e in (0, 17, 95, 96, 127):
        unit, col = torch.zeros_like(x), torch.empty_like(x)
        unit[..., e] = 1.0
        xkv.xkv_rope(plan, unit, pos, col)
        assert bool((((col * w).double().sum(-1) - grad[..., e].double()).abs() <= 2.0 ** -18 * 1.5 * 2 * w.abs().amax(-1)).all())


def test_tensors_that_are_refused(xkv):
    plan = xkv.make_rope(d_h=64)
    x, pos = torch.zeros((6, 2, 64), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (x[0], x[..., :32], x.transpose(1, 2), x.double(), x.cpu(), torch.zeros((2, 6, 2, 64), device="cuda")[:, :5], x[:5]):
        with pytest.raises(ValueError):
            xkv.xkv_rope(plan, bad, pos)
    for out in (x[:3], x.half(), x[:, :1], x.cpu()):
        with pytest.raises(ValueError):
            xkv.xkv_rope(plan, x, pos, out)
    for second in (x[:3], x.half()):
        with pytest.raises(ValueError):
            xkv.xkv_rope(plan, x, pos, None, second)
    with pytest.raises(TypeError):
        xkv.xkv_rope(plan, None, pos)
    with pytest.raises(TypeError):
        xkv.xkv_rope(plan, x, pos, 5)


def test_nothing_to_do(xkv):
    plan = xkv.make_rope(d_h=64)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    xkv.xkv_rope(plan, torch.empty((0, 3, 64), device="cuda"), pos)
    xkv.xkv_rope(plan, torch.empty((2, 0, 64), device="cuda"), pos)


def test_many_rows_beyond_32_bit_offsets(xkv):
    """2.2e9 elements: the last rows are where 32-bit offsets would wrap."""
    plan = xkv.make_rope(d_h=128)
    f, gain = R.frequencies(128)
    rows = (1 << 32) // (128 * 4) // 2 + 77
    x = torch.zeros((rows, 4, 128), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((90, 4, 128), device="cuda").to(torch.bfloat16)
    x[-90:] = tail
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    xkv.xkv_rope(plan, x, pos)
    check(x[-90:], tail, pos[-90:], f, gain, "half", "forward", torch.bfloat16)
    assert not bool(x[:-90].any())


def test_streams_and_graphs(xkv):
    plan = xkv.make_rope(d_h=128)
    f, gain = R.frequencies(128)
    x = torch.randn((64, 8, 128), device="cuda")
    pos = torch.arange(64, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    xkv.xkv_rope(plan, x, pos, out, stream=s)
    s.synchronize()
    check(out, x, pos, f, gain, "half", "forward", torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.xkv_rope(plan, x, pos, out)
    x.normal_()
    pos += 12345
    graph.replay()
    torch.cuda.synchronize()
    check(out, x, pos, f, gain, "half", "forward", torch.float32)
