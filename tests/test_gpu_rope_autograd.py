"""Rotation where gradients are recorded: what is written into says so, and what autograd would not learn of is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import xkv as m
    return m


@pytest.fixture()
def case(xkv):
    plan, pos = xkv.make_rope(d_h=64), torch.arange(5, dtype=torch.int32, device="cuda")
    return plan, pos, torch.randn((5, 2, 64), device="cuda")


def test_a_tensor_saved_for_backward_and_then_rotated(xkv, case):
    plan, pos, x = case
    w = torch.ones_like(x).requires_grad_()
    for args in ((x, pos), (torch.zeros_like(x), pos, x), (torch.zeros_like(x), pos, None, x), (torch.zeros_like(x), pos, None, torch.zeros_like(x), x),
                 (x[:, :1], pos)):
        y = (w * x).sum()
        before = x._version
        xkv.xkv_rope(plan, *args)
        assert x._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_what_requires_a_gradient_is_not_written_into(xkv, case):
    plan, pos, x = case
    leaf = x.clone().requires_grad_()
    made = leaf * 2.0
    for t in (leaf, made, made[:, :1]):
        before = t.detach().clone()
        with pytest.raises(ValueError, match="requires a gradient"):
            xkv.xkv_rope(plan, t, pos)
        with pytest.raises(ValueError, match="requires a gradient"):
            xkv.xkv_rope(plan, torch.zeros_like(t).detach(), pos, t)
        with pytest.raises(ValueError, match="requires a gradient"):
            xkv.xkv_rope(plan, torch.zeros_like(t).detach(), pos, None, t)
        assert torch.equal(t.detach(), before)
    with torch.no_grad():
        xkv.xkv_rope(plan, leaf, pos)            # as torch's own calls in place
    assert leaf._version > 0
    out = torch.empty_like(x)
    xkv.xkv_rope(plan, leaf, pos, out)           # it is only read
    assert not out.requires_grad


def test_a_function_with_the_adjoint_as_its_gradient(xkv, case):
    """As a program records the rotation: the gradient against inner products in 64 bits and differences."""
    plan, pos, x = case

    class Rope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            out = torch.empty_like(x)
            xkv.xkv_rope(plan, x, pos, out)
            return out

        @staticmethod
        def backward(ctx, g):
            out = torch.empty_like(g)
            xkv.xkv_rope(plan, g.contiguous(), pos, out, direction="adjoint")
            return out

    x = x.requires_grad_()
    w = torch.randn_like(x)
    (Rope.apply(x) * w).sum().backward()
    e = torch.randn_like(x)
    with torch.no_grad():
        step = Rope.apply(x + e) - Rope.apply(x)             # linear: a difference of any size
    one, two = (step.double() * w).sum(), (e.double() * x.grad).sum()
    assert abs(float(one - two)) <= 2.0 ** -20 * float(((x.detach().abs() + e.abs()) * 4 * w.abs().amax()).double().sum())


def test_a_lazy_clone_is_not_written_through(xkv, case):
    plan, pos, x = case
    other = torch._lazy_clone(x)
    before = other.clone()
    xkv.xkv_rope(plan, x, pos)
    assert torch.equal(other, before) and not torch.equal(x, before)


def test_inference_tensors(xkv, case):
    plan, pos, _ = case
    with torch.inference_mode():
        x = torch.randn((5, 2, 64), device="cuda")
        want = torch.empty_like(x)
        xkv.xkv_rope(plan, x, pos, want)
        xkv.xkv_rope(plan, x, pos)
    assert torch.equal(x, want)
    xkv.xkv_rope(plan, x, pos)                   # outside as well
