"""kv4.rope as a differentiable function: the gradient is the rotation turned back, bit for bit, whatever the gradient's strides."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import kv4
    return kv4, torch, torch.device("cuda:0")


def inputs(env, T=9, H=3, D=64, rot=32, dtype="float32"):
    kv4, torch, dev = env
    g = torch.Generator(device=dev).manual_seed(T + D)
    table = kv4.rope_table(500, rot, magnitude=1.25, device=dev)
    pos = torch.randint(0, 500, (T,), generator=g, device=dev, dtype=torch.int32)
    return torch.randn(T, H, D, generator=g, device=dev).to(getattr(torch, dtype)), pos, table, g


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 32), (20, 12)])
def test_gradient(env, dtype, interleaved, inverse, D, rot):
    kv4, torch, dev = env
    x, pos, table, g = inputs(env, D=D, rot=rot, dtype=dtype)
    plain = kv4.rope(x, pos, table, interleaved=interleaved, inverse=inverse)
    assert not plain.requires_grad
    x.requires_grad_()
    y = kv4.rope(x, pos, table, interleaved=interleaved, inverse=inverse)
    assert y.requires_grad and torch.equal(y.detach(), plain)
    up = torch.randn(y.shape, generator=g, device=dev).to(x.dtype)
    y.backward(up)
    assert torch.equal(x.grad, kv4.rope(up, pos, table, interleaved=interleaved, inverse=not inverse))
    with torch.no_grad():
        assert not kv4.rope(x, pos, table).requires_grad


def test_gradients_of_any_strides(env):
    kv4, torch, dev = env
    x, pos, table, g = inputs(env)
    x.requires_grad_()
    kv4.rope(x, pos, table).sum().backward()                                  # one number, strides of 0
    assert torch.equal(x.grad, kv4.rope(torch.ones_like(x), pos, table, inverse=True))
    up = torch.randn(64, 3, 9, generator=g, device=dev).permute(2, 1, 0)      # channels outermost
    (got,) = torch.autograd.grad(kv4.rope(x, pos, table), x, up)
    assert torch.equal(got, kv4.rope(up.contiguous(), pos, table, inverse=True))


def test_against_differences(env):
    """The directional derivative of a loss, against differences of its value: steps of 2^-3 on values below 8 whose rotation is rounded to
    2^-24 of them; the loss is quadratic, so that central differences have no error of their own."""
    kv4, torch, dev = env
    x, pos, table, g = inputs(env)
    w = torch.randn(x.shape, generator=g, device=dev, dtype=torch.float64)
    d = torch.sign(torch.randn(x.shape, generator=g, device=dev))
    loss = lambda z: (w * kv4.rope(z, pos, table).double() ** 2).sum()  # noqa: E731
    x.requires_grad_()
    (grad,) = torch.autograd.grad(loss(x), x)
    h = 2.0 ** -3
    with torch.no_grad():
        diff = float((loss(x + h * d) - loss(x - h * d)) / (2 * h))
    # per element: two losses w y^2 off by 2 w |y| 4 |y| 2^-24, over 2 h; the gradient, 2 w y rounded to fp32 and turned, by 4 2^-24 of its size
    y = kv4.rope(x.detach(), pos, table).double().abs() + 1
    bound = float((w.abs() * (8 * y * y / h + 16 * y)).sum()) * 2.0 ** -24
    assert abs(diff - float((grad.double() * d).sum())) <= bound


def test_second_order_and_forward_mode(env):
    kv4, torch, dev = env
    import torch.autograd.forward_ad as fwad
    x, pos, table, g = inputs(env)
    x.requires_grad_()
    up = torch.randn(x.shape, generator=g, device=dev, requires_grad=True)
    (grad,) = torch.autograd.grad(kv4.rope(x, pos, table), x, up, create_graph=True)
    other = torch.randn(x.shape, generator=g, device=dev)
    (second,) = torch.autograd.grad(grad, up, other)                          # linear: the map itself
    assert torch.equal(second, kv4.rope(other, pos, table))
    with fwad.dual_level():
        t = fwad.unpack_dual(kv4.rope(fwad.make_dual(x.detach(), other), pos, table)).tangent
    assert torch.equal(t, kv4.rope(other, pos, table))


def test_refusals(env):
    kv4, torch, dev = env
    x, pos, table, g = inputs(env)
    x.requires_grad_()
    with pytest.raises(RuntimeError):
        kv4.rope(x, pos, table, out=torch.empty_like(x))
    with pytest.raises(RuntimeError):
        kv4.rope(x.detach(), pos, table.clone().requires_grad_())
    import torch.autograd.forward_ad as fwad
    with fwad.dual_level():                                                   # (a level alone tracks nothing)
        y = x.detach().clone()
        assert kv4.rope(y, pos, table, out=y) is y
    with torch.no_grad():                                                     # as before
        out = torch.empty_like(x)
        assert kv4.rope(x, pos, table, out=out) is out and np.isfinite(out.cpu().numpy()).all()
