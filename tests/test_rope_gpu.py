"""Rotary positions against the formula in 64 bits.

Tolerances: bf16 results are one rounding (2^-9 of the value, rms; 2^-8 at most) from the formula; fp32 ones
have sine and cosine to about 2^-22 and two roundings: 1e-6 of the pair's length."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def plain(x, rope, pos, inverse=False):
    x = x.double()
    y = x.clone()
    h = rope.dim // 2
    ang = pos.double()[..., None] * torch.tensor(rope.angles, dtype=torch.float64, device=x.device)
    c, s = rope.gain * ang.cos()[:, :, None], rope.gain * ang.sin()[:, :, None] * (-1 if inverse else 1)
    ia = torch.arange(0, rope.dim, 2) if rope.interleaved else torch.arange(h)
    ib = ia + 1 if rope.interleaved else ia + h
    a, b = x[..., ia.to(x.device)], x[..., ib.to(x.device)]
    y[..., ia.to(x.device)], y[..., ib.to(x.device)] = a * c - b * s, a * s + b * c
    return y


def close(got, want, dtype, gain):
    scale = want.abs().amax(-1, keepdim=True).clamp_min(1e-30)
    err = float(((got.double() - want).abs() / scale).max())
    assert err <= (1e-6 if dtype == "f32" else 2.0 ** -8) * max(1.0, gain), err


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("shape, rot", [((1, 1, 1, 2), 2), ((2, 3, 5, 64), 64), ((3, 1001, 4, 80), 32), ((2, 77, 3, 50), 18), ((1, 300, 40, 128), 128),
                                        ((4, 1, 7, 96), 96), ((1, 5, 2, 136), 8), ((2, 9, 1, 24), 24)])
def test_turns(dtype, interleaved, inverse, shape, rot):
    from paper_2411_03742_b200 import Rope
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(shape, generator=g, device="cuda").to(TYPES[dtype])
    pos = torch.randint(0, 100_000, shape[:2], generator=g, device="cuda", dtype=torch.int32)
    with Rope(rot, interleaved=interleaved) as rope:
        close(rope.apply(x, pos, inverse=inverse), plain(x, rope, pos, inverse), dtype, 1.0)
        p0 = torch.arange(shape[1], device="cuda").repeat(shape[0], 1) + 11
        close(rope.apply(x, first=11, inverse=inverse), plain(x, rope, p0, inverse), dtype, 1.0)
        y = x.clone()
        rope.apply(y, pos, out=y, inverse=inverse)
        assert torch.equal(y, rope.apply(x, pos, inverse=inverse)), "in place"


@pytest.mark.parametrize("scaling", [("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0, 4096), ("yarn", 4.0, 2048, 16, 2)])
def test_scalings_and_far_positions(scaling):
    """Up to position 2^30 the angle is as exact as in 64 bits."""
    from paper_2411_03742_b200 import Rope
    x = torch.randn((1, 64, 2, 64), device="cuda")
    pos = torch.tensor([[0, 1, 2 ** 20, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1] + list(range(58))], dtype=torch.int32, device="cuda")
    with Rope(64, scaling=scaling) as rope:
        want = plain(x, rope, pos)
        got = rope.apply(x, pos)
        # a 64-bit angle of 2^31 radians has 2^-22 of absolute error itself
        assert float((got.double() - want).abs().max()) <= 4e-6 * 4
        close(got[:, :2], want[:, :2], "f32", rope.gain)


def test_strides_and_slices():
    """Slices of a packed projection, head-major memory, odd offsets: read and written in place."""
    from paper_2411_03742_b200 import Rope
    with Rope(32) as rope:
        for dtype in TYPES.values():
            packed = torch.randn((2, 50, 9, 64), device="cuda").to(dtype)
            keep = packed.clone()
            view = packed[:, :, 1:6]
            rope.apply(view, out=view)
            pos = torch.arange(50, device="cuda").repeat(2, 1)
            close(view, plain(keep[:, :, 1:6], rope, pos), "f32" if dtype == torch.float32 else "bf16", 1.0)
            assert torch.equal(packed[:, :, 0], keep[:, :, 0]) and torch.equal(packed[:, :, 6:], keep[:, :, 6:])
            heads_first = keep.transpose(1, 2).contiguous().transpose(1, 2)
            assert torch.equal(rope.apply(heads_first), rope.apply(keep))
            odd = torch.zeros(2 * 50 * 9 * 64 + 1, dtype=dtype, device="cuda")[1:].view(2, 50, 9, 64)
            odd.copy_(keep)
            assert torch.equal(rope.apply(odd), rope.apply(keep))
            flip = keep[:, :1].expand(2, 50, 9, 64)                    # a broadcast input
            assert torch.equal(rope.apply(flip), rope.apply(flip.contiguous()))


def test_gradient():
    """The gradient is the transposed map: <R x, y> = <x, R^T y>; R^T R = gain^2; differences of a linear map."""
    from paper_2411_03742_b200 import Rope
    with Rope(48, scaling=("yarn", 8.0, 512), interleaved=True) as rope:
        x = torch.randn((2, 33, 3, 64), device="cuda", requires_grad=True)
        y = torch.randn((2, 33, 3, 64), device="cuda")
        pos = torch.randint(0, 4000, (2, 33), device="cuda", dtype=torch.int32)
        out = rope(x, pos)
        (out * y).sum().backward()
        lhs, rhs = float((out.double() * y.double()).sum()), float((x.double() * x.grad.double()).sum())
        assert abs(lhs - rhs) <= 1e-6 * float(x.detach().norm() * y.norm()) * rope.gain
        back = rope.apply(out.detach(), pos, inverse=True)
        want = x.detach().clone()
        want[..., :48] *= rope.gain ** 2
        assert float((back - want).abs().max()) <= 1e-5
        h = torch.randn_like(y)
        d = (plain(x.detach() + h, rope, pos) - plain(x.detach() - h, rope, pos)) / 2
        assert abs(float((d * y.double()).sum()) - float((x.grad.double() * h.double()).sum())) <= 1e-5 * float(h.norm() * y.norm())
        z = x.detach().clone().requires_grad_()
        rope(z, pos).sum().backward()                                  # a broadcast gradient
        assert float((z.grad.double() - plain(torch.ones_like(y), rope, pos, inverse=True)).abs().max()) <= 1e-5


def test_empty_long_and_streams():
    from paper_2411_03742_b200 import Rope
    with Rope(16) as rope:
        for shape in [(0, 4, 2, 16), (2, 0, 2, 16), (2, 4, 0, 16)]:
            assert rope.apply(torch.empty(shape, device="cuda")).shape == shape
        # strides past 32 bits
        far = torch.zeros((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
        x = far.as_strided((2, 3, 2, 16), (1 << 31, 32, 16, 1))
        src = torch.randn((2, 3, 2, 16), device="cuda").bfloat16()
        x.copy_(src)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        rope.apply(x, out=x, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(x, rope.apply(src))


def test_refusals():
    from paper_2411_03742_b200 import Rope
    x = torch.zeros((1, 2, 3, 16), device="cuda")
    with Rope(16) as rope:
        for bad in (x.half(), x[0], x.cpu(), torch.zeros((1, 2, 3, 8), device="cuda")):
            with pytest.raises(ValueError):
                rope.apply(bad)
        with pytest.raises(ValueError):
            rope.apply(x, positions=torch.zeros((1, 2), device="cuda"))
        with pytest.raises(ValueError):
            rope.apply(x, positions=torch.zeros((1, 3), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        Rope(16, angles=[1.0])


def test_second_derivatives():
    """|R y|^2 = gain^2 |y|^2 where all is turned, so the gradient of the gradient's norm through y = x^3 is known."""
    from paper_2411_03742_b200 import Rope
    x = torch.randn((2, 33, 3, 64), device="cuda", dtype=torch.float32, requires_grad=True)
    pos = torch.randint(0, 4000, (2, 33), device="cuda", dtype=torch.int32)
    with Rope(64, scaling=("yarn", 8.0, 512)) as rope:
        g = torch.autograd.grad(rope(x * x * x, pos).square().sum(), x, create_graph=True)[0]
        h = torch.autograd.grad(g.square().sum(), x)[0]
        y = x.detach().double().requires_grad_()
        g2 = torch.autograd.grad(rope.gain ** 2 * (y ** 3).square().sum(), y, create_graph=True)[0]
        want = torch.autograd.grad(g2.square().sum(), y)[0]
    # fp32 throughout: two turns each way at 1e-6 of their pairs
    assert float((h.double() - want).norm() / want.norm()) <= 1e-5


def test_empty_slices():
    """No tokens, no sequences, no heads, in slices of a packed projection; and back through autograd."""
    from paper_2411_03742_b200 import Rope
    with Rope(16) as rope:
        for shape, heads in (((2, 0, 6, 16), 4), ((0, 3, 6, 16), 4), ((2, 3, 6, 16), 0)):
            packed = torch.zeros(shape, device="cuda", requires_grad=True)
            y = rope(packed[:, :, :heads])
            assert y.shape == (*shape[:2], heads, 16)
            y.sum().backward()
            assert packed.grad.shape == shape and not packed.grad.any()
