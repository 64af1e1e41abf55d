"""Layouts that the norms', the feed-forward block's and the distillation's calls take: rows without unit stride in the differentiable form, slices for a few tokens, far offsets, long
batches of rows off 16 bytes; and inference, which keeps nothing for a gradient.

Where a call copies, its results are those of the copy, bit by bit.  Elsewhere the tolerances of test_norms_gpu.py and test_feedforward_gpu.py.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


def randn(*s, seed=0, dtype=torch.bfloat16):
    return torch.randn(s, generator=torch.Generator(device="cuda").manual_seed(seed + sum(s)), device="cuda").to(dtype)


def odd(t, how):
    """t's values, laid out without unit stride along rows."""
    if how == "turned":
        return t.transpose(-1, -2).contiguous().transpose(-1, -2) if t.dim() > 1 else torch.stack([t, t], -1)[..., 0]
    return torch.stack([t, t + 1], -1).flatten(-2)[..., ::2]


@pytest.mark.parametrize("how", ["turned", "stepped"])
@pytest.mark.parametrize("gate_shape", [(72,), (3, 72), (3, 20, 72)])
def test_norms_copy_rows_without_unit_stride(how, gate_shape):
    from paper_2411_03742_b200 import residual_norm
    base = [randn(3, 20, 72, dtype=torch.float32), randn(3, 20, 72, seed=1), randn(*gate_shape, seed=2), randn(72, seed=3, dtype=torch.float32), randn(72, seed=4, dtype=torch.float32)]
    douts = randn(3, 20, 72, seed=5, dtype=torch.float32), randn(3, 20, 72, seed=6)

    def step(tensors):
        leaves = [t.detach().requires_grad_() for t in tensors]
        x, f, gate, post, pre = leaves
        out = residual_norm(x, f, gate=gate, gate_by="tanh", post=post, scale=0.5, pre=pre)
        return (*out, *torch.autograd.grad(out, leaves, douts))

    want = step(base)
    for k in range(5):
        got = step([odd(t, how) if i == k else t for i, t in enumerate(base)])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
    assert all(torch.equal(a, b) for a, b in zip(step([odd(t, how) for t in base]), want))
    x = odd(base[0], how).requires_grad_()             # without f the stream passes through as it is
    same, h = residual_norm(x, pre=base[4], dtype=torch.bfloat16)
    assert same is x and torch.equal(h, residual_norm(base[0], pre=base[4], dtype=torch.bfloat16)[1])
    g1, = torch.autograd.grad(h, x, douts[1])
    plain = base[0].clone().requires_grad_()
    g2, = torch.autograd.grad(residual_norm(plain, pre=base[4], dtype=torch.bfloat16)[1], plain, douts[1])
    assert torch.equal(g1, g2)


def test_norms_take_one_gate_value_a_token():
    """A gate of one value for each token or sequence, broadcast over its row: the gradient is the sum over the row, as torch has it."""
    from paper_2411_03742_b200 import residual_norm
    x, f = randn(3, 20, 72, dtype=torch.float32), randn(3, 20, 72, seed=1)
    for shape in ((3, 20, 1), (3, 1)):
        gate = randn(*shape, seed=2, dtype=torch.float32).requires_grad_()
        wide = gate.detach().expand(*shape[:-1], 72).contiguous().requires_grad_()
        outs = [residual_norm(x, f, gate=g, gate_by="sigmoid")[0] for g in (gate.expand(*shape[:-1], 72), wide)]
        assert torch.equal(*outs)
        dout = randn(3, 20, 72, seed=5, dtype=torch.float32)
        (a,), (b,) = (torch.autograd.grad(o, g, dout) for o, g in zip(outs, (gate, wide)))
        assert a.shape == shape and torch.equal(a, b.sum(-1, keepdim=True))


def test_inference_keeps_nothing():
    """Without gradients neither gate nor up is made, whether or not the weights are parameters."""
    from paper_2411_03742_b200 import gated_feedforward
    T, D, F = 4096, 64, 2048
    x, wg, wu, wd = randn(T, D), randn(F, D, seed=1), randn(F, D, seed=2), randn(D, F, seed=3)
    want = gated_feedforward(x, wg, wu, wd)
    weights = [torch.nn.Parameter(w) for w in (wg, wu, wd)]
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            torch.cuda.synchronize()
            torch.cuda.reset_peak_memory_stats()
            before = torch.cuda.memory_allocated()
            got = gated_feedforward(x, *weights)
            used = torch.cuda.max_memory_allocated() - before
        assert torch.equal(got, want) and not got.requires_grad
        # the result and one matrix (token, hidden) of working memory, and the allocator's rounding
        assert used <= 2 * T * D + 2 * T * F + (1 << 21), used
    y = gated_feedforward(x, *weights)
    assert y.requires_grad and torch.equal(y, want)
    y.sum().backward()
    assert all(w.grad is not None for w in weights)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T, D, F", [(1, 1024, 4096), (7, 520, 1368), (16, 128, 384), (17, 264, 520), (32, 1024, 512)])
def test_a_few_tokens_from_and_into_slices(T, D, F, dtype):
    from paper_2411_03742_b200 import feedforward_forward
    from test_feedforward_gpu import check, make
    inputs, dout = make(T, D, F, dtype, wide=24)
    made, _ = check(T, D, F, dtype=dtype, given=(inputs, dout))
    rooms = [torch.full((m + 2, n + 16), 7.0, dtype=dtype, device="cuda") for m, n in ((T, D), (T, F), (T, F))]
    spots = [r[1:-1, 8:-8] for r in rooms]
    feedforward_forward(*inputs, out=spots[0], gate=spots[1], up=spots[2])
    for r, spot, want in zip(rooms, spots, made):
        assert torch.equal(spot, want)
        spot.fill_(7.0)
        assert bool((r == 7).all())


@pytest.mark.parametrize("T", [3, 200])
def test_feedforward_far_offsets(T):
    """Tokens beyond 2^31 elements from where their matrix starts, read and written."""
    from paper_2411_03742_b200 import feedforward_backward, feedforward_forward
    from test_feedforward_gpu import make
    (x, wg, wu, wd), dout = make(T, 64, 136)
    apart = (2 ** 31 // (T - 1) + 64) // 64 * 64
    big = torch.empty(apart * (T - 1) + 4096, dtype=torch.bfloat16, device="cuda")
    far = lambda n, at: torch.as_strided(big, (T, n), (apart, 1), at)  # noqa: E731
    want = feedforward_forward(x, wg, wu, wd)
    grads = feedforward_backward(dout, x, wg, wu, wd, want[1], want[2])
    spots = [far(64, 0), far(64, 64), far(136, 128), far(136, 264), far(64, 400), far(64, 464)]
    spots[0].copy_(x)
    spots[4].copy_(dout)
    feedforward_forward(spots[0], wg, wu, wd, out=spots[1], gate=spots[2], up=spots[3])
    assert all(torch.equal(a, b) for a, b in zip(spots[1:4], want))
    got = feedforward_backward(spots[4], spots[0], wg, wu, wd, spots[2], spots[3], dx=spots[5])
    assert all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B, S, D, wide", [(2, 1500, 1001, 0), (3, 900, 4096, 13), (1, 2500, 513, 8), (2, 700, 4097, 0)])
def test_norms_of_many_rows_off_16_bytes(B, S, D, wide, dtype):
    """Long batches of rows of odd widths, or whose stride is odd."""
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    from test_norms_gpu import F32, TYPES, plain_backward, plain_forward
    t = TYPES[dtype]
    r = lambda seed, dt: randn(B, S, D + wide, seed=seed, dtype=dt)[..., :D]  # noqa: E731
    x, f, post, pre, gate = r(0, torch.float32), r(1, t), 1 + 0.2 * randn(D, seed=2, dtype=torch.float32), 1 + 0.2 * randn(D, seed=3, dtype=torch.float32), randn(D, seed=4, dtype=torch.float32)
    how = dict(gate=gate, gate_by="sigmoid", post=post, scale=0.5, pre=pre)
    out, normed, rows = residual_norm_forward(x, f, **how)
    want = plain_forward(x, f, gate, "sigmoid", post, 0.5, pre, 1e-6)
    u = lambda v: torch.finfo(v.dtype).eps / 2  # noqa: E731
    for got, value, size in ((out, want[0], want[3]), (normed, want[1], want[4])):
        assert bool(((got.double() - value).abs() <= u(got) * value.abs() + F32 * size + torch.finfo(got.dtype).smallest_normal * 2 * u(got)).all())
    dout, dnormed = r(5, torch.float32), r(6, t)
    grads = residual_norm_backward(dout, dnormed, out, f, rows, **how)
    wants, sizes = plain_backward(dout, dnormed, out, f, rows, gate, "sigmoid", post, 0.5, pre)
    # sums over B S tokens: chains of at most B S / 148 + 32 additions with trees beside them
    for k, (got, value, size) in enumerate(zip(grads, wants, sizes)):
        more = 2.0 ** -24 * (B * S / 148 + 64) if k > 1 else 0.0
        assert bool(((got.double() - value).abs() <= u(got) * value.abs() + (F32 + more) * size + torch.finfo(got.dtype).smallest_normal * 2 * u(got)).all()), k


def test_status_words_are_read_by_one_caller():
    """A wait that expires while another stream looks at the status again and again is told once, to whoever looks next."""
    from paper_2411_03742_b200 import feedforward
    x, w = randn(100, 128), randn(64, 128, seed=1)
    assert feedforward.status() == 0
    work, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(work):
        feedforward.selftest_bounded_wait(x, w, w, False)
    seen = []
    while not work.query():
        seen.append(feedforward.status(side))
    work.synchronize()
    seen.append(feedforward.status(side))
    assert [v for v in seen if v] == [0x100] and feedforward.status() == 0
