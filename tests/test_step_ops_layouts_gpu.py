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
