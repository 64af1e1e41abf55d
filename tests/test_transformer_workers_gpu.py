"""The example that runs the operators together: gradients of N workers through rotary positions and attention,
aggregation, orthogonalised updates."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_loss_falls():
    from paper_2411_03742_b200.examples.transformer_workers import run
    losses = run(workers=4, size=8, length=64, steps=40)
    assert all(math.isfinite(x) for x in losses)
    # from the uniform guess over 61 tokens (ln 61 = 4.1) to well under half of it
    assert losses[0] > 3.0 and sum(losses[-5:]) / 5 < 0.5 * losses[0], losses


def test_gradients_match_plain_attention():
    """One worker's gradient against the same model with rotary positions and attention in plain fp32 torch."""
    from paper_2411_03742_b200.examples import transformer_workers as tw
    model = tw.Model(61)
    tokens = tw.batch(1, 4, 50, 61, torch.Generator().manual_seed(3), "cuda:0")[0]
    got, = torch.autograd.grad(model.loss(tokens), model.flat)

    def plain_attention(q, k, v, causal):
        r = q.shape[2] // k.shape[2]
        q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
        k, v = k.repeat_interleave(r, 1), v.repeat_interleave(r, 1)
        s = q @ k.mT / math.sqrt(q.shape[-1])
        S = s.shape[-1]
        s = s.masked_fill(torch.ones(S, S, dtype=torch.bool, device=s.device).triu(1), -math.inf)
        return (s.softmax(-1) @ v).transpose(1, 2).bfloat16()

    class PlainRope:
        def __init__(self, rope):
            self.angles = torch.tensor(rope.angles, device="cuda:0")

        def __call__(self, x):
            t = torch.arange(x.shape[1], device=x.device)[:, None].double() * self.angles
            c, s = t.cos().float()[None, :, None], t.sin().float()[None, :, None]
            a, b = x.float().chunk(2, -1)
            return torch.cat((a * c - b * s, a * s + b * c), -1).to(x.dtype)

    keep = tw.attention
    try:
        tw.attention, model.rope = plain_attention, PlainRope(model.rope)
        want, = torch.autograd.grad(model.loss(tokens), model.flat)
    finally:
        tw.attention = keep
    # both run the projections in bf16: 2^-8 per rounding, a dozen roundings deep
    assert float((got - want).norm() / want.norm()) <= 2e-2
