"""The example's gated model and its teacher: norms, attention, feed-forward blocks, distillation, aggregation and orthogonalised updates in one run, and
a worker's gradient against the same model with the operators' formulas in fp32."""
import math

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu


def test_runs_and_changes_its_parameters():
    from paper_2411_03742_b200.examples import transformer_workers as tw
    teacher = tw.GatedModel(61, seed=4)
    before = teacher.flat.detach().clone()
    losses = tw.run(workers=3, size=4, length=33, steps=3, model=teacher)
    assert all(math.isfinite(v) for v in losses)
    assert (teacher.flat.detach() != before).float().mean() > 0.9
    student = tw.GatedModel(61, seed=5)
    losses = tw.run(workers=3, size=4, length=33, steps=3, model=student, teacher=teacher, top=5)
    assert all(math.isfinite(v) for v in losses)
    assert not torch.equal(student.flat.detach(), tw.GatedModel(61, seed=5).flat.detach())
    # the plain model learns from a teacher as well
    assert math.isfinite(tw.run(workers=2, size=2, length=20, steps=1, teacher=teacher, top=61)[0])


@pytest.mark.parametrize("taught", [False, True])
def test_gradients_match_plain_operations(taught, monkeypatch):
    from paper_2411_03742_b200.examples import transformer_workers as tw
    model = tw.GatedModel(61)
    tokens = tw.batch(1, 4, 50, 61, torch.Generator().manual_seed(3), "cuda:0")[0]
    teacher = tw.GatedModel(61, seed=9).top_logits(tokens, 6) if taught else None
    got, = torch.autograd.grad(model.loss(tokens, teacher), model.flat)

    def plain_attention(q, k, v, causal):
        r = q.shape[2] // k.shape[2]
        q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
        k, v = k.repeat_interleave(r, 1), v.repeat_interleave(r, 1)
        s = q @ k.mT / math.sqrt(q.shape[-1])
        S = s.shape[-1]
        s = s.masked_fill(torch.ones(S, S, dtype=torch.bool, device=s.device).triu(1), -math.inf)
        return (s.softmax(-1) @ v).transpose(1, 2).bfloat16()

    def plain_norm(x, f=None, *, post=None, gate=None, gate_by=None, pre=None, dtype=None):
        norm = lambda t, w: t.float() * (t.float().square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w  # noqa: E731
        if f is not None:
            x = x + torch.sigmoid(gate) * norm(f, post)
        return x, norm(x, pre).to(torch.bfloat16)

    def plain_feedforward(x, wg, wu, wd, act):
        x, wg, wu, wd = (t.float() for t in (x, wg, wu, wd))
        return ((F.silu(x @ wg.T) * (x @ wu.T)) @ wd.T).bfloat16()

    def plain_distill(z, ids, top, *, temperature, labels, mix):
        p = (top / temperature).softmax(-1)
        kl = (p * (p.log() - (z / temperature).log_softmax(-1).gather(1, ids))).sum(-1)
        return mix * temperature ** 2 * kl + (1 - mix) * F.cross_entropy(z, labels, reduction="none")

    class PlainRope:
        def __init__(self, rope):
            self.angles = torch.tensor(rope.angles, device="cuda:0")

        def __call__(self, x):
            t = torch.arange(x.shape[1], device=x.device)[:, None].double() * self.angles
            c, s = t.cos().float()[None, :, None], t.sin().float()[None, :, None]
            a, b = x.float().chunk(2, -1)
            return torch.cat((a * c - b * s, a * s + b * c), -1).to(x.dtype)

    for name, f in (("attention", plain_attention), ("residual_norm", plain_norm), ("gated_feedforward", plain_feedforward), ("distill", plain_distill)):
        monkeypatch.setattr(tw, name, f)
    model.rope = PlainRope(model.rope)
    want, = torch.autograd.grad(model.loss(tokens, teacher), model.flat)
    # both run the products in bf16: 2^-8 per rounding, two dozen roundings deep, independent: sqrt(24) * 0.43 * 2^-8, taken twice
    assert float((got - want).norm() / want.norm()) <= 2 * math.sqrt(24) * 0.43 * 2.0 ** -8


def test_a_captured_step():
    """The step's gradient captured into a graph and replayed on other tokens.  (No eager graph of the same leaves may live meanwhile: torch's autograd would
    wait for the stream of its leaves' nodes, which a capture forbids.)"""
    from paper_2411_03742_b200.examples import transformer_workers as tw
    model = tw.GatedModel(61)
    draw = lambda seed: tw.batch(1, 2, 24, 61, torch.Generator().manual_seed(seed), "cuda:0")[0]  # noqa: E731
    tokens, other = draw(3), draw(4)
    ids, top = tw.GatedModel(61, seed=9).top_logits(tokens, 6)
    ids2, top2 = tw.GatedModel(61, seed=9).top_logits(other, 6)
    want, = torch.autograd.grad(model.loss(other, (ids2, top2)), model.flat)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(model.loss(tokens, (ids, top)), model.flat)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(model.loss(tokens, (ids, top)), model.flat)
    for a, b in ((tokens, other), (ids, ids2), (top, top2)):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    # the embedding's gradient is a library sum in fp32 whose order may vary
    assert float((got - want).norm() / want.norm()) <= 1e-5
