"""Distillation from top logits against the formula in 64 bits.

Tolerances.  An exponential is good to 2^-21 of itself plus 2^-23 of its argument's parts (z / tau and the log-sum-exp), a sum over the vocabulary to
2^-20 more: rows to 4e-6 (1 + |L|), a loss to 4e-6 of its terms by magnitude, a gradient to 2^-21 (8 + |z / tau| + |L|) of its terms' magnitudes and half a
step of its type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def plain(z, ids, top, tau, labels=None, mix=1.0):
    """(loss, rows, per-token size of the loss' terms, dz for dloss = 1, sizes of dz), one token at a time."""
    T, V = z.shape
    losses, rows, sizes, grads, grad_sizes = [], [], [], [], []
    for r in range(T):
        zr = z[r].double()
        kept = [j for j in range(ids.shape[1]) if 0 <= int(ids[r, j]) < V and float(top[r, j]) != -math.inf]
        y = -1 if labels is None or not 0 <= int(labels[r]) < V else int(labels[r])
        zero = torch.zeros((), dtype=torch.float64, device=z.device)
        loss = size = L = L1 = zero
        grad, grad_size = torch.zeros_like(zr), torch.zeros_like(zr)
        if kept or y >= 0:
            L, L1 = torch.logsumexp(zr / tau, 0), torch.logsumexp(zr, 0) if labels is not None else zero
        if kept:
            at = ids[r, kept].long()
            logp = torch.log_softmax(top[r, kept].double() / tau, 0)
            p, there = logp.exp(), zr[at] / tau
            terms = torch.where(p > 0, p * (logp - there + L), torch.zeros_like(p))
            loss = loss + mix * tau ** 2 * terms.sum()
            size = size + mix * tau ** 2 * torch.where(p > 0, p * (logp.abs() + there.abs() + L.abs() + 1), torch.zeros_like(p)).sum()
            q = (zr / tau - L).exp()
            grad = grad + mix * tau * (q - torch.zeros_like(q).index_add_(0, at, p))
            grad_size = grad_size + mix * tau * (q + torch.zeros_like(q).index_add_(0, at, p)) * (8 + torch.where(zr.isinf(), zero, zr.abs() / tau) + L.abs())
        if y >= 0:
            loss = loss + (1 - mix) * (L1 - zr[y])
            size = size + (1 - mix) * (L1.abs() + zr[y].abs() + 1)
            q = (zr - L1).exp()
            grad = grad + (1 - mix) * q
            grad_size = grad_size + (1 - mix) * q * (8 + torch.where(zr.isinf(), zero, zr.abs()) + L1.abs())
            grad[y] -= 1 - mix
            grad_size[y] += 1 - mix
        losses.append(loss), rows.append(torch.stack([L, L1])), sizes.append(size), grads.append(grad), grad_sizes.append(grad_size)
    stack = lambda v: torch.stack(v) if v else torch.zeros((0,), dtype=torch.float64, device=z.device)  # noqa: E731
    return stack(losses), stack(rows).T if rows else torch.zeros((2, 0), dtype=torch.float64, device=z.device), stack(sizes), stack(grads), stack(grad_sizes)


def check(z, ids, top, tau, labels=None, mix=None):
    from paper_2411_03742_b200 import distill_backward, distill_forward
    loss, rows = distill_forward(z, ids, top, temperature=tau, labels=labels, mix=mix)
    m = 1.0 if mix is None else mix
    want, want_rows, size, grad, grad_size = plain(z, ids, top, tau, labels, m)
    assert bool(((loss.double() - want).abs() <= 4e-6 * size + 1e-30).all()), float((loss.double() - want).abs().max())
    assert bool(((rows.double() - want_rows).abs() <= 4e-6 * (1 + want_rows.abs())).all())
    dloss = torch.rand(z.shape[0], generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") + 0.5       # the same at every call
    dz = distill_backward(dloss, z, ids, top, rows, temperature=tau, labels=labels, mix=mix)
    assert dz.shape == z.shape and dz.dtype == z.dtype
    u = torch.finfo(z.dtype).eps / 2
    # a step among the smallest numbers of a 16-bit type; exponentials below fp32's smallest normal number, 2^-126, count as 0
    least = torch.finfo(z.dtype).smallest_normal * (1.0 if z.dtype == torch.float32 else torch.finfo(z.dtype).eps)
    w = dloss.double()[:, None]
    bad = (dz.double() - w * grad).abs() > u * (w * grad).abs() + 2.0 ** -21 * w * grad_size + least
    assert not bool(bad.any()), (int(bad.sum()), float((dz.double() - w * grad).abs().max()))
    return loss, rows, dz


def make(T, V, K, dtype="f32", labels=False, wide=0, ids=torch.int64, seed=0, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (scale * torch.randn((T, V + wide), generator=g, device="cuda")).to(TYPES[dtype])[:, :V]
    full = 0.5 * z.float() + 2 * torch.randn((T, V), generator=g, device="cuda")
    top, at = full.topk(K)
    return z, at.to(ids), top, torch.randint(0, V, (T,), generator=g, device="cuda").to(ids) if labels else None


@pytest.mark.parametrize("tau, mix", [(1.0, None), (2.0, None), (1.0, 0.6), (2.0, 0.6), (3.0, 0.5), (4.0, 0.9), (1.7, 0.3), (0.5, 0.0), (2.5, 1.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V, K", [(5, 333, 7), (3, 9001, 64)])
def test_against_the_formula(tau, mix, dtype, T, V, K):
    z, ids, top, labels = make(T, V, K, dtype, mix is not None)
    check(z, ids, top, tau, labels, mix)


@pytest.mark.parametrize("T, V, K", [(1, 1, 1), (1, 2, 2), (2, 7, 7), (9, 64, 1), (4, 1025, 5), (2, 8193, 100), (1, 50021, 32), (19, 50021, 32), (1, 131072, 128), (2, 2048, 1024), (3, 700, 513)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes(T, V, K, dtype):
    """One token to a few, a vocabulary of one to a long one shared between blocks, all of it as entries."""
    z, ids, top, labels = make(T, V, K, dtype, True)
    check(z, ids, top, 2.0, labels, 0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [1, 8, 71])
def test_padded_rows_and_types_of_indices(dtype, wide):
    z, ids, top, labels = make(6, 1003, 20, dtype, True, wide, torch.int32)
    first = check(z, ids, top, 2.0, labels, 0.5)
    again = check(z.contiguous(), ids.long(), top, 2.0, labels.long(), 0.5)
    # a row's start relative to 16 bytes decides which thread adds what: the same values to rounding, not the same bits
    assert torch.allclose(first[0], again[0], rtol=1e-5, atol=1e-6)
    low = top.to(torch.bfloat16)
    check(z, ids, low, 2.0, labels, 0.5)
    packed = torch.stack([ids, ids], 1)[:, 0], torch.stack([top, top], 1)[:, 1]          # rows apart
    check(z, *packed, 2.0, labels, 0.5)


def test_entries_that_are_not_there():
    z, ids, top, labels = make(8, 600, 12, "bf16", True)
    ids[0] = -1                                        # no teacher
    ids[1, 3:] = -100
    ids[2, ::2] = 600                                  # outside
    top[3, 4:] = -math.inf
    top[4] = -math.inf                                 # as none
    labels[4], labels[5] = -100, 600
    ids[6], labels[6] = -1, -1
    ids[7, :] = 2 ** 40
    top[1, 0] = -3.4e38                                # the type's lowest: there, with probability 0
    loss, rows, dz = check(z, ids, top, 2.0, labels, 0.4)
    assert float(loss[6]) == 0 and not dz[6].any() and not rows[:, 6].any() and float(loss[4]) == 0 and not dz[4].any()
    z[6] = math.nan                                    # a padding token's logits are not read
    loss2, rows2, dz2 = check(z, ids, top, 2.0, labels, 0.4)
    assert torch.equal(loss, loss2) and torch.equal(dz, dz2)
    check(z[:5], ids[:5], top[:5], 2.0)


def test_the_same_index_twice():
    z, ids, top, labels = make(4, 90, 10, "f32", True)
    ids[0, 5] = ids[0, 0]
    ids[1, :] = 17
    ids[2, 3] = ids[2, 4] = ids[2, 9] = labels[2]
    check(z, ids, top, 2.0, labels, 0.6)


def test_masked_and_extreme_logits():
    """Logits of -inf and of the type's lowest value; far larger and smaller ones; only one that is not masked."""
    for dtype in ("f32", "bf16", "f16"):
        z, ids, top, labels = make(5, 400, 6, dtype, True)
        seen = torch.zeros_like(z, dtype=torch.bool)
        seen.scatter_(1, ids, True)
        seen.scatter_(1, labels[:, None], True)
        z[0, ~seen[0]] = -math.inf
        z[1, ~seen[1]] = torch.finfo(z.dtype).min
        z[2] *= 100
        z[3] *= 1e-3
        z[4, 0] = 60000.0 if dtype == "f16" else 1e5
        for tau, mix in ((1.0, 0.5), (2.0, 0.5), (1.3, 0.5)):
            check(z, ids, top, tau, labels, mix)
    z = torch.full((1, 50), -math.inf, device="cuda")
    z[0, 9] = 3.0
    check(z, torch.tensor([[9]], device="cuda"), torch.zeros((1, 1), device="cuda"), 2.0)


def test_nan_and_infinity_stay_in_their_token():
    from paper_2411_03742_b200 import distill_backward, distill_forward
    z, ids, top, _ = make(6, 3000, 8, "bf16")
    want = distill_forward(z, ids, top, temperature=2.0)
    bad = z.clone()
    bad[1, 77], bad[4, 5] = math.nan, math.inf
    loss, rows = distill_forward(bad, ids, top, temperature=2.0)
    keep = [0, 2, 3, 5]
    assert torch.equal(loss[keep], want[0][keep]) and torch.equal(rows[:, keep], want[1][:, keep]) and loss[[1, 4]].isnan().all()
    one = torch.ones(6, device="cuda")
    dz, ref = distill_backward(one, bad, ids, top, rows, temperature=2.0), distill_backward(one, z, ids, top, want[1], temperature=2.0)
    assert torch.equal(dz[keep], ref[keep]) and dz[[1, 4]].isnan().any(1).all()


def test_in_place_and_given_results():
    from paper_2411_03742_b200 import distill_backward, distill_forward
    for dtype, V in (("bf16", 4096), ("f32", 20011)):
        z, ids, top, labels = make(3, V, 16, dtype, True)
        how = {"temperature": 2.0, "labels": labels, "mix": 0.5}
        loss, rows = distill_forward(z, ids, top, **how)
        mine = torch.empty_like(loss), torch.empty_like(rows)
        got = distill_forward(z, ids, top, loss=mine[0], rows=mine[1], **how)
        assert got[0] is mine[0] and torch.equal(loss, mine[0]) and torch.equal(rows, mine[1])
        dloss = torch.rand(3, device="cuda")
        want = distill_backward(dloss, z, ids, top, rows, **how)
        for out in (torch.empty((3, V + 3), dtype=z.dtype, device="cuda")[:, :V], z.clone()):
            logits = out if out.is_contiguous() else z
            if logits is out:
                assert torch.equal(distill_backward(dloss, out, ids, top, rows, out=out, **how), want)
            else:
                assert torch.equal(distill_backward(dloss, z, ids, top, rows, out=out, **how), want)


def test_no_tokens_and_one_gradient_for_all():
    from paper_2411_03742_b200 import distill, distill_backward, distill_forward
    z, ids, top, _ = make(4, 100, 5)
    loss, rows = distill_forward(z[:0], ids[:0], top[:0])
    assert loss.shape == (0,) and rows.shape == (2, 0)
    assert distill_backward(loss, z[:0], ids[:0], top[:0], rows).shape == (0, 100)
    leaf = z.clone().requires_grad_()
    distill(leaf, ids, top, temperature=2.0).sum().backward()                            # autograd hands on one expanded value
    rows = distill_forward(z, ids, top, temperature=2.0)[1]
    assert torch.equal(leaf.grad, distill_backward(torch.ones(4, device="cuda"), z, ids, top, rows, temperature=2.0))


def test_autograd_and_differences():
    from paper_2411_03742_b200 import distill
    z, ids, top, labels = make(4, 150, 9, "f32", True)
    leaf = z.clone().requires_grad_()
    weight = torch.rand(4, device="cuda")
    g, = torch.autograd.grad((distill(leaf, ids, top, temperature=2.0, labels=labels, mix=0.6) * weight).sum(), leaf)
    Z = z.double().requires_grad_()
    p = torch.softmax(top.double() / 2, 1)
    logq = torch.log_softmax(Z / 2, 1).gather(1, ids)
    loss = 0.6 * 4 * (p * (p.log() - logq)).sum(1) + 0.4 * torch.nn.functional.cross_entropy(Z, labels, reduction="none")
    want, = torch.autograd.grad((loss * weight.double()).sum(), Z)
    assert float((g.double() - want).norm() / want.norm()) <= 2e-6
    d = torch.randn_like(z).double()
    d = d / d.norm()
    f = lambda s: float((plain(z.double() + s * d, ids, top, 2.0, labels, 0.6)[0] * weight.double()).sum())  # noqa: E731
    assert abs((f(1e-4) - f(-1e-4)) / 2e-4 - float((g.double() * d).sum())) <= 1e-6
    with pytest.raises(NotImplementedError, match="once"):
        one, = torch.autograd.grad(distill(leaf, ids, top).sum(), leaf, create_graph=True)
        torch.autograd.grad(one.sum(), leaf)


def test_repeats_graphs_and_streams():
    from paper_2411_03742_b200 import distill_backward, distill_forward
    z, ids, top, labels = make(19, 50021, 32, "bf16", True)
    how = {"temperature": 2.0, "labels": labels, "mix": 0.5}
    dloss = torch.rand(19, device="cuda")

    def step(stream=None):
        loss, rows = distill_forward(z, ids, top, stream=stream, **how)
        return loss, rows, distill_backward(dloss, z, ids, top, rows, stream=stream, **how)

    want = step()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    keep = z.clone()
    z.zero_()
    g.replay()
    z.copy_(keep)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = step(side)
    rubbish = [torch.full((19 * 50021,), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del rubbish


def test_far_offsets():
    """Tokens beyond 2^31 elements from the matrix' start."""
    from paper_2411_03742_b200 import distill_backward, distill_forward
    big = torch.empty(2 ** 31 + 2 ** 17, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(big, (2, 3000), (2 ** 31, 1))
    z.copy_(torch.randn((2, 3000), device="cuda"))
    _, ids, top, _ = make(2, 3000, 9)
    loss, rows = distill_forward(z, ids, top)
    want, want_rows = distill_forward(z.contiguous(), ids, top)
    assert torch.equal(loss, want) and torch.equal(rows, want_rows)
    one = torch.ones(2, device="cuda")
    dz = distill_backward(one, z.contiguous(), ids, top, rows)
    assert torch.equal(distill_backward(one, z, ids, top, rows, out=z), dz)
