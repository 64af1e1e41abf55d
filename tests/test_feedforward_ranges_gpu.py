"""What float16 holds between the products of the feed-forward block's gradient: dg = dh u act'(g) and du = dh act(g), times a power of two 2^k.

k is 0, or brings dy's largest element to [1/2, 1) where it is smaller; it is less only where the largest of dg and du would round to infinity, and then by as
little as keeps it finite.  So nothing is held with fewer bits than without a factor, unless that would be infinite.

Tolerances.  u = 2^-11 is the largest relative error of a rounding, 2^-25 the largest below 2^-14: an element of dg or du is held to u of itself plus 2^-25 2^-k.  Sums in fp32 take
2^-13 of the products by magnitude, the activation's approximation 4e-7 of its parts.  Token by token, in the 2-norm: independent roundings of 0.43 u each make
0.6 u, u is allowed; the 2^-25 2^-k of every element go through a row of each weight.
"""
import math

import pytest
import torch
import torch.nn.functional as fn

pytestmark = pytest.mark.gpu
U, STEP = 2.0 ** -11, 2.0 ** -25
SHAPES = [(64, 256, 512), (231, 520, 1368), (900, 512, 1024), (600, 64, 200)]       # shared K, lone blocks, pairs


def make(T, D, F, seed=0, dy=1.0, up=1.0, gate=1.0, down=1.0, weights=1.0, x=1.0):
    """Inputs of the backward pass, each as large as is said."""
    g = torch.Generator(device="cuda").manual_seed(seed + T)
    r = lambda m, n, s: (s * torch.randn((m, n), generator=g, device="cuda")).half()  # noqa: E731
    return {"x": r(T, D, x), "w_gate": r(F, D, weights * D ** -0.5), "w_up": r(F, D, weights * D ** -0.5), "w_down": r(D, F, down * F ** -0.5), "gate": r(T, F, gate),
            "up": r(T, F, up), "dout": r(T, D, dy)}


def formula(i):
    """The four gradients in 64 bits, with the magnitudes that errors go by, and k."""
    X, G, W, Dn, g, p, dy = (i[n].double() for n in ("x", "w_gate", "w_up", "w_down", "gate", "up", "dout"))
    s = torch.sigmoid(g)
    a, slope = g * s, s * (1 + g * (1 - s))
    dh, dh_size = dy @ Dn, dy.abs() @ Dn.abs()
    dg, du, h = dh * p * slope, dh * a, a * p
    top = float(dy.abs().max())
    k = 0 if top >= 0.5 or top == 0 else -1 - math.floor(math.log2(top))
    largest = max(float(dg.abs().max()), float(du.abs().max())) * 2.0 ** k
    if largest >= 65520:
        k -= next(n for n in range(1, 200) if largest * 2.0 ** -n < 65520)
    held = STEP * 2.0 ** -k
    near = U + 2.0 ** -13
    dg_size = near * dg.abs() + 2.0 ** -13 * dh_size * (p * slope).abs() + 4e-7 * dh_size * p.abs() * (1 + g.abs()) + held
    du_size = near * du.abs() + 2.0 ** -13 * dh_size * a.abs() + 4e-7 * dh_size * g.abs() + held
    h_size = near * h.abs() + 2e-7 * (g * p).abs() + STEP
    wants = (dg @ G + du @ W, dg.T @ X, du.T @ X, dy.T @ h)
    sizes = (dg_size @ G.abs() + du_size @ W.abs(), dg_size.T @ X.abs(), du_size.T @ X.abs(), dy.abs().T @ h_size)
    sums = (dg.abs() @ G.abs() + du.abs() @ W.abs(), dg.abs().T @ X.abs(), du.abs().T @ X.abs(), dy.abs().T @ h.abs())
    through = held * (float(G.norm()) + float(W.norm()))
    return wants, [a + 2.0 ** -13 * b + STEP for a, b in zip(sizes, sums)], k, through


def check(i, workspace=None, want_k=None):
    from paper_2411_03742_b200 import feedforward, feedforward_backward
    args = [i[n] for n in ("dout", "x", "w_gate", "w_up", "w_down", "gate", "up")]
    got = feedforward_backward(*args, workspace=workspace)
    wants, sizes, k, through = formula(i)
    assert want_k is None or want_k(k), k
    for name, a, b, size in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, wants, sizes):
        assert float(b.abs().max()) < 65504 and bool(a.isfinite().all()), name
        diff = (a.double() - b).abs()
        assert not bool((diff > U * b.abs() + size).any()), (name, k, float(diff.max()))
    diff, size = (got[0].double() - wants[0]).norm(dim=1), wants[0].norm(dim=1)
    allowed = U * size + through + STEP * math.sqrt(wants[0].shape[1])
    assert not bool((diff > allowed).any()), (k, float((diff / size).max()), int((diff > allowed).sum()))
    assert feedforward.status() == 0
    return got


@pytest.mark.parametrize("T, D, F", SHAPES)
@pytest.mark.parametrize("beside", [30.0, 300.0, 3000.0])
def test_small_tokens_beside_a_large_one(T, D, F, beside):
    """One token of a batch with a far larger gradient: the others keep their bits."""
    i = make(T, D, F, dy=1e-3, gate=0.3, x=0.1)
    i["dout"][T // 3] *= beside / 1e-3
    check(i, want_k=lambda k: k == 0)


@pytest.mark.parametrize("T, D, F", SHAPES)
@pytest.mark.parametrize("dy, up, gate", [(1e-5, 1.2e4, 0.3), (1e-5, 0.3, 1.2e4), (1e-6, 1.2e4, 0.3), (1e-7, 6e3, 0.3)])
def test_large_factors_on_small_gradients(T, D, F, dy, up, gate):
    """dg and du are far larger than dy, beyond the range if dy were brought near 1, but not without a factor or with a smaller one."""
    check(make(T, D, F, dy=dy, up=up, gate=gate, down=16.0), want_k=lambda k: k >= 0)


@pytest.mark.parametrize("T, D, F", SHAPES)
@pytest.mark.parametrize("dy, up, down, gate, x", [(3000.0, 100.0, 1.0, 1e-3, 1e-3), (1.0, 1.2e4, 8.0, 1e-3, 1e-3), (1e4, 1e3, 1.0, 1e-5, 1e-5)])
def test_results_in_range_of_operands_beyond_it(T, D, F, dy, up, down, gate, x):
    """dg would be infinite without a factor, the gradients that it leads to are not."""
    check(make(T, D, F, dy=dy, up=up, down=down, gate=gate, weights=1e-4, x=x), want_k=lambda k: k < 0)


@pytest.mark.parametrize("T, D, F", SHAPES)
def test_one_workspace_for_calls_of_every_kind(T, D, F):
    """What a call leaves in its workspace, or what was there before, does not reach the next one; results repeat bit by bit, in graphs and by parts."""
    from paper_2411_03742_b200 import feedforward, feedforward_backward
    calm, wild = make(T, D, F, dy=0.1), make(T, D, F, seed=1, dy=3000.0, up=100.0, gate=1e-3, weights=1e-4, x=1e-3)
    work = torch.full((feedforward.workspace_bytes(calm["x"], calm["w_gate"], True),), 255, dtype=torch.uint8, device="cuda")
    first = [check(calm, work), check(wild, work), check(calm, work), check(wild, work)]
    for a, b in ((0, 2), (1, 3)):
        assert all(torch.equal(s, t) for s, t in zip(first[a], first[b]))
    order = ("dout", "x", "w_gate", "w_up", "w_down", "gate", "up")
    for pick in ((True, False, False, False), (False, True, False, True)):
        got = feedforward_backward(*(wild[n] for n in order), want=pick)
        assert all(b is None if not p else torch.equal(a, b) for a, b, p in zip(first[1], got, pick))
    graph, now = torch.cuda.CUDAGraph(), {n: t.clone() for n, t in calm.items()}
    with torch.cuda.graph(graph):
        made = feedforward_backward(*(now[n] for n in order))
    for of, want in ((wild, first[1]), (calm, first[0]), (wild, first[1])):
        for n in order:
            now[n].copy_(of[n])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(made, want))


@pytest.mark.parametrize("T, D, F", SHAPES)
def test_infinite_gradients_stay_in_their_token(T, D, F):
    """A token whose gradient is infinite or not a number: the other tokens' dx is what it is without that token."""
    from paper_2411_03742_b200 import feedforward_backward
    i = make(T, D, F, dy=0.1)
    args = [i[n] for n in ("dout", "x", "w_gate", "w_up", "w_down", "gate", "up")]
    for value in (math.inf, math.nan):
        i["dout"][5] = 0.0
        want = feedforward_backward(*args)[0]
        i["dout"][5, 3] = value
        got = feedforward_backward(*args)[0]
        keep = [t for t in range(T) if t != 5]
        assert torch.equal(got[keep], want[keep]) and not bool(got[5].isfinite().all())
