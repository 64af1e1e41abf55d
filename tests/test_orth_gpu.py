"""Orthogonalisation of a flat vector's matrices against the formula in 64 bits.

Tolerances (relative to the result's norm).  bf16: the result's own rounding is at most 2^-9 (rms, relative to
the elements), the products' operands are fp16 (2^-11 of an element at most): independent errors that average
over the short side and that five steps carry along, another 2^-9; together 2^-8.  On sides below 16 nothing averages: the rounding
of the result alone can reach 2^-8, the operands' roundings of a single singular value are amplified by the
polynomial's slope (up to 4 near 1.2): 2e-2.  fp32: operands of 22 bits and sums in fp32 (2^-22 = 2.4e-7 per
operation), small singular values grown 3.44-fold five times against errors that do not grow with them: 2e-5.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
COEFFS = (3.4445, -4.7750, 2.0315)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def tol(dtype, m, n):
    return 2e-5 if dtype == "f32" else 2.0 ** -8 if min(m, n) >= 16 else 2e-2


def plain(G, triples, eps):
    x = G.double()
    x = x / (x.norm() + eps)
    for a, b, c in triples:
        s = x @ x.mT if x.shape[0] <= x.shape[1] else x.mT @ x
        q = b * s + c * (s @ s)
        x = a * x + (q @ x if x.shape[0] <= x.shape[1] else x @ q)
    return x


def run(shapes, dtype, gap=0, lead=0, kind="gauss", steps=5, coeffs=COEFFS, eps=1e-7, scaling=False, seed=0, in_place=False):
    from paper_2411_03742_b200 import Orthogonalizer
    at, offsets = lead, []
    for m, n in shapes:
        offsets.append(at)
        at += m * n + gap
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.randn(at, generator=g, device="cuda") * 1e-3
    if kind == "low rank":
        for (m, n), o in zip(shapes, offsets):
            u[o:o + m * n] += (torch.randn((m, 4), generator=g, device="cuda") @ torch.randn((4, n), generator=g, device="cuda")).reshape(-1) * 1e-2
    u = u.to(TYPES[dtype])
    with Orthogonalizer(shapes, dtype, offsets=offsets, d=at, steps=steps, coeffs=coeffs, eps=eps, scaling=scaling) as plan:
        keep = u.clone()
        out = u if in_place else torch.full_like(u, 7.0)
        plan.apply(u, out)
        torch.cuda.synchronize()
        assert plan.status() == 0
    if not in_place:
        assert torch.equal(u, keep), "the input changed"
    triples = [coeffs] * steps if not hasattr(coeffs[0], "__len__") else coeffs
    inside = torch.zeros(at, dtype=torch.bool, device="cuda")
    for (m, n), o in zip(shapes, offsets):
        inside[o:o + m * n] = True
        want = plain(keep[o:o + m * n].view(m, n), triples, eps) * (math.sqrt(max(1.0, m / n)) if scaling else 1.0)
        got = out[o:o + m * n].view(m, n).double()
        err = float((got - want).norm() / want.norm())
        assert err <= tol(dtype, m, n), (m, n, err)
    rest = keep if in_place else torch.full_like(keep, 7.0)
    assert torch.equal(out[~inside], rest[~inside]), "elements between the matrices changed"
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (9, 1), (3, 5), (16, 16), (31, 33), (63, 65), (64, 64), (127, 129), (128, 128), (129, 127), (128, 257), (96, 200),
                                   (200, 96), (255, 256), (257, 255), (300, 40), (40, 1300), (385, 513), (513, 2049), (1030, 700)])
def test_one_matrix(dtype, shape):
    run([shape], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["gauss", "low rank"])
def test_many_matrices_between_other_parameters(dtype, kind):
    run([(130, 70), (1, 17), (64, 300), (257, 257), (500, 129), (33, 33), (8, 640)], dtype, gap=5, lead=3, kind=kind)


def test_enough_tiles_for_pairs_of_blocks():
    # 24 x 2 x 4 tiles of 256 x 256 and more: the paired tiling in every product
    run([(512, 1024)] * 24 + [(1000, 500)] * 8, "bf16", gap=8)
    run([(512, 1024)] * 24, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(1, 100003)], [(29, 3381)], [(4096, 64)], [(130, 4001)], [(300, 5000), (40, 40)], [(16, 4096)] * 8 + [(2051, 17)]])
def test_long_rows_split_over_their_length(dtype, shapes):
    out = run(shapes, dtype, gap=3)
    assert torch.equal(out, run(shapes, dtype, gap=3)), "partial sums are added in one order"


def test_vectors_larger_than_the_cache_go_in_turns():
    run([(1024, 4096)] * 8 + [(2000, 1000)] * 10, "bf16", gap=8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_scaling(dtype):
    run([(200, 96), (96, 200)], dtype, gap=1, in_place=True)
    run([(200, 96), (96, 200)], dtype, scaling=True)


def test_other_coefficients_per_step():
    run([(150, 90)], "f32", steps=3, coeffs=[(1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)])
    run([(150, 90)], "bf16", steps=1, coeffs=(1.5, -0.5, 0.0))


def test_magnitudes_and_degenerate_matrices():
    from paper_2411_03742_b200 import Orthogonalizer
    for scale in (1e-30, 1e-6, 1e6, 1e30):          # the norm is taken in fp64
        u = torch.randn(64 * 80, device="cuda") * scale
        out = torch.empty_like(u)
        with Orthogonalizer([(64, 80)], "f32", eps=0.0) as plan:
            plan.apply(u, out)
        want = plain(u.view(64, 80), [COEFFS] * 5, 0.0)
        assert float((out.view(64, 80).double() - want).norm() / want.norm()) <= 2e-5, scale
    # a matrix of zeros gives zeros; Inf and NaN stay in their matrix
    shapes = [(40, 50)] * 4
    u = torch.randn(4 * 2000, device="cuda")
    u[:2000] = 0
    u[2500] = math.inf
    u[4100] = math.nan
    out = torch.empty_like(u)
    with Orthogonalizer(shapes, "f32") as plan:
        plan.apply(u, out)
    assert not out[:2000].any()
    assert out[2000:4000].isnan().all() and out[4000:6000].isnan().all()
    want = plain(u[6000:].view(40, 50), [COEFFS] * 5, 1e-7)
    assert float((out[6000:].view(40, 50).double() - want).norm() / want.norm()) <= 2e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_buffers_streams_and_repeats(dtype):
    """Buffers off any vector boundary give the bytes of aligned ones; so do other streams and repeats."""
    from paper_2411_03742_b200 import Orthogonalizer
    shapes = [(72, 136), (136, 72), (65, 31)]
    with Orthogonalizer(shapes, dtype) as plan:
        u = torch.randn(plan.d, device="cuda").to(TYPES[dtype])
        out = torch.zeros_like(u)
        plan.apply(u, out)
        wide = torch.zeros(plan.d + 9, dtype=TYPES[dtype], device="cuda")
        far = torch.full((plan.d + 9,), 7.0, dtype=TYPES[dtype], device="cuda")
        for k in (1, 3, 8):
            wide[k:k + plan.d] = u
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            plan.apply(wide[k:k + plan.d], far[k:k + plan.d], stream=side)
            torch.cuda.synchronize()
            assert torch.equal(far[k:k + plan.d], out), k
            assert (far[k + plan.d:] == 7.0).all()


def test_captured_in_a_graph():
    from paper_2411_03742_b200 import Orthogonalizer
    with Orthogonalizer([(130, 260)], "bf16") as plan:
        u = torch.randn(plan.d, device="cuda").bfloat16()
        out, want = torch.empty_like(u), torch.empty_like(u)
        plan.apply(u, want)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            plan.apply(u, out)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_offsets_past_32_bits():
    from paper_2411_03742_b200 import Orthogonalizer
    m, n, at = 40, 56, (1 << 31) + 12345
    d = at + m * n + 3
    src, want = torch.randn(m * n, device="cuda").bfloat16(), torch.empty(m * n, dtype=torch.bfloat16, device="cuda")
    with Orthogonalizer([(m, n)], "bf16") as near:
        near.apply(src, want)
    u = torch.zeros(d, dtype=torch.bfloat16, device="cuda")
    u[at:at + m * n] = src
    with Orthogonalizer([(m, n)], "bf16", offsets=[at], d=d) as plan:
        plan.apply(u, u)
        torch.cuda.synchronize()
    assert torch.equal(u[at:at + m * n], want)
    assert not u[:at].any() and not u[at + m * n:].any()


def test_refuses_wrong_tensors():
    from paper_2411_03742_b200 import Orthogonalizer
    with Orthogonalizer([(8, 8)], "bf16") as plan:
        good = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
        for bad in (good.float(), good[:63], good.cpu(), good.view(8, 8)):
            with pytest.raises(ValueError):
                plan.apply(bad, good)
            with pytest.raises(ValueError):
                plan.apply(good, bad)
    with pytest.raises(ValueError):
        Orthogonalizer([], "bf16")
    with pytest.raises(ValueError):
        Orthogonalizer([(2, 2)], "bf16", offsets=[0, 4])
    with pytest.raises(ValueError):
        Orthogonalizer([(2, 2)], "bf16", steps=2, coeffs=[(1, 0, 0)])


@pytest.mark.parametrize("shape", [(64, 80), (150, 300), (300, 150), (131, 257)])
def test_norms_whose_inverse_leaves_fp32(shape):
    """fp32 matrices down to the smallest numbers of the type and up to near its largest, in one block and in the general kernel; with eps
    of no weight.  A matrix of such small numbers carries few bits itself: the formula is taken from what it holds."""
    from paper_2411_03742_b200 import Orthogonalizer
    g = torch.Generator(device="cuda").manual_seed(3)
    for dtype in ("f32", "bf16"):
        for scale in (1e-44, 1e-40, 1e-37, 1e-35, 1e20, 3e37):
            u = (torch.randn(shape[0] * shape[1], generator=g, device="cuda", dtype=torch.float64) * scale).clamp(-3.3e38, 3.3e38).to(TYPES[dtype])
            if not u.any():                             # bf16 has nothing as small as 1e-44
                assert dtype == "bf16" and scale == 1e-44
                continue
            out = torch.empty_like(u)
            with Orthogonalizer([shape], dtype, eps=0.0) as plan:
                plan.apply(u, out)
            want = plain(u.view(shape), [COEFFS] * 5, 0.0)
            assert float((out.view(shape).double() - want).norm() / want.norm()) <= tol(dtype, *shape), (dtype, scale)
    u = torch.zeros(shape[0] * shape[1], device="cuda")
    out = torch.full_like(u, 7.0)
    with Orthogonalizer([shape], "f32", eps=1e-310) as plan:       # zeros give zeros for any eps > 0
        plan.apply(u, out)
    assert not out.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 80), (150, 300), (300, 150)])
def test_coefficients_up_to_the_limit_of_the_products(dtype, shape):
    """One row (or column) of the matrix is not zero, so the first step makes its length a, and S = a^2 in the second: right below
    8, not finite from there on."""
    from paper_2411_03742_b200 import Orthogonalizer
    u = torch.zeros(shape, dtype=TYPES[dtype], device="cuda")
    if shape[0] < shape[1]:
        u[3] = torch.randn(shape[1], generator=torch.Generator().manual_seed(1)).cuda()
    else:
        u[:, 3] = torch.randn(shape[0], generator=torch.Generator().manual_seed(1)).cuda()
    u = u.flatten()
    for a, inside in ((2.82, True), (2.84, False)):
        triples, out = [(a, 0.0, 0.0), (1.0, 0.0, 0.0)], torch.empty_like(u)
        with Orthogonalizer([shape], dtype, steps=2, coeffs=triples) as plan:
            plan.apply(u, out)
        if inside:
            want = plain(u.view(shape), triples, 1e-7)
            assert float((out.view(shape).double() - want).norm() / want.norm()) <= tol(dtype, *shape)
        else:
            assert not out.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(150, 300), (300, 150), (40, 1000)])
def test_magnitudes_and_degenerate_matrices_of_the_general_kernel(dtype, shape):
    from paper_2411_03742_b200 import Orthogonalizer
    n = shape[0] * shape[1]
    g = torch.Generator(device="cuda").manual_seed(n)
    for scale in (1e-30, 1e-6, 1e6, 1e30):
        u = (torch.randn(n, generator=g, device="cuda") * scale).to(TYPES[dtype])
        out = torch.empty_like(u)
        with Orthogonalizer([shape], dtype, eps=0.0) as plan:
            plan.apply(u, out)
        want = plain(u.view(shape), [COEFFS] * 5, 0.0)
        assert float((out.view(shape).double() - want).norm() / want.norm()) <= tol(dtype, *shape), scale
    u = torch.randn(4 * n, generator=g, device="cuda").to(TYPES[dtype])
    u[:n] = 0
    u[n + 500] = math.inf
    u[2 * n + 100] = math.nan
    out = torch.full_like(u, 7.0)
    with Orthogonalizer([shape] * 4, dtype) as plan:
        plan.apply(u, out)
        torch.cuda.synchronize()
        assert plan.status() == 0
    assert not out[:n].any()
    assert out[n:3 * n].isnan().all()
    want = plain(u[3 * n:].view(shape), [COEFFS] * 5, 1e-7)
    assert float((out[3 * n:].view(shape).double() - want).norm() / want.norm()) <= tol(dtype, *shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_buffers_and_far_offsets_in_the_general_kernel(dtype):
    """The same bytes wherever buffers and matrices start, 2^31 elements in among them, in place and not."""
    from paper_2411_03742_b200 import Orthogonalizer
    shapes = [(160, 296), (296, 160), (150, 301)]
    sizes = [m * n for m, n in shapes]
    near = [0, sizes[0], sizes[0] + sizes[1]]
    u = torch.randn(sum(sizes), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(TYPES[dtype])
    want = torch.empty_like(u)
    with Orthogonalizer(shapes, dtype) as plan:
        plan.apply(u, want)
        wide, far = (torch.full((plan.d + 9,), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2))
        for k in (1, 3, 8):
            wide[k:k + plan.d] = u
            plan.apply(wide[k:k + plan.d], far[k:k + plan.d])
            assert torch.equal(far[k:k + plan.d], want), k
            assert (far[k + plan.d:] == 7.0).all()
            far.fill_(7.0)
    at = [5, (1 << 31) + 12345, (1 << 31) + 12345 + sizes[1] + 1]
    d = at[2] + sizes[2] + 3
    big = torch.zeros(d, dtype=TYPES[dtype], device="cuda")
    for o, p, s in zip(at, near, sizes):
        big[o:o + s] = u[p:p + s]
    with Orthogonalizer(shapes, dtype, offsets=at, d=d) as plan:
        plan.apply(big, big)
        torch.cuda.synchronize()
        assert plan.status() == 0
    for o, p, s in zip(at, near, sizes):
        assert torch.equal(big[o:o + s], want[p:p + s])
        big[o:o + s] = 0
    assert not any(part.any() for part in big.split(1 << 28))
