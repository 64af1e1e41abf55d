"""Hang protection of the training operators: with one tile missing the kernels' own waits run out after 2 s each, the blocks
release their tensor memory, meet what they have to meet and return, the status word says so once, and the next call is right.
Nothing here faults, traps or waits without bound."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu
TIMEOUT = 0x100


def timed(call):
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    call()
    torch.cuda.synchronize()
    return time.perf_counter() - t0


@pytest.mark.parametrize("dtype, shapes", [("f32", [(300, 520)]), ("bf16", [(300, 520), (40, 1000)]), ("f32", [(64, 4096)]), ("bf16", [(512, 1024)] * 24 + [(1000, 500)] * 8)],
                         ids=["fp32", "lone-blocks", "split-rows", "pairs"])
def test_a_tile_that_nobody_computes(dtype, shapes):
    from paper_2411_03742_b200 import Orthogonalizer
    with Orthogonalizer(shapes, dtype) as plan:
        u = torch.randn(plan.d, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        want, out = torch.empty_like(u), torch.empty_like(u)
        plan.apply(u, want)
        torch.cuda.synchronize()
        assert plan.status() == 0
        waited = timed(lambda: plan.selftest_bounded_wait(u, out))
        assert 1.5 < waited < 30.0, waited              # gave up at the limit, not before, not never
        assert plan.status() == TIMEOUT and plan.status() == 0
        for _ in range(2):
            plan.apply(u, out)
            torch.cuda.synchronize()
            assert plan.status() == 0 and torch.equal(out, want)


def test_matrices_of_one_block_have_no_such_wait():
    from paper_2411_03742_b200 import AdaConsError, Orthogonalizer
    with Orthogonalizer([(96, 200)], "bf16") as plan:
        u = torch.randn(plan.d, device="cuda").bfloat16()
        with pytest.raises(AdaConsError):
            plan.selftest_bounded_wait(u, torch.empty_like(u))


@pytest.mark.parametrize("B, Sq, Sk", [(2, 300, 300), (1, 1, 4000), (1, 4000, 200), (1, 130, 100)], ids=["blocks", "shared-keys", "shared-queries", "one-tile"])
def test_tiles_that_never_come(B, Sq, Sk):
    from paper_2411_03742_b200 import attention, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sk)
    q = torch.randn((B, Sq, 4, 64), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((B, Sk, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    out, lse = attention_forward(q, k, v)
    grads = attention_backward(out, q, k, v, out, lse)
    torch.cuda.synchronize()
    assert attention.status() == 0
    spare = [torch.empty_like(t) for t in (out, lse, *grads)]
    for call in (lambda: attention.selftest_bounded_wait(q, k, v, spare[0], spare[1]), lambda: attention.selftest_bounded_wait(q, k, v, out, lse, spare[2:])):
        waited = timed(call)
        assert 1.5 < waited < 30.0, waited
        assert attention.status() == TIMEOUT and attention.status() == 0
        again = attention_forward(q, k, v)
        again += attention_backward(out, q, k, v, *again)
        torch.cuda.synchronize()
        assert attention.status() == 0 and all(torch.equal(a, b) for a, b in zip(again, (out, lse, *grads)))


def test_selftest_refusals():
    from paper_2411_03742_b200 import AdaConsError, attention
    for dtype, D in ((torch.float16, 64), (torch.bfloat16, 128)):
        q = torch.zeros((1, 8, 2, D), dtype=dtype, device="cuda")
        with pytest.raises(AdaConsError):
            attention.selftest_bounded_wait(q, q, q, torch.empty_like(q), torch.empty((1, 2, 8), device="cuda"))
