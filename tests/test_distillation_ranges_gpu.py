"""Distillation where few bits are left: gradients of logits that are hardly possible, logits that start off 16 bytes.

Tolerances as in test_distillation_gpu.py: a gradient to 2^-21 (8 + |z / tau| + |L|) of its terms, by magnitude, and half a step of its type; what is below fp32's smallest
normal number, 2^-126, counts as 0.
"""
import pytest
import torch

from test_distillation_gpu import TYPES, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0, 4.0, 2.5])
@pytest.mark.parametrize("mix", [0.0, 0.5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_labels_alone_far_below_the_likeliest(tau, mix, dtype):
    """Tokens with a label and no entries, or labels that have all of the loss: probabilities down to 4e-37 have gradients."""
    V = 4096
    z = -torch.linspace(0.0, 80.0, V, device="cuda").repeat(3, 1)[:, torch.randperm(V, generator=torch.Generator().manual_seed(1)).cuda()].to(TYPES[dtype])
    ids = torch.full((3, 2), -1, device="cuda")
    if mix == 0.0:
        ids[0] = torch.tensor([5, 9])
    labels = torch.tensor([7, 100, 4000], device="cuda")
    _, _, dz = check(z, ids, torch.zeros((3, 2), device="cuda"), tau, labels, mix)
    far = z.float() < -70
    far[torch.arange(3), labels] = False               # a label's own gradient is negative
    assert bool((dz[far] > 0).all()) and float(dz[far].float().max()) < 1e-28


@pytest.mark.parametrize("tau", [2.0, 4.0])
def test_a_large_vocabulary(tau):
    g = torch.Generator(device="cuda").manual_seed(3)
    z = 6 * torch.randn((2, 131072), generator=g, device="cuda")
    ids = torch.tensor([[-1, -1], [3, 7]], device="cuda")
    check(z, ids, torch.ones((2, 2), device="cuda"), tau, torch.tensor([11, 131071], device="cuda"), 0.25)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V, first", [(3, 1001, 1), (1, 5000, 1), (5, 4096, 3), (2, 9000, 2)])
def test_logits_off_16_bytes(dtype, T, V, first):
    """Logits that start inside a row: the gradient lies as they do relative to 16 bytes, at every call, and is what it is from a copy of them."""
    from paper_2411_03742_b200 import distill_backward, distill_forward
    wide, ids, top, labels = make(T, V + 8, 4, dtype, labels=True)
    ids, labels = ids.clamp(max=V - 1), labels.clamp(max=V - 1)
    dloss = torch.rand(T, device="cuda") + 0.5
    for at in (first, 0, first + 1):                   # the same layout, another start
        z = wide[:, at:at + V]
        how = dict(temperature=2.0, labels=labels, mix=0.4)
        loss, rows = distill_forward(z, ids, top, **how)
        dz = distill_backward(dloss, z, ids, top, rows, **how)
        assert dz.shape == z.shape and (dz.data_ptr() - z.data_ptr()) % 16 == 0
        assert T == 1 or (dz.stride(0) - z.stride(0)) * z.element_size() % 16 == 0
        leaf = z.clone().requires_grad_()
        copied = distill_forward(leaf.detach(), ids, top, **how)
        # sums over the vocabulary take another order: a few roundings, each 2^-24
        assert bool(((rows - copied[1]).abs() <= 2.0 ** -20 * (1 + rows.abs())).all())
        assert torch.equal(dz, distill_backward(dloss, leaf.detach(), ids, top, rows, **how))
        assert torch.equal(dz, distill_backward(dloss, z, ids, top, rows, out=torch.empty_like(z, memory_format=torch.contiguous_format), **how))
