"""Distillation where few bits are left: gradients of logits that are hardly possible.

Tolerances as in test_distillation_gpu.py: a gradient to 2^-21 (8 + |z / tau| + |L|) of its terms, by magnitude, and half a step of its type; what is below fp32's smallest
normal number, 2^-126, counts as 0.
"""
import pytest
import torch

from test_distillation_gpu import TYPES, check

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
