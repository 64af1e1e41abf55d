"""A small causal transformer trained by N simulated workers, every step through the library's operators.

Each worker computes the gradient of its own batch (rotary positions and attention, forward and backward,
through `Rope` and `attention`), the N flat gradients are stacked and aggregated with `AdaCons`, and the
aggregated direction, smoothed by a momentum, is orthogonalised matrix by matrix with `Orthogonalizer` before
it is applied.  The task is synthetic: sequences of an affine recurrence modulo a prime, whose next element
follows from the one before it and the sequence's own hidden multiplier.

    python -m paper_2411_03742_b200.examples.transformer_workers --workers 8 --steps 100
"""
from __future__ import annotations

import argparse
import math

import torch
import torch.nn.functional as F

from .. import binding
from ..attention import attention
from ..orth import Orthogonalizer
from ..rope import Rope


class Model:
    """Parameters live in one flat fp32 vector: `flat`; `views` are its pieces, `matrices` the (rows, cols) and offset of
    those that are orthogonalised (attention and feed-forward weights)."""

    def __init__(self, vocab: int, dim: int = 128, heads: int = 4, kv_heads: int = 2, layers: int = 2, device="cuda:0", seed: int = 0):
        self.dim, self.heads, self.kv_heads, self.layers, self.head_dim = dim, heads, kv_heads, layers, dim // heads
        qkv = (heads + 2 * kv_heads) * self.head_dim
        shapes = [("embed", (vocab, dim))]
        for i in range(layers):
            shapes += [(f"{i}.gain1", (dim,)), (f"{i}.qkv", (qkv, dim)), (f"{i}.out", (dim, dim)), (f"{i}.gain2", (dim,)),
                       (f"{i}.up", (4 * dim, dim)), (f"{i}.down", (dim, 4 * dim))]
        shapes += [("gain", (dim,))]
        g = torch.Generator().manual_seed(seed)
        pieces, self.views, self.matrices, at = [], {}, [], 0
        for name, shape in shapes:
            n = math.prod(shape)
            w = torch.ones(shape) if len(shape) == 1 else torch.randn(shape, generator=g) / math.sqrt(shape[1])
            pieces.append(w.reshape(-1))
            if len(shape) == 2 and name != "embed":
                self.matrices.append((shape, at))
            self.views[name] = (at, shape)
            at += n
        self.flat = torch.cat(pieces).to(device).requires_grad_()
        self.rope = Rope(self.head_dim)

    def _w(self, name):
        at, shape = self.views[name]
        return self.flat[at:at + math.prod(shape)].view(shape)

    def loss(self, tokens):
        """Mean next-token cross entropy of (batch, length) tokens."""
        x = self._w("embed")[tokens]
        B, S = tokens.shape
        H, K, D = self.heads, self.kv_heads, self.head_dim
        for i in range(self.layers):
            h = F.rms_norm(x, (self.dim,)) * self._w(f"{i}.gain1")
            qkv = (h.bfloat16() @ self._w(f"{i}.qkv").bfloat16().T).view(B, S, H + 2 * K, D)
            turned = self.rope(qkv[:, :, :H + K])                  # queries and keys in one call
            a = attention(turned[:, :, :H], turned[:, :, H:], qkv[:, :, H + K:], causal=True)
            x = x + (a.reshape(B, S, self.dim) @ self._w(f"{i}.out").bfloat16().T).float()
            h = F.rms_norm(x, (self.dim,)) * self._w(f"{i}.gain2")
            x = x + (F.gelu(h.bfloat16() @ self._w(f"{i}.up").bfloat16().T) @ self._w(f"{i}.down").bfloat16().T).float()
        x = F.rms_norm(x, (self.dim,)) * self._w("gain")
        logits = x @ self._w("embed").T
        return F.cross_entropy(logits[:, :-1].reshape(-1, logits.shape[-1]), tokens[:, 1:].reshape(-1))


def batch(workers: int, size: int, length: int, prime: int, gen: torch.Generator, device):
    """(workers, size, length) tokens: x_{k+1} = a x_k + 1 mod prime, with a drawn per sequence from a few multipliers."""
    a = torch.randint(2, 6, (workers, size), generator=gen)
    x = torch.randint(0, prime, (workers, size), generator=gen)
    seq = []
    for _ in range(length):
        seq.append(x)
        x = (a * x + 1) % prime
    return torch.stack(seq, -1).to(device)


def run(workers: int = 8, size: int = 16, length: int = 96, steps: int = 60, prime: int = 61, lr: float = 0.02, beta: float = 0.9, seed: int = 0,
        device: str = "cuda:0", orthogonalise: bool = True):
    """Mean loss over the workers, one value per step."""
    dev = torch.device(device)
    model = Model(prime, device=dev, seed=seed)
    d = model.flat.numel()
    grads = torch.empty((workers, d), device=dev)
    psi, momentum = torch.empty(d, device=dev), torch.zeros(d, device=dev)
    rest = torch.ones(d, dtype=torch.bool, device=dev)
    for (m, n), at in model.matrices:
        rest[at:at + m * n] = False
    gen = torch.Generator().manual_seed(seed + 1)
    losses = []
    with binding.AdaCons(workers, d, "f32") as agg, Orthogonalizer([s for s, _ in model.matrices], "f32", offsets=[o for _, o in model.matrices], d=d,
                                                                  scaling=True) as orth:
        for _ in range(steps):
            tokens = batch(workers, size, length, prime, gen, dev)
            total = 0.0
            for w in range(workers):
                loss = model.loss(tokens[w])
                grads[w], = torch.autograd.grad(loss, model.flat)
                total += float(loss.detach())
            agg.aggregate(grads, psi)
            momentum.mul_(beta).add_(psi)
            direction = momentum * (1 - beta)
            # embeddings and gains: the direction with unit mean square
            update = torch.where(rest, direction / (direction[rest].square().mean().sqrt() + 1e-12), torch.zeros_like(direction))
            if orthogonalise:
                orth.apply(direction, update)
            else:
                for (m, n), at in model.matrices:
                    g = direction[at:at + m * n]
                    update[at:at + m * n] = g / (g.square().mean().sqrt() * math.sqrt(max(m, n)) + 1e-12)
            with torch.no_grad():
                model.flat -= lr * update * torch.where(rest, 0.2, 1.0)
            losses.append(total / workers)
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--length", type=int, default=96)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--plain", action="store_true", help="scaled instead of orthogonalised updates")
    a = ap.parse_args(argv)
    losses = run(a.workers, a.batch, a.length, a.steps, lr=a.lr, orthogonalise=not a.plain)
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {k:4d}  loss {losses[k]:.4f}")
    print(f"step {a.steps - 1:4d}  loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
