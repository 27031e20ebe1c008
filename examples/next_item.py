"""A next-item model on top of the cache: the cached table and the dense operators in one training step, and one step of serving.

A sample has context features (one id each, in one large table behind the cache, pooled per feature) and a sequence of items it has met, padded to
SEQ.  Items and positions have small dense tables.

    x = lookup(items) * sqrt(DIM)        token_embed_fwd, bf16 out of an f32 table
    y = rms_norm(x + lookup(positions))  rms_norm_fwd, the position rows are the residual
    logits = (mean of y over the sequence | context rows) @ head

The backward pass gives the norm's weight, the item table (padding left out) and the position table their gradients; they are clipped together with
the head's and the pooled context rows' by one global norm, and stepped by plain SGD, the cached table by its fused backward pass (the update is
linear in the pooled rows' gradient, so that clipping that clips the step; its share of the norm is that of the pooled rows, which is not the table's where a
bag or a batch has an id more than once).

    python examples/next_item.py [--steps 30]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2208_05321_amd import DenseOps, FreqCache  # noqa: E402

ROWS, CACHE_ROWS, FEATURES = 200_000, 6000, 8      # the table behind the cache
ITEMS, SEQ, DIM, PAD = 5000, 48, 64, 0
SAMPLES, LR, MAX_NORM = 256, 0.5, 1.0


class Model:
    def __init__(self, seed: int = 0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.cache = FreqCache(ROWS, DIM, CACHE_ROWS, rng.permutation(ROWS).astype(np.int32))
        self.cache.host_weight()[:] = rng.standard_normal((ROWS, DIM), dtype=np.float32) * 0.05
        self.cache.warm()
        self.ops = DenseOps()
        new = lambda *shape: torch.randn(shape, generator=g, device="cuda") * 0.05  # noqa: E731
        self.items, self.positions, self.head = new(ITEMS, DIM), new(SEQ, DIM), new(DIM * (1 + FEATURES), ITEMS)
        self.weight = torch.ones(DIM, device="cuda")
        self.at = torch.arange(SEQ, device="cuda", dtype=torch.int32).repeat(SAMPLES)
        self.offsets = torch.arange(SAMPLES * FEATURES + 1, device="cuda")

    def encode(self, items, at):
        """Normed rows of the sequences, with what the backward pass needs."""
        x = self.ops.token_embed_fwd(self.items, items, scale=DIM ** 0.5, out_dtype=torch.bfloat16)
        r = self.ops.token_embed_fwd(self.positions, at, out_dtype=torch.bfloat16)
        y, h, _ = self.ops.rms_norm_fwd(x, self.weight, residual=r, h_out=x)
        return y, h

    def step(self, context, items, target) -> torch.Tensor:
        """One training step; the loss and the gradients' norm (before clipping), on the GPU."""
        ops, cache = self.ops, self.cache
        slots = cache.prepare(context, self.offsets)
        pooled = cache.embedding_bag_fwd(slots, self.offsets).requires_grad_()
        y, h = self.encode(items, self.at)
        y.requires_grad_()
        real = (items != PAD).view(SAMPLES, SEQ, 1)
        state = (y.float().view(SAMPLES, SEQ, DIM) * real).sum(1) / real.sum(1)
        head = self.head.requires_grad_()
        loss = torch.nn.functional.cross_entropy(torch.cat([state, pooled.view(SAMPLES, -1)], 1) @ head, target)
        gy, gp, gh = torch.autograd.grad(loss, (y, pooled, head))
        self.head.requires_grad_(False)

        gx, gw = ops.rms_norm_bwd(gy, h, self.weight)
        gi = ops.token_embed_bwd(gx, items, ITEMS, scale=DIM ** 0.5, padding_id=PAD)
        gpos = ops.token_embed_bwd(gx, self.at, SEQ)
        norm = ops.grad_norm_clip([gi, gpos, gw, gh, gp], MAX_NORM)
        for p, d in ((self.items, gi), (self.positions, gpos), (self.weight, gw), (self.head, gh)):
            p.sub_(d, alpha=LR)
        cache.embedding_bag_bwd_sgd(slots, self.offsets, gp, LR)
        return torch.stack([loss.detach(), norm[0]])

    def serve(self, item):
        """One new item of one sequence: its normed row in 8 bits with its scale, as a product in 8 bits takes it."""
        x = self.ops.token_embed_fwd(self.items, item, scale=DIM ** 0.5, out_dtype=torch.bfloat16)
        y, _, scale = self.ops.rms_norm_fwd(x, self.weight, out_dtype=torch.float8_e4m3fn)
        return y, scale

    def close(self):
        self.ops.check()
        self.cache.check()
        self.ops.close()
        self.cache.close()


def batches(seed: int = 1):
    """Sequences whose last item says what comes next; popular ids come up more often."""
    rng = np.random.default_rng(seed)
    while True:
        items = np.minimum(rng.zipf(1.3, (SAMPLES, SEQ)), ITEMS - 1).astype(np.int64)
        items[np.arange(SEQ)[None, :] >= rng.integers(SEQ // 2, SEQ + 1, SAMPLES)[:, None]] = PAD
        favourite = rng.integers(1, 40, SAMPLES)
        items[:, :SEQ // 3] = favourite[:, None]
        context = np.minimum(rng.zipf(1.2, (SAMPLES, FEATURES)) - 1, ROWS // FEATURES - 1) + np.arange(FEATURES) * (ROWS // FEATURES)
        yield tuple(torch.from_numpy(a.reshape(-1)).cuda() for a in (context, items, 100 + favourite))


def train(steps: int):
    """(losses, gradient norms, model) of that many steps."""
    model, data, seen = Model(), batches(), []
    for _ in range(steps):
        seen.append(model.step(*next(data)))
    losses, norms = torch.stack(seen).T.tolist()
    return losses, norms, model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    losses, norms, model = train(ap.parse_args().steps)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:3d}  loss {losses[k]:.3f}  gradient norm {norms[k]:.3f}")
    row, scale = model.serve(torch.tensor([7], device="cuda"))
    print(f"served: {row.dtype} {tuple(row.shape)}, scale {float(scale):.4f}; cache {model.cache.stats()}")
    model.close()
