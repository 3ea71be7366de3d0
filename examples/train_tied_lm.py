"""A small language model trained with every operator of the library together, on one GPU.

    x      = embed(table, ids) * sqrt(d)                 cast_embed
    h      = x + relu(x W1^T) W2^T                       W1, W2 pruned 2:4 by the AdamS plan (its masked bf16 forward weights)
    z      = h W3^T                                      W3 unpruned: momentum orthogonalised by cast_orthogonalize
    loss   = cross entropy of z table^T                  cast_linear_ce: dz and the head's part of dtable
    dtable += gradient of the lookup                     cast_embed_grad onto the head's gradient: table and head are one matrix

The table is trained by the same AdamS kernel with nothing pruned (4:4).  The data are a random walk over the vocabulary whose
next token is a fixed function of the last one most of the time, so the loss has somewhere to go.

    python examples/train_tied_lm.py [--steps N]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2509_25996_b200 import binding as B  # noqa: E402
from paper_2509_25996_b200 import ops, runner  # noqa: E402


class TiedModel:
    def __init__(self, vocab: int = 1000, d: int = 256, ffn: int = 512, seed: int = 0, device: str = "cuda:0"):
        self.vocab, self.d, self.device = vocab, d, torch.device(device)
        self.pruned = runner.DeviceModelState([(ffn, d), (d, ffn)], N=2, M=4, seed=seed, device=device, scale_mode="none")
        self.table = runner.DeviceModelState([(vocab, d)], N=4, M=4, seed=seed + 1, device=device, scale_mode="none")
        for state, std in ((self.pruned, 1.0), (self.table, 1.0)):
            for m in state.mats:
                m.w.mul_(std / math.sqrt(m.cols) / 0.02)
                m.m.zero_()
                m.v.zero_()
                m.g.zero_()
        gen = torch.Generator(device=device).manual_seed(seed + 2)
        self.w3 = torch.randn((d, d), generator=gen, device=device) / math.sqrt(d)
        self.momentum = torch.zeros_like(self.w3)
        self.w3_fwd = self.w3.to(torch.bfloat16)
        # a step with lr = 0 chooses the first mask and emits the first forward weights
        self._adams(runner.Hyper(lr=0.0, l1_coeff=0.0, step=1, total_steps=1))

    def _adams(self, h: runner.Hyper) -> None:
        self.pruned.step(h, B.CAST_F_RESELECT)
        self.table.step(h, B.CAST_F_RESELECT | B.CAST_F_META_BITMASK)

    def step(self, ids: torch.Tensor, labels: torch.Tensor, t: int, total: int, lr: float = 2e-3, lr_ortho: float = 0.02) -> torch.Tensor:
        """One training step on int32 ids and labels (labels < 0: no target); returns the mean loss (on the device)."""
        w1, w2 = (m.w_fwd for m in self.pruned.mats)
        table = self.table.mats[0].w_fwd
        scale = math.sqrt(self.d)
        # forward
        x = ops.embed(table, ids, scale)
        a = torch.relu(x @ w1.T)
        h = x + a @ w2.T
        z = h @ self.w3_fwd.T
        # loss, dz, dtable (head)
        loss, dz, dtable = ops.linear_ce(z, table, labels, grad_scale=1.0 / ids.numel())
        # backward
        dw3 = dz.T @ h
        dh = dz @ self.w3_fwd
        dw2 = dh.T @ a
        da = (dh @ w2) * (a > 0)
        dw1 = da.T @ x
        dx = dh + da @ w1
        ops.embed_grad(dx, ids, self.vocab, scale, grad_table=dtable, accumulate=True)
        # updates
        for m, g in zip(self.pruned.mats + self.table.mats, (dw1, dw2, dtable)):
            m.g.copy_(g)
        self._adams(runner.Hyper(lr=lr, l1_coeff=1e-5, step=t, total_steps=total))
        self.momentum.mul_(0.95).add_(dw3)
        update, = ops.orthogonalize([self.momentum])
        self.w3.sub_(update, alpha=lr_ortho)
        self.w3_fwd.copy_(self.w3)
        return loss.mean()


def batch(vocab: int, sequences: int, length: int, gen: torch.Generator, device):
    """Token ids and their successors: (7 t + 13) mod vocab nine times in ten, anything otherwise; the last label is none."""
    tok = torch.randint(0, vocab, (sequences,), generator=gen, device=device)
    out = [tok]
    for _ in range(length - 1):
        noise = torch.randint(0, vocab, (sequences,), generator=gen, device=device)
        keep = torch.rand(sequences, generator=gen, device=device) < 0.9
        tok = torch.where(keep, (7 * tok + 13) % vocab, noise)
        out.append(tok)
    ids = torch.stack(out, 1)
    labels = torch.full_like(ids, -1)
    labels[:, :-1] = ids[:, 1:]
    return ids.reshape(-1).int(), labels.reshape(-1).int()


def train(steps: int = 200, sequences: int = 16, length: int = 64, seed: int = 0, report=None):
    model = TiedModel(seed=seed)
    gen = torch.Generator(device=model.device).manual_seed(seed + 3)
    losses = []
    for t in range(1, steps + 1):
        ids, labels = batch(model.vocab, sequences, length, gen, model.device)
        losses.append(model.step(ids, labels, t, steps))
        if report and (t % 20 == 0 or t == 1):
            report(f"step {t:4d}  loss {float(losses[-1]):.3f}")
    return [float(x) for x in torch.stack(losses)], model


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=200)
    train(p.parse_args().steps, report=print)
