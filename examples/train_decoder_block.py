"""One decoder block of a small language model, trained with gradient accumulation and clipping, on one GPU.

    h0 = embed(table, ids)                               cast_embed
    n1 = norm(h0)                                        cast_rms_norm
    q, k, v = n1 Wqkv^T; q and k turned                  cast_rotary: two axes (a token's place in its line, and the line)
    h1 = h0 + attention(q, k, v) Wo^T, n2 = norm(h1)     cast_rms_norm adds the residual
    h2 = h1 + relu(n2 Wup^T) Wdown^T, n3 = norm(h2)      cast_rms_norm
    loss = cross entropy of n3 table^T                   cast_linear_ce

and back: cast_rms_norm_grad adds the gradient that comes down the residual stream, cast_rotary turns the gradients of q and k back into
the fused projection's gradient.  The gradients of all micro-batches are accumulated in fp32, then scaled, clipped to a global
norm and written as the bf16 gradients that the AdamS plan takes, in one call of cast_grads_clip; the norms' weights take a
plain Adam step (cast_scale_adam_step).  The attention itself is elementary torch.

    python examples/train_decoder_block.py [--steps N]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from typing import Dict, List

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2509_25996_b200 as cast  # noqa: E402
from paper_2509_25996_b200 import binding as B  # noqa: E402
from paper_2509_25996_b200 import ops, runner  # noqa: E402

EPS = 1e-5


class DecoderBlock:
    def __init__(self, vocab: int = 512, d: int = 128, heads: int = 4, key_heads: int = 2, ffn: int = 256, lines: int = 4, line: int = 16, seed: int = 0,
                 device: str = "cuda:0"):
        self.vocab, self.d, self.heads, self.key_heads, self.head_dim, self.device = vocab, d, heads, key_heads, d // heads, torch.device(device)
        self.length = lines * line
        self.names = ("qkv", "o", "up", "down", "table")
        shapes = [((heads + 2 * key_heads) * self.head_dim, d), (d, d), (ffn, d), (d, ffn)]
        self.pruned = runner.DeviceModelState(shapes, N=2, M=4, seed=seed, device=device, scale_mode="none")
        self.dense = runner.DeviceModelState([(vocab, d)], N=4, M=4, seed=seed + 1, device=device, scale_mode="none")
        self.mats = self.pruned.mats + self.dense.mats
        for m in self.mats:
            m.w.mul_(1.0 / math.sqrt(m.cols) / 0.02)
            for t in (m.m, m.v, m.g):
                t.zero_()
        self.norms = torch.ones((3, d), device=device)
        self.norm_state = torch.zeros((2, 3, d), device=device)
        # every gradient in fp32; the clipped ones go to the places that the optimizers read
        self.grads = {name: torch.zeros((m.rows, m.cols), device=device) for name, m in zip(self.names, self.mats)}
        self.norm_grads = torch.zeros_like(self.norms)
        self.all_grads = ops.GradientSet(list(self.grads.values()) + [self.norm_grads], [m.g for m in self.mats] + [self.norm_grads])
        place = torch.arange(self.length, dtype=torch.int32, device=device)
        self.positions = torch.stack((place % line, place // line))
        self.spectrum = ops.RotarySpectrum.of(self.head_dim, base=100.0, sections=[self.head_dim // 4, self.head_dim // 2 - self.head_dim // 4],
                                              per_axis=True, device=device)
        self.hidden = torch.ones((self.length, self.length), dtype=torch.bool, device=device).triu(1)          # tokens that come later
        self._adams(runner.Hyper(lr=0.0, l1_coeff=0.0, step=1, total_steps=1))                                # first masks and forward weights

    def _adams(self, h: runner.Hyper) -> None:
        self.pruned.step(h, B.CAST_F_RESELECT)
        self.dense.step(h, B.CAST_F_RESELECT | B.CAST_F_META_BITMASK)

    def weights(self) -> Dict[str, torch.Tensor]:
        return {name: m.w_fwd for name, m in zip(self.names, self.mats)}

    def _split(self, qkv: torch.Tensor):
        """q, k and v as [tokens, heads, head_dim] inside the rows of the fused projection."""
        t, hd = qkv.shape[0], self.head_dim
        a, b = self.heads * hd, (self.heads + self.key_heads) * hd
        return (x.view(t, -1, hd) for x in (qkv[:, :a], qkv[:, a:b], qkv[:, b:]))

    def _by_sequence(self, x: torch.Tensor) -> torch.Tensor:
        """[tokens, heads, head_dim] -> fp32 [sequences, heads of q, length, head_dim]"""
        x = x.float().view(-1, self.length, x.shape[1], self.head_dim).transpose(1, 2)
        return x.repeat_interleave(self.heads // x.shape[1], 1)

    def _by_token(self, x: torch.Tensor, heads: int) -> torch.Tensor:
        """The reverse, summed over the heads that share one of `heads`."""
        x = x.view(x.shape[0], heads, -1, self.length, self.head_dim).sum(2)
        return x.transpose(1, 2).reshape(-1, heads, self.head_dim).to(torch.bfloat16)

    def accumulate(self, ids: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        """Adds the gradients of one micro-batch (int32 ids and labels of whole sequences) and returns its mean loss."""
        w, (g1, g2, g3) = self.weights(), self.norms
        tokens = ids.numel()
        positions = self.positions.repeat(1, tokens // self.length)
        # forward
        x = ops.embed(w["table"], ids)
        n1, h0 = ops.rms_norm(x, g1, eps=EPS)
        q, k, v = self._split(n1 @ w["qkv"].T)
        q, k = ops.rotary(q, k, positions, self.spectrum)
        qs, ks, vs = (self._by_sequence(t) for t in (q, k, v))
        p = (qs @ ks.mT / math.sqrt(self.head_dim)).masked_fill(self.hidden, -math.inf).softmax(-1)
        a = self._by_token(p @ vs, self.heads).view(tokens, -1)
        n2, h1 = ops.rms_norm(a @ w["o"].T, g2, h0, eps=EPS)
        u = torch.relu(n2 @ w["up"].T)
        n3, h2 = ops.rms_norm(u @ w["down"].T, g3, h1, eps=EPS)
        loss, dn3, dtable = ops.linear_ce(n3, w["table"], labels, grad_scale=1.0 / tokens)
        # backward
        grads: Dict[str, torch.Tensor] = {}
        dh2, dg3 = ops.rms_norm_grad(dn3, h2, g3, eps=EPS)
        grads["down"] = dh2.T @ u
        du = (dh2 @ w["down"]) * (u > 0)
        grads["up"] = du.T @ n2
        dh1, dg2 = ops.rms_norm_grad(du @ w["up"], h1, g2, dh2, eps=EPS)
        grads["o"] = dh1.T @ a
        da = self._by_sequence((dh1 @ w["o"]).view(tokens, self.heads, self.head_dim))
        dp = da @ vs.mT
        ds = p * (dp - (dp * p).sum(-1, keepdim=True)) / math.sqrt(self.head_dim)
        dqkv = torch.empty((tokens, (self.heads + 2 * self.key_heads) * self.head_dim), dtype=torch.bfloat16, device=self.device)
        dq, dk, dv = self._split(dqkv)
        dv.copy_(self._by_token(p.mT @ da, self.key_heads))
        ops.rotary(self._by_token(ds @ ks, self.heads), self._by_token(ds.mT @ qs, self.key_heads), positions, self.spectrum, inverse=True, out=(dq, dk))
        grads["qkv"] = dqkv.T @ n1
        dx, dg1 = ops.rms_norm_grad(dqkv @ w["qkv"], h0, g1, dh1, eps=EPS)
        grads["table"] = ops.embed_grad(dx, ids, self.vocab, grad_table=dtable, accumulate=True)
        for name, g in grads.items():
            self.grads[name].add_(g)
        self.norm_grads.add_(torch.stack((dg1, dg2, dg3)))
        return loss.mean()

    def step(self, t: int, total: int, micro_batches: int, max_norm: float = 1.0, lr: float = 2e-3) -> torch.Tensor:
        """Clips what has been accumulated, updates every weight and returns the gradients' norm (on the device)."""
        norm = self.all_grads.clip(max_norm, scale=1.0 / micro_batches)
        self._adams(runner.Hyper(lr=lr, l1_coeff=1e-5, step=t, total_steps=total))
        m, v = self.norm_state
        cast.check(cast.cast_scale_adam_step(self.norms, m, v, self.norm_grads, self.norms.numel(), lr, 0.9, 0.95, 1e-8, t, True,
                                             torch.cuda.current_stream(self.device)))
        for g in self.grads.values():
            g.zero_()
        return norm


def batch(vocab: int, sequences: int, length: int, gen: torch.Generator, device):
    """Token ids that count upwards by a step of the sequence's own, and their successors; the last label is none."""
    start, by = (torch.randint(1, vocab, (sequences, 1), generator=gen, device=device) for _ in range(2))
    ids = (start + by % 7 * torch.arange(length, device=device)) % vocab
    labels = torch.full_like(ids, -1)
    labels[:, :-1] = ids[:, 1:]
    return ids.reshape(-1).int(), labels.reshape(-1).int()


def train(steps: int = 100, micro_batches: int = 4, sequences: int = 8, seed: int = 0, report=None):
    model = DecoderBlock(seed=seed)
    gen = torch.Generator(device=model.device).manual_seed(seed + 2)
    losses: List[torch.Tensor] = []
    norms: List[torch.Tensor] = []
    for t in range(1, steps + 1):
        losses.append(sum(model.accumulate(*batch(model.vocab, sequences, model.length, gen, model.device)) for _ in range(micro_batches)) / micro_batches)
        norms.append(model.step(t, steps, micro_batches))
        if report and (t % 20 == 0 or t == 1):
            report(f"step {t:4d}  loss {float(losses[-1]):.3f}  gradient norm {float(norms[-1]):.3f}")
    return [float(x) for x in torch.stack(losses)], [float(x) for x in torch.stack(norms)], model


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=100)
    train(p.parse_args().steps, report=print)
