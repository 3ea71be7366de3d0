"""The example that runs the norms, rotary positions and clipping together with the framework's step, embedding and loss: it runs,
and its gradients are those of the model."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def reference_loss(model, w, norms, ids, labels):
    """The mean loss in fp64, written down again with torch's own operators."""
    L, hd, H, K = model.length, model.head_dim, model.heads, model.key_heads

    def norm(x, g):
        return torch.nn.functional.rms_norm(x, (x.shape[-1],), g, 1e-5)

    pairs = hd // 2
    angle = (model.positions.double()[model.spectrum.axes.long()] * model.spectrum.frequencies[:, None]).T[None, :, None]

    def turn(x):
        z = torch.complex(x[..., :pairs], x[..., pairs:]) * torch.polar(torch.ones_like(angle), angle)
        return torch.cat((z.real, z.imag), -1)
    h = w["table"][ids.long()]
    qkv = (norm(h, norms[0]) @ w["qkv"].T).view(-1, L, H + 2 * K, hd)
    q, k, v = qkv.split((H, K, K), 2)
    q, k, v = (t.transpose(1, 2) for t in (turn(q), turn(k).repeat_interleave(H // K, 2), v.repeat_interleave(H // K, 2)))
    a = torch.nn.functional.scaled_dot_product_attention(q, k, v, is_causal=True).transpose(1, 2).reshape(-1, H * hd)
    h = h + a @ w["o"].T
    h = h + torch.relu(norm(h, norms[1]) @ w["up"].T) @ w["down"].T
    logits = norm(h, norms[2]) @ w["table"].T
    return torch.nn.functional.cross_entropy(logits, labels.long(), ignore_index=-1, reduction="sum") / ids.numel()


def test_gradients_are_those_of_the_model():
    """Between a gradient and the exact one lie at most 26 roundings to bf16 (13 tensors on the way forward, as many back), each of at most half a
    step, 2^-8 of its tensor's norm; the layers between them have gains near 1 at these sizes (norms before every product, weights of
    1/sqrt(columns)), so that 26 2^-8 bounds their sum in norm.  A missing or doubled term is of the order of 1."""
    import train_decoder_block as ex
    model = ex.DecoderBlock(seed=3)
    gen = torch.Generator(device=model.device).manual_seed(4)
    batches = [ex.batch(model.vocab, 4, model.length, gen, model.device) for _ in range(2)]
    model.norms.copy_(1 + 0.3 * torch.randn(model.norms.shape, generator=gen, device=model.device))
    losses = [model.accumulate(*b) for b in batches]
    w = {name: t.double().requires_grad_() for name, t in model.weights().items()}
    norms = model.norms.double().requires_grad_()
    want = [reference_loss(model, w, norms, *b) for b in batches]
    sum(want).backward()
    tol = 26 * 2.0 ** -8
    for got, exact in zip(losses, want):
        assert abs(float(got) - float(exact.detach())) <= tol * float(exact.detach())
    for name, t in w.items():
        err = float(torch.linalg.norm(model.grads[name].double() - t.grad) / torch.linalg.norm(t.grad))
        assert err <= tol, (name, err)
    for i in range(3):
        err = float(torch.linalg.norm(model.norm_grads[i].double() - norms.grad[i]) / torch.linalg.norm(norms.grad[i]))
        assert err <= tol, (i, err)
    # the clipped gradients: one factor for all of them, from the norm of the mean over the micro-batches
    before = [g.clone() for g in list(model.grads.values()) + [model.norm_grads]]
    exact = 0.5 * math.sqrt(sum(float(g.double().square().sum()) for g in before))
    norm = model.all_grads.clip(exact / 3, scale=0.5)
    assert abs(float(norm) - exact) <= 2.0 ** -20 * exact
    for out, g in zip([m.g for m in model.mats] + [model.norm_grads], before):
        err = (out.double() - g.double() / 6).abs()
        assert bool((err <= (2.0 ** -8 + 2.0 ** -18) * g.double().abs() / 6 + 2.0 ** -134).all())


def test_it_trains():
    import train_decoder_block as ex
    losses, norms, model = ex.train(steps=12)
    assert all(math.isfinite(x) for x in losses + norms) and all(n > 0 for n in norms)
    for m in model.pruned.mats:
        assert int((m.w_fwd.reshape(-1, 4) != 0).sum(1).max()) <= 2
    assert bool(model.norms.isfinite().all()) and not bool((model.norms == 1).all())
    assert not any(bool(g.any()) for g in model.grads.values()) and not bool(model.norm_grads.any())
