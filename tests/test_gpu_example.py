"""The example that runs the embedding, the pruned layers, the linear cross entropy, the tied gradient and the orthogonalised
update together: it learns, its masks stay 2:4, and its tied gradient is the sum of both parts."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_training_reduces_the_loss():
    import train_tied_lm as ex
    losses, model = ex.train(steps=120)
    assert all(math.isfinite(x) for x in losses)
    first, last = sum(losses[:5]) / 5, sum(losses[-5:]) / 5
    assert first > 5.0 and last < 0.7 * first          # ln(1000) = 6.9 at the start
    for m in model.pruned.mats:
        kept = (m.w_fwd.reshape(-1, 4) != 0).sum(1)
        assert int(kept.max()) <= 2
    s = torch.linalg.svdvals(model.w3.double())
    assert bool(torch.isfinite(s).all())


def test_tied_gradient_is_the_sum_of_both_parts(monkeypatch):
    """The table's gradient of one step against fp64 autograd through the lookup and the head, from the step's own hidden
    states and gradients (so that what torch rounds in between is on both sides).  Four roundings to bf16 of at most 2^-9
    each lie between the two (exponentials, scaled hidden states, the head's part, the sum): 4 2^-9 in norm."""
    import train_tied_lm as ex
    from paper_2509_25996_b200 import ops
    seen = {}
    linear_ce, embed_grad = ops.linear_ce, ops.embed_grad

    def spy_ce(z, table, labels, **kw):
        seen["z"], seen["table"] = z.clone(), table.clone()
        return linear_ce(z, table, labels, **kw)

    def spy_grad(dx, ids, vocab, scale, **kw):
        seen["dx"] = dx.clone()
        return embed_grad(dx, ids, vocab, scale, **kw)
    monkeypatch.setattr(ops, "linear_ce", spy_ce)
    monkeypatch.setattr(ops, "embed_grad", spy_grad)
    model = ex.TiedModel(vocab=300, d=128, ffn=256, seed=5)
    gen = torch.Generator(device=model.device).manual_seed(1)
    ids, labels = ex.batch(300, 4, 50, gen, model.device)
    model.step(ids, labels, 1, 10)
    head, lookup = seen["table"].double().requires_grad_(), seen["table"].double().requires_grad_()
    loss = torch.nn.functional.cross_entropy(seen["z"].double() @ head.T, labels.long(), ignore_index=-1, reduction="sum") / ids.numel()
    loss.backward()
    (lookup[ids.long()] * math.sqrt(128)).backward(seen["dx"].double())
    want = head.grad + lookup.grad
    err = float(torch.linalg.norm(model.table.mats[0].g.double() - want) / torch.linalg.norm(want))
    assert err <= 4 * 2.0 ** -9, err
