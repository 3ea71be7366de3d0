"""cast_embed and cast_embed_grad against plain 64-bit evaluations.

Forward: bf16(fl32(scale * entry)): a product of a 24- and an 8-bit significand is exact in fp64, so the two roundings
can be repeated exactly and the bits have to agree.
Gradient of a row with n tokens: fp32 sums in some order are within n 2^-24 sum|x| of the exact sum; the product with the
scale adds 2^-24, the rounding to bf16 2^-9 of the result:
    |cuda - exact| <= 2^-8 |exact| + (n + 2) 2^-23 |scale| sum|x|"""
import numpy as np
import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import gpu_util as U

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def draw(shape, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * std).to(torch.bfloat16)


def draw_ids(tokens, vocab, seed, kind):
    gen = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((tokens,), vocab // 2, dtype=torch.int32)
    if kind == "hot":          # half of the tokens on one row, the rest skewed
        ids = (torch.rand(tokens, generator=gen) ** 4 * vocab).int().clamp(max=vocab - 1)
        ids[torch.rand(tokens, generator=gen) < 0.5] = vocab - 1
    elif kind == "sorted":
        ids = torch.sort(torch.randint(0, vocab, (tokens,), generator=gen)).values.flip(0).int()
    else:
        ids = torch.randint(0, vocab, (tokens,), generator=gen).int()
    bad = torch.tensor([-1, vocab, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    where = torch.rand(tokens, generator=gen) < 0.05
    ids[where] = bad[torch.randint(0, 4, (int(where.sum()),), generator=gen)]
    return ids


def guarded(t, offset=0):
    g = U.Guarded(t.numel() + offset, t.dtype, DEV)
    g.view[offset:].copy_(t.reshape(-1))
    return g, g.view[offset:]


@pytest.mark.parametrize("tokens,vocab,dim,offset", [(1, 5, 8, 0), (1, 1, 1, 0), (7, 50, 61, 0), (33, 100, 64, 1), (300, 257, 768, 0), (1025, 40, 4096, 0),
                                                     (5, 9, 13000, 0)])
@pytest.mark.parametrize("scale", [1.0, -0.7071])
def test_embed(tokens, vocab, dim, offset, scale):
    table, ids = draw((vocab, dim), 1), draw_ids(tokens, vocab, 2, "any")
    gt, tv = guarded(table, offset)
    go = U.Guarded(tokens * dim + offset, torch.bfloat16, DEV)
    cast.check(cast.cast_embed(tv, ids.to(DEV), go.view[offset:], tokens, vocab, dim, scale, torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert gt.intact() and go.intact()
    valid = (ids >= 0) & (ids < vocab)
    want = torch.zeros((tokens, dim), dtype=torch.bfloat16)
    want[valid] = (table[ids[valid].long()].double() * float(np.float32(scale))).float().to(torch.bfloat16)
    assert torch.equal(go.view[offset:].cpu().reshape(tokens, dim).view(torch.int16), want.view(torch.int16))


def reference(grad, ids, vocab, scale, base=None):
    valid = (ids >= 0) & (ids < vocab)
    at = ids[valid].long()
    x = grad[valid].double()
    s = float(np.float32(scale))
    total = torch.zeros((vocab, grad.shape[1]), dtype=torch.float64).index_add_(0, at, x) * s
    size = torch.zeros((vocab, grad.shape[1]), dtype=torch.float64).index_add_(0, at, x.abs()) * abs(s)
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    if base is not None:
        total, size, count = total + base.double(), size + base.double().abs(), count + 1
    return total, 2.0 ** -8 * total.abs() + (count + 2) * 2.0 ** -23 * size, count


CASES = [(1, 1, 8, "any"), (1, 7, 61, "any"), (63, 40, 64, "one"), (64, 40, 64, "one"), (65, 40, 64, "one"), (127, 3, 72, "hot"), (1000, 400, 768, "any"),
         (1024, 50, 8, "any"), (1025, 50, 16, "hot"), (2048, 5000, 24, "sorted"), (5000, 90, 61, "hot"), (16384, 3000, 32, "hot"), (16385, 30, 40, "any"),
         (20000, 10, 8, "one"), (40000, 100000, 8, "hot"), (270000, 500, 8, "hot"),
         (3000, 5, 4096, "hot"), (5000, 3, 300, "one"), (9000, 6, 777, "hot")]


@pytest.mark.parametrize("tokens,vocab,dim,kind", CASES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(tokens, vocab, dim, kind, accumulate):
    grad, ids, base = draw((tokens, dim), 3), draw_ids(tokens, vocab, 4, kind), draw((vocab, dim), 5)
    scale = 0.7071
    want, bound, count = reference(grad, ids, vocab, scale, base if accumulate else None)
    gg, gv = guarded(grad)
    gt, tv = guarded(base)
    rc, need = cast.cast_embed_grad_workspace(tokens, dim)
    cast.check(rc)
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    ws[need:] = 77
    cast.check(cast.cast_embed_grad(gv, ids.to(DEV), tv, tokens, vocab, dim, scale, accumulate, ws, need, torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert gg.intact() and gt.intact() and bool((ws[need:] == 77).all())
    got = tv.cpu().reshape(vocab, dim)
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), f"worst {float((err / bound.clamp(min=1e-300)).max()):.3g} x the bound"
    untouched = (count[:, 0] == (1 if accumulate else 0)).nonzero()[:, 0]
    if accumulate:
        assert torch.equal(got[untouched].view(torch.int16), base[untouched].view(torch.int16))
    else:
        assert not got[untouched].view(torch.int16).any()


@pytest.mark.parametrize("dim", [61, 64])
def test_embed_grad_off_alignment_and_repeatable(dim):
    tokens, vocab = 3000, 70
    grad, ids = draw((tokens, dim), 6), draw_ids(tokens, vocab, 7, "hot")
    want, bound, _ = reference(grad, ids, vocab, 1.0)
    gg, gv = guarded(grad, 1)
    gt = U.Guarded(vocab * dim + 3, torch.bfloat16, DEV)
    rc, need = cast.cast_embed_grad_workspace(tokens, dim)
    got = []
    for _ in range(2):
        ws = torch.randint(0, 255, (need,), dtype=torch.uint8, device=DEV)
        cast.check(cast.cast_embed_grad(gv, ids.to(DEV), gt.view[3:], tokens, vocab, dim, 1.0, False, ws, need, torch.cuda.current_stream()))
        got.append(gt.view[3:].cpu().reshape(vocab, dim))
    assert gg.intact() and gt.intact()
    assert bool(((got[0].double() - want).abs() <= bound).all())
    assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))


def test_values_of_dropped_tokens_do_not_matter():
    vocab, dim = 20, 64
    grad = draw((6, dim), 8).to(DEV)
    ids = torch.tensor([3, -1, 3, 20, 0, 19], dtype=torch.int32, device=DEV)
    clean = ops.embed_grad(grad, ids, vocab)
    grad[1] = float("nan")
    grad[3] = float("inf")
    assert torch.equal(ops.embed_grad(grad, ids, vocab), clean)


def test_gradient_is_the_transpose_of_the_lookup():
    """<embed(E), G> = <E, embed_grad(G)> for the linear map, which differences of the lookup give exactly: values are
    small integers, so that nothing is rounded on either side."""
    gen = torch.Generator().manual_seed(9)
    tokens, vocab, dim = 500, 60, 40
    ids = draw_ids(tokens, vocab, 10, "any").to(DEV)
    e0 = torch.randint(-3, 4, (vocab, dim), generator=gen).to(torch.bfloat16).to(DEV)
    step = torch.randint(-3, 4, (vocab, dim), generator=gen).to(torch.bfloat16).to(DEV)
    g = torch.randint(-1, 2, (tokens, dim), generator=gen).to(torch.bfloat16).to(DEV)
    moved = (ops.embed(e0 + step, ids, 2.0).double() - ops.embed(e0, ids, 2.0).double())
    assert float((moved * g.double()).sum()) == float((step.double() * ops.embed_grad(g, ids, vocab, 2.0).double()).sum())


def test_offsets_beyond_32_bits():
    """A table of more than 2^31 entries (5.7 GB): rows at both ends."""
    vocab, dim = 700001, 4096
    table = torch.zeros((vocab, dim), dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([0, vocab - 1, 600000, vocab - 1, vocab], dtype=torch.int32, device=DEV)
    for r in (0, 600000, vocab - 1):
        table[r] = draw((dim,), r).to(DEV)
    out = ops.embed(table, ids)
    assert torch.equal(out[:4], table[ids[:4].long()]) and not out[4].any()
    table.fill_(7.0)
    ops.embed_grad(out, ids, vocab, grad_table=table)
    assert torch.equal(table[600000], out[2])
    assert torch.equal(table[vocab - 1], (out[1].float() * 2).to(torch.bfloat16)) and torch.equal(table[0], out[0])
    assert float(table[1:600000].abs().max()) == 0.0 and float(table[600001:vocab - 1].abs().max()) == 0.0


def test_side_stream_and_shapes_of_the_torch_calls():
    vocab, dim = 100, 72
    table, ids = draw((vocab, dim), 11).to(DEV), draw_ids(24, vocab, 12, "any").reshape(4, 6).to(DEV)
    here = ops.embed(table, ids, 3.0)
    assert here.shape == (4, 6, dim)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = ops.embed(table, ids, 3.0)
        grad = ops.embed_grad(there, ids, vocab)
    s.synchronize()
    assert torch.equal(here, there) and torch.equal(grad, ops.embed_grad(here, ids, vocab))
    assert ops.embed(table, ids[:0]).shape == (0, 6, dim)
    assert not ops.embed_grad(here[:0], ids[:0], vocab).any()
    with pytest.raises(ValueError, match="not contiguous"):
        ops.embed(table.t().contiguous().t(), ids)
    with pytest.raises(ValueError, match="int64"):
        ops.embed(table, ids.long())
    with pytest.raises(ValueError, match="accumulate"):
        ops.embed_grad(here, ids, vocab, accumulate=True)
    with pytest.raises(ValueError, match="grad_out"):
        ops.embed_grad(here[:2].contiguous(), ids, vocab)


def test_host_memory_is_refused():
    x = torch.zeros((4, 8), dtype=torch.bfloat16, device=DEV)
    y = torch.zeros((4, 8), dtype=torch.bfloat16, device=DEV)
    ids = torch.zeros(4, dtype=torch.int32)
    assert cast.cast_embed(x, ids, y, 4, 4, 8) == B.CAST_ERR_MEMORY


@pytest.mark.parametrize("tokens,dim", [(40, 64), (40, 61), (2000, 64), (2000, 61)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_not_a_number_stays_in_its_row(tokens, dim, value):
    vocab = 30
    ids = draw_ids(tokens, vocab, 14, "any").to(DEV)
    table, grad = draw((vocab, dim), 15).to(DEV), draw((tokens, dim), 16).to(DEV)
    out, back = ops.embed(table, ids), ops.embed_grad(grad, ids, vocab)
    at = int(((ids >= 0) & (ids < vocab)).nonzero()[3])
    row = int(ids[at])
    table[row, 9] = value
    grad[at, 9] = value
    out2, back2 = ops.embed(table, ids), ops.embed_grad(grad, ids, vocab)
    hit = ids == row
    assert torch.equal(out2[~hit], out[~hit]) and not out2[hit][:, 9].isfinite().any()
    rest = torch.arange(vocab, device=DEV) != row
    assert torch.equal(back2[rest], back[rest]) and not bool(back2[row, 9].isfinite())
    cols = torch.arange(dim, device=DEV) != 9
    assert torch.equal(back2[row, cols], back[row, cols])
