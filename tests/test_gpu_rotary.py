"""cast_rotary against a plain 64-bit evaluation.

The angle in half turns is reduced in fp64 and rounded to fp32: off by at most 2^-25 half turns, and before that by |angle| 2^-51 (two products);
cosine and sine by 2 units in the last place, the two products and their sum by 3 2^-24 of |a| + |b|.  Together 2^-21 (|a| + |b|)
covers that twice over; the rounding to bf16 adds half a step, 2^-8."""
import math

import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import more_ops_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def draw(shape, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen).to(torch.bfloat16).to(DEV)


def spectrum_lists(pairs, n_axes, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return [10000.0 ** (-i / pairs) for i in range(pairs)], torch.randint(0, n_axes, (pairs,), generator=gen).tolist()


def check(got, x, positions, f, axes, adjacent, inverse):
    p = len(f)
    want = R.rotary(x.double(), positions, f, axes, adjacent, inverse)
    size = R.rotary(x.double().abs(), torch.zeros_like(positions), f, axes, adjacent, False)
    a, b = (size[..., 0:2 * p:2], size[..., 1:2 * p:2]) if adjacent else (size[..., :p], size[..., p:2 * p])
    both = torch.stack((a + b, a + b), -1).flatten(-2) if adjacent else torch.cat((a + b, a + b), -1)
    far = float(positions.double().abs().max()) * max(abs(v) for v in f)
    bound = 2.0 ** -8 * want[..., :2 * p].abs() + (2.0 ** -21 + far * 2.0 ** -50) * both
    err = (got[..., :2 * p].double() - want[..., :2 * p]).abs()
    assert bool((err <= bound).all()), f"worst {float((err / bound).max()):.3g} x the bound"
    assert torch.equal(got[..., 2 * p:], x[..., 2 * p:])


CASES = [  # tokens, heads, key heads, head_dim, pairs, axes
    (1, 1, 0, 2, 1, 1), (1, 1, 1, 64, 32, 1), (3, 2, 1, 64, 32, 2), (8, 32, 8, 128, 64, 1), (5, 7, 3, 80, 40, 3), (17, 4, 4, 96, 20, 2), (33, 3, 0, 128, 64, 3),
    (70, 1, 1, 256, 128, 1), (4, 64, 64, 128, 64, 3), (9, 5, 2, 66, 33, 1), (11, 6, 6, 72, 12, 2), (2, 300, 10, 64, 32, 1), (3, 2, 2, 1024, 512, 1), (2, 9, 3, 1000, 500, 2),
    (1000, 2, 1, 64, 24, 1), (257, 12, 12, 128, 64, 3), (3, 40, 0, 70, 35, 1)]


@pytest.mark.parametrize("tokens,heads,key_heads,head_dim,pairs,n_axes", CASES)
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(tokens, heads, key_heads, head_dim, pairs, n_axes, adjacent, inverse):
    f, axes = spectrum_lists(pairs, n_axes)
    spectrum = ops.RotarySpectrum(f, axes, adjacent)
    gen = torch.Generator().manual_seed(3)
    positions = torch.randint(-50, 5000, (n_axes, tokens), generator=gen, dtype=torch.int32).to(DEV)
    total = (heads + 2 * key_heads) * head_dim
    fused = draw((tokens + 2, total), 4)
    before = fused.clone()
    rows = fused[1:-1]
    q = rows[:, :heads * head_dim].view(tokens, heads, head_dim)
    k = rows[:, heads * head_dim:(heads + key_heads) * head_dim].view(tokens, key_heads, head_dim) if key_heads else None
    q2, k2 = ops.rotary(q, k, positions, spectrum, inverse)
    assert torch.equal(fused, before) and q2.is_contiguous()
    check(q2, q, positions, f, axes, adjacent, inverse)
    if key_heads:
        check(k2, k, positions, f, axes, adjacent, inverse)
    else:
        assert k2 is None
    # in place, inside the fused array
    got = ops.rotary(q, k, positions, spectrum, inverse, out=(q, k))
    assert got[0] is q and torch.equal(q, q2) and (k is None or torch.equal(k, k2))
    rest = slice((heads + key_heads) * head_dim, None)
    assert torch.equal(fused[0], before[0]) and torch.equal(fused[-1], before[-1]) and torch.equal(rows[:, rest], before[1:-1][:, rest])


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("offset,stride", [(0, 200), (1, 200), (8, 201), (3, 133), (0, 128)])
def test_strides_and_alignment(adjacent, offset, stride):
    """Heads first, with gaps between the rows, from and to places off the 16-byte grid."""
    tokens, heads, dim, pairs = 21, 5, 128, 48
    f, axes = spectrum_lists(pairs, 1)
    spectrum = ops.RotarySpectrum(f, axes, adjacent)
    positions = torch.arange(100, 100 + tokens, dtype=torch.int32, device=DEV)
    flat = draw((offset + heads * tokens * stride,), 5)
    x = flat[offset:].view(heads, tokens, stride)[..., :dim].transpose(0, 1)
    target = torch.full_like(flat, 7.0)
    out = target[offset:].view(heads, tokens, stride)[..., :dim].transpose(0, 1)
    q, _ = ops.rotary(x, None, positions, spectrum, out=(out, None))
    check(q, x, positions[None], f, axes, adjacent, False)
    plain, _ = ops.rotary(x.contiguous(), None, positions, spectrum)
    assert torch.equal(plain, q)
    out.fill_(7.0)
    assert bool((target == 7.0).all())          # nothing was written between the rows
    shared = x[:, :1].expand(tokens, 3, dim)
    q, _ = ops.rotary(shared, None, positions, spectrum)
    assert torch.equal(q[:, 1], plain[:, 0]) and torch.equal(q[:, 2], plain[:, 0])


def test_far_positions():
    """At a position of 2^31 - 1 the angle of the fastest pair is known to 2^31 2^-51 radians, and so is the result."""
    pairs = 64
    f = [500000.0 ** (-i / pairs) for i in range(pairs)]
    positions = torch.tensor([[0, 1, (1 << 20) - 1, 1 << 24, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31, -5]], dtype=torch.int32, device=DEV)
    x = draw((8, 4, 128), 6)
    for adjacent in (False, True):
        q, _ = ops.rotary(x, None, positions, ops.RotarySpectrum(f, None, adjacent))
        check(q, x, positions, f, [0] * pairs, adjacent, False)


def test_quarter_turns_are_exact():
    """Frequencies of a quarter turn: cosines and sines of 0, 1 and -1 move the entries about without a rounding."""
    x = draw((9, 2, 16), 7)
    positions = torch.arange(-4, 5, dtype=torch.int32, device=DEV)
    q, _ = ops.rotary(x, None, positions, ops.RotarySpectrum([math.pi / 2] * 8))
    a, b = x[..., :8], x[..., 8:]
    turned = [torch.cat(p, -1) for p in ((a, b), (-b, a), (-a, -b), (b, -a))]
    for t in range(9):
        # cos(pi/2) is formed from 0.25 turns, off by 2^-53: below half a step of every entry
        assert torch.allclose(q[t].float(), turned[(t - 4) % 4][t].float(), rtol=0, atol=1e-7)


@pytest.mark.parametrize("adjacent", [False, True])
def test_inverse_is_the_gradient(adjacent):
    """<turned x, g> = <x, g turned back>, up to the roundings of both results (half a step of each entry)."""
    tokens, heads, dim = 50, 6, 96
    spectrum = ops.RotarySpectrum.of(dim, sections=[10, 18, 20], per_axis=True, adjacent=adjacent)
    gen = torch.Generator().manual_seed(8)
    positions = torch.randint(0, 300, (3, tokens), generator=gen, dtype=torch.int32).to(DEV)
    x, g = draw((tokens, heads, dim), 9), draw((tokens, heads, dim), 10)
    y, _ = ops.rotary(x, None, positions, spectrum)
    back, _ = ops.rotary(g, None, positions, spectrum, inverse=True)
    left, right = y.double() * g.double(), x.double() * back.double()
    assert abs(float(left.sum() - right.sum())) <= (2.0 ** -8 + 2.0 ** -20) * float(left.abs().sum() + right.abs().sum())
    again, _ = ops.rotary(y, None, positions, spectrum, inverse=True)
    p = dim // 2
    pair = (lambda t: t.view(tokens, heads, p, 2).norm(dim=-1)) if adjacent else (lambda t: t.view(tokens, heads, 2, p).norm(dim=-2))
    assert bool((pair(again.double() - x.double()) <= 2 * 2.0 ** -8 * 1.5 * pair(x.double())).all())


def test_axes_outside_do_not_turn_and_values_that_are_not_finite_stay():
    x = draw((6, 2, 16), 11)
    positions = torch.arange(5, 11, dtype=torch.int32, device=DEV)
    spectrum = ops.RotarySpectrum([1.0] * 8)
    plain, _ = ops.rotary(x, None, positions, spectrum)
    spectrum.axes[3] = 7
    spectrum.axes[4] = -2
    q, _ = ops.rotary(x, None, positions, spectrum)
    for c in range(16):
        assert torch.equal(q[..., c], x[..., c] if c % 8 in (3, 4) else plain[..., c])
    spectrum = ops.RotarySpectrum([1.0] * 8)
    bad = x.clone()
    bad[2, 1, 3] = float("nan")
    q, _ = ops.rotary(bad, None, positions, spectrum)
    hit = torch.zeros_like(q, dtype=torch.bool)
    hit[2, 1, [3, 11]] = True
    assert torch.equal(q.isnan(), hit) and torch.equal(q[~hit], plain[~hit])


def test_offsets_beyond_32_bits():
    tokens, heads, dim = 20000, 130, 1024            # 2.66e9 entries, 5.3 GB
    spectrum = ops.RotarySpectrum.of(128)
    x = torch.zeros((tokens, heads, dim), dtype=torch.bfloat16, device=DEV)
    part = draw((3, heads, dim), 12)
    x[-3:] = part
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV)
    ops.rotary(x, None, positions, spectrum, out=(x, None))
    assert torch.equal(x[-3:], ops.rotary(part, None, positions[-3:], spectrum)[0]) and not bool(x[:-3].any())


def test_streams_capture_and_refusals_of_the_torch_calls():
    spectrum = ops.RotarySpectrum.of(64, sections=[20, 12])
    q, k = draw((10, 4, 64), 13), draw((10, 2, 64), 14)
    positions = torch.arange(20, dtype=torch.int32, device=DEV).view(2, 10)
    here = ops.rotary(q, k, positions, spectrum)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = ops.rotary(q, k, positions, spectrum)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(here, there))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.rotary(q, k, positions, spectrum)
    positions.add_(3)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ops.rotary(q, k, positions, spectrum)))
    assert ops.rotary(q[:0], k[:0], positions[:, :0].contiguous(), spectrum)[0].shape == (0, 4, 64)
    assert ops.rotary(q[:, :0], k, positions, spectrum)[1].shape == k.shape
    for bad, match in ((lambda: ops.rotary(q.float(), k, positions, spectrum), "float32"), (lambda: ops.rotary(q, k[:5], positions, spectrum), "shape"),
                       (lambda: ops.rotary(q, k, positions[0], spectrum), "axes"), (lambda: ops.rotary(q, k, positions.long(), spectrum), "int64"),
                       (lambda: ops.rotary(q, k, positions.t().contiguous().t(), spectrum), "not contiguous"),
                       (lambda: ops.rotary(q.transpose(1, 2), None, positions, spectrum), "columns"),
                       (lambda: ops.rotary(q[..., :60], None, positions, spectrum), "columns"),
                       (lambda: ops.rotary(q, None, positions, spectrum, out=(q, k)), "no k"),
                       (lambda: ops.rotary(q, k, positions, spectrum, out=(q, k[:, :1])), "shape")):
        with pytest.raises(ValueError, match=match):
            bad()
    with pytest.raises(cast.CastError):
        ops.rotary(q, None, positions, spectrum, out=(q.flip(0)[:, :1].expand(10, 4, 64), None))
    assert cast.cast_rotary([B.make_heads(q.cpu(), q, 4, 256, 64, 256, 64)], positions, spectrum.frequencies, spectrum.axes, 2, 32, False, False, 10,
                            64) == B.CAST_ERR_MEMORY


@pytest.mark.parametrize("seed", range(40))
def test_arrangements_drawn_at_random(seed):
    """Queries and keys of any order, gaps and places, each to a place of its own, against the 64-bit evaluation; nothing else is written."""
    import random
    rng = random.Random(seed)
    tokens, head_dim = rng.choice((1, 2, 3, 17, 150, 600)), rng.choice((8, 24, 34, 64, 80, 128, 130))
    pairs, n_axes, adjacent = rng.randint(1, head_dim // 2), rng.randint(1, 3), rng.random() < 0.5
    f, axes = spectrum_lists(pairs, n_axes, seed)
    spectrum = ops.RotarySpectrum(f, axes, adjacent)
    gen = torch.Generator().manual_seed(seed)
    positions = torch.randint(-9, 3000, (max(n_axes, 1), tokens), generator=gen, dtype=torch.int32).to(DEV)

    def place(heads, fill):
        grain = rng.choice((1, 2, 4, 8))
        head_stride = head_dim + grain * rng.randint(0, 3)
        offset = grain * rng.randint(0, 5)
        if rng.random() < 0.5:
            token_stride = heads * head_stride + grain * rng.randint(0, 4)
        else:
            token_stride = head_dim + grain * rng.randint(0, 2)
            head_stride = tokens * token_stride + grain * rng.randint(0, 3)
        n = offset + (tokens - 1) * token_stride + (heads - 1) * head_stride + head_dim
        flat = fill(n)
        return flat, flat[offset:].as_strided((tokens, heads, head_dim), (token_stride, head_stride, 1), flat.storage_offset() + offset)
    heads = [rng.randint(1, 40), rng.randint(1, 9)]
    ins = [place(h, lambda n: draw((n,), seed))[1] for h in heads]
    outs = [place(h, lambda n: torch.full((n,), 7.0, dtype=torch.bfloat16, device=DEV)) for h in heads]
    inverse = rng.random() < 0.5
    got = ops.rotary(ins[0], ins[1], positions, spectrum, inverse, out=(outs[0][1], outs[1][1]))
    for x, y, (flat, view) in zip(ins, got, outs):
        check(y, x, positions, f, axes, adjacent, inverse)
        view.fill_(7.0)
        assert bool((flat == 7.0).all())


@pytest.mark.parametrize("adjacent", [False, True])
def test_inverse_takes_every_pair_back(adjacent):
    """<turned x, g> = <x, g turned back> pair by pair, each up to the roundings of the two results: half a step of an entry, times what
    multiplies it, is 2^-8 |pair of x| |pair of g| at most on either side (the sum of two entries' products is within the product of the pairs' lengths).  Turned
    the wrong way, or not at all, a pair is off by the sine of its angle times those lengths: the oracle turned the wrong way fails."""
    tokens, heads, dim = 50, 6, 96
    sections = [10, 18, 20]
    spectrum = ops.RotarySpectrum.of(dim, sections=sections, per_axis=True, adjacent=adjacent)
    gen = torch.Generator().manual_seed(8)
    positions = torch.randint(1, 300, (3, tokens), generator=gen, dtype=torch.int32).to(DEV)
    x, g = draw((tokens, heads, dim), 9), draw((tokens, heads, dim), 10)
    p = dim // 2

    def pairs(t):
        return t.double().view(tokens, heads, p, 2) if adjacent else t.double().view(tokens, heads, 2, p).transpose(2, 3)

    def disagree(y, back):
        off = ((pairs(y) * pairs(g)).sum(-1) - (pairs(x) * pairs(back)).sum(-1)).abs()
        return off > (2 * 2.0 ** -8 + 2.0 ** -18) * pairs(x).norm(dim=-1) * pairs(g).norm(dim=-1) + 1e-30
    y, _ = ops.rotary(x, None, positions, spectrum)
    back, _ = ops.rotary(g, None, positions, spectrum, inverse=True)
    assert not bool(disagree(y, back).any())
    args = (positions, spectrum.frequencies.tolist(), spectrum.axes.tolist(), adjacent)
    assert not bool(disagree(R.rotary(x.double(), *args, inverse=False), R.rotary(g.double(), *args, inverse=True)).any())
    assert float(disagree(y, R.rotary(g.double(), *args, inverse=False)).double().mean()) > 0.4 and float(disagree(y, g).double().mean()) > 0.4


def test_a_dual_tensor_is_refused():
    from torch.autograd import forward_ad
    spectrum = ops.RotarySpectrum.of(64)
    q, positions = draw((10, 4, 64), 21), torch.arange(10, dtype=torch.int32, device=DEV)
    want, _ = ops.rotary(q, q, positions, spectrum)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        for bad in ((dual, None), (q, dual)):
            with pytest.raises(ValueError, match="forward-mode tangent"):
                ops.rotary(*bad, positions, spectrum)
        with pytest.raises(ValueError, match="forward-mode tangent"):
            ops.rms_norm(q, torch.ones(64, device=DEV), residual=dual)
        assert torch.equal(ops.rotary(q, q, positions, spectrum)[1], want)
