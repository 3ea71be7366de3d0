"""cast_rms_norm, cast_rms_norm_mx and cast_rms_norm_grad against plain 64-bit evaluations.

The stored sum h is fp32 addition and one rounding to bf16, which is the rounding of the exact sum (24 >= 2 * 8 + 2 bits): the same bits.
Results are compared with the exact ones for the stored h.  A fp32 sum of n terms of one sign whose longest chain of
additions has c links is within c 2^-24 of itself; here c <= 32 (entries of a thread) + 5 (shuffles) + 32 (warps) + 2, half of which reaches the
square root's result; the root, its operand, two products and the division add 6 2^-24.  That is DELTA = 2^-18 of a result, before its
rounding to bf16 of at most half a step, 2^-8."""
import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import more_ops_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DELTA = 2.0 ** -18
HALF = 2.0 ** -8
LEAST = 2.0 ** -134          # half a step of the smallest bf16 numbers


class Banded:
    """A device array between two bands of bytes that no kernel may touch, `offset` entries off its 256-byte alignment."""

    def __init__(self, shape, dtype, offset=0, fill=None):
        self.item = torch.empty((), dtype=dtype).element_size()
        n = 1
        for s in shape:
            n *= s
        self.lo, self.hi = 256 + offset * self.item, 256 + (offset + n) * self.item
        self.raw = torch.full((self.hi + 256,), 0xA5, dtype=torch.uint8, device=DEV)
        self.t = self.raw[self.lo:self.hi].view(dtype).view(shape)
        if fill is not None:
            self.t.copy_(fill)

    def intact(self):
        return bool((self.raw[:self.lo] == 0xA5).all()) and bool((self.raw[self.hi:] == 0xA5).all())


def draw(shape, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * std).to(torch.bfloat16).to(DEV)


def weights(dim, fp32, seed=7):
    gen = torch.Generator().manual_seed(seed)
    return (1.0 + 0.3 * torch.randn(dim, generator=gen)).to(torch.float32 if fp32 else torch.bfloat16).to(DEV)


def stored_sum(x, r):
    return x if r is None else (x.float() + r.float()).to(torch.bfloat16)


def check_y(y, h, w, eps, scale_of=1.0):
    want = R.norm(h.double(), w.double(), eps)
    err = (y.double() - want).abs()
    bound = (HALF + DELTA) * want.abs() + LEAST
    assert bool((err <= bound).all()), f"worst {float((err / bound).max()):.3g} x the bound"


def check_mx(q, scales, h, w, eps):
    """Each value is the rounding of something within DELTA of the exact one, under the least scale that holds, or may, within DELTA."""
    want = R.norm(h.double(), w.double(), eps)
    T, D = want.shape
    G = (D + 31) // 32
    assert q.dtype == torch.float8_e4m3fn and scales.dtype == torch.float8_e8m0fnu and scales.shape == (T, G)
    top = torch.nn.functional.pad(want.abs(), (0, 32 * G - D)).view(T, G, 32).amax(-1)
    s = scales.double()
    assert bool((448.0 * s >= top * (1 - DELTA)).all())
    small = s == 2.0 ** -127
    assert bool(((224.0 * s < top * (1 + DELTA)) | small).all()) and bool((top[small] <= 448 * 2.0 ** -127).all())
    v = want / s.repeat_interleave(32, 1)[:, :D]
    lo, hi = R.to_e4m3((v.abs() * (1 - DELTA)).clamp(max=448)), R.to_e4m3((v.abs() * (1 + DELTA)).clamp(max=448))
    got = q.double() * torch.where(v < 0, -1.0, 1.0)
    assert bool(((got >= lo) & (got <= hi)).all())


SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (7, 61), (33, 72), (9, 128), (70, 256), (4, 257), (6, 320), (40, 768), (13, 1000), (5, 1016), (3, 1024), (3, 1032),
          (9, 2048), (4, 4096), (3, 4097), (2, 5120), (2, 8191), (3, 8192), (2, 8200), (2, 11008), (2, 16384), (1, 16392), (1, 20001), (2, 32768)]


@pytest.mark.parametrize("tokens,dim", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("fp32", [False, True])
def test_norm(tokens, dim, residual, fp32):
    eps = 1e-5
    x, r, w = draw((tokens, dim), 1), draw((tokens, dim), 2, 3.0) if residual else None, weights(dim, fp32)
    h = stored_sum(x, r)
    for offset in (0, 1) if dim <= 4097 else (0,):
        bx, bw = Banded(x.shape, x.dtype, offset, x), Banded(w.shape, w.dtype, offset, w)
        br = Banded(x.shape, x.dtype, offset, r) if residual else None
        by, bh = Banded(x.shape, x.dtype, offset), Banded(x.shape, x.dtype, offset)
        y, got = ops.rms_norm(bx.t, bw.t, br.t if residual else None, eps, out=by.t, sum_out=bh.t if residual else None)
        assert y is by.t and torch.equal(got.view(torch.int16), h.view(torch.int16))
        check_y(y, h, w, eps)
        assert all(b.intact() for b in (bx, bw, by, bh)) and torch.equal(bx.t, x)
        bq, bs = Banded(x.shape, torch.float8_e4m3fn, offset), Banded((tokens, (dim + 31) // 32), torch.float8_e8m0fnu, offset)
        cast.check(cast.cast_rms_norm_mx(bx.t, br.t if residual else None, bw.t, fp32, bq.t, bs.t, bh.t if residual else None, tokens, dim, eps,
                                         torch.cuda.current_stream()))
        check_mx(bq.t, bs.t, h, w, eps)
        assert all(b.intact() for b in (bx, bw, bq, bs, bh))
        q, scales, got = ops.rms_norm_mx(bx.t, bw.t, br.t if residual else None, eps)
        assert torch.equal(q.view(torch.uint8), bq.t.view(torch.uint8)) and torch.equal(scales.view(torch.uint8), bs.t.view(torch.uint8))
        assert torch.equal(got.view(torch.int16), h.view(torch.int16))


def check_grad(dx, dw, dy, h, w, dh, eps):
    """mean(g n) is within 2 DELTA of the mean of the magnitudes; dweight's sums have at most `tokens` + 64 links."""
    h64, dy64, w64 = h.double(), dy.double(), w.double()
    want, want_w = R.norm_grad(dy64, h64, w64, None if dh is None else dh.double(), eps)
    r = 1.0 / (h64.square().mean(-1, keepdim=True) + eps).sqrt()
    n, g = h64 * r, w64 * dy64
    size = r * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True))
    bound = HALF * want.abs() + (1 + HALF) * (2 * DELTA * size + (0 if dh is None else DELTA * dh.double().abs())) + LEAST
    err = (dx.double() - want).abs()
    assert bool((err <= bound).all()), f"dx: worst {float((err / bound).max()):.3g} x the bound"
    if dw is not None:
        bound = (DELTA + (h.shape[0] + 64) * 2.0 ** -24) * (dy64 * n).abs().sum(0) + 1e-44
        err = (dw.double() - want_w).abs()
        assert bool((err <= bound).all()), f"dw: worst {float((err / bound).max()):.3g} x the bound"


GRAD_SHAPES = SHAPES + [(1000, 64), (3001, 128), (2500, 120), (1500, 61), (700, 768), (1201, 1000), (900, 4096), (640, 4097), (600, 512), (601, 520), (333, 16384),
                        (400, 24)]


@pytest.mark.parametrize("tokens,dim", GRAD_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("fp32", [False, True])
def test_norm_grad(tokens, dim, residual, fp32):
    eps = 1e-5
    dy, h, w = draw((tokens, dim), 3, 1e-2), draw((tokens, dim), 4, 2.0), weights(dim, fp32)
    dh = draw((tokens, dim), 5, 1e-2) if residual else None
    for offset in (0, 1) if dim <= 1024 else (0,):
        bdy, bh, bw = Banded(dy.shape, dy.dtype, offset, dy), Banded(dy.shape, dy.dtype, offset, h), Banded(w.shape, w.dtype, offset, w)
        bdh = Banded(dy.shape, dy.dtype, offset, dh) if residual else None
        bdx, bdw = Banded(dy.shape, dy.dtype, offset), Banded((dim,), torch.float32, offset)
        rc, need = cast.cast_rms_norm_grad_workspace(tokens, dim)
        cast.check(rc)
        ws = Banded((need,), torch.uint8)
        args = (bdy.t, bh.t, bw.t, fp32, bdh.t if residual else None, bdx.t, bdw.t, tokens, dim, eps, ws.t, need, torch.cuda.current_stream())
        cast.check(cast.cast_rms_norm_grad(*args))
        check_grad(bdx.t, bdw.t, dy, h, w, dh, eps)
        assert all(b.intact() for b in (bdy, bh, bw, bdx, bdw, ws))
        assert torch.equal(bdy.t, dy) and torch.equal(bh.t, h)
        again, again_w = ops.rms_norm_grad(bdy.t, bh.t, bw.t, bdh.t if residual else None, eps)
        assert torch.equal(again, bdx.t) and torch.equal(again_w, bdw.t)
        alone, none = ops.rms_norm_grad(bdy.t, bh.t, bw.t, bdh.t if residual else None, eps, weight_grad=False)
        assert torch.equal(alone, bdx.t) and none is None


@pytest.mark.parametrize("dim", [64, 61, 1000, 4096, 4097, 5120])
def test_in_place(dim):
    x, r, w = draw((50, dim), 11), draw((50, dim), 12), weights(dim, False)
    y, h = ops.rms_norm(x, w, r)
    for target in (0, 1):
        xc, rc = x.clone(), r.clone()
        y2, h2 = ops.rms_norm(xc, w, rc, sum_out=rc if target else xc)
        assert h2 is (rc if target else xc) and torch.equal(h2, h) and torch.equal(y2, y)
    dx, dw = ops.rms_norm_grad(y, h, w, r)
    stream = r.clone()
    dx2, dw2 = ops.rms_norm_grad(y, h, w, stream, out=stream)
    assert dx2 is stream and torch.equal(dx2, dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("dim", [64, 61, 768, 4096, 4097])
def test_rows_outside_the_range_of_fp32_squares(dim):
    """Rows of entries near the ends of bf16's range beside ordinary ones and rows of zeros."""
    eps = 1e-5
    h, w = draw((24, dim), 21), weights(dim, True)
    size = torch.tensor([2.0 ** 100, 2.0 ** 60, 2.0 ** 125, 1.0, 0.0, 2.0 ** -40, 2.0 ** -120, 2.0 ** 64], device=DEV).repeat(3)
    h = (h.float().clamp(-3.9, 3.9) * size[:, None]).to(torch.bfloat16)
    assert bool(h.isfinite().all())
    y, _ = ops.rms_norm(h, w, eps=eps)
    check_y(y, h, w, eps)
    q, s, _ = ops.rms_norm_mx(h, w, eps=eps)
    check_mx(q, s, h, w, eps)
    ordinary = (size == 1.0).nonzero()[:, 0]
    assert torch.equal(y[ordinary], ops.rms_norm(h[ordinary].contiguous(), w, eps=eps)[0])
    dy = draw((24, dim), 22)
    dx, dw = ops.rms_norm_grad(dy, h, w, None, eps)
    check_grad(dx, dw, dy, h, w, None, eps)
    tiny = (draw((4, dim), 23).float() * 2.0 ** -110).to(torch.bfloat16)
    for e in (0.0, 1e-38):
        y, _ = ops.rms_norm(tiny, w, eps=e)
        check_y(y, tiny, w, float(torch.tensor(e, dtype=torch.float32)))


@pytest.mark.parametrize("dim", [64, 61, 1000, 4096, 4097])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_row(dim, value):
    h, w, dy = draw((40, dim), 31), weights(dim, False), draw((40, dim), 32)
    y, _ = ops.rms_norm(h, w)
    q, s, _ = ops.rms_norm_mx(h, w)
    dx, _ = ops.rms_norm_grad(dy, h, w)
    bad = h.clone()
    bad[17, 5] = value
    rest = torch.arange(40, device=DEV) != 17
    y2, _ = ops.rms_norm(bad, w)
    q2, s2, _ = ops.rms_norm_mx(bad, w)
    dx2, _ = ops.rms_norm_grad(dy, bad, w)
    for a, b in ((y, y2), (q.view(torch.uint8), q2.view(torch.uint8)), (s.view(torch.uint8), s2.view(torch.uint8)), (dx, dx2)):
        assert torch.equal(a[rest], b[rest])
    want = R.norm(bad[17:18].double(), w.double(), 1e-6)
    assert torch.equal(y2[17].isnan(), want[0].isnan()) and not bool(y2[17][y2[17].isfinite()].any())
    groups = torch.nn.functional.pad(want[0].isnan(), (0, -dim % 32)).view(-1, 32).any(1)
    assert torch.equal(s2[17].view(torch.uint8) == 255, groups)
    assert torch.equal(q2[17].float().isnan(), groups.repeat_interleave(32)[:dim])
    dx2, dw2 = ops.rms_norm_grad(torch.where(rest[:, None], dy, 0.0).to(torch.bfloat16), h, w)
    assert bool(dw2.isfinite().all())


def test_zero_groups_and_borders_of_the_scale():
    """Rows of +-1 (mean square 1, eps 0): y is the weight.  The scale doubles just above 448 times a power of two."""
    top = [448.0, 448.0 * (1 + 2.0 ** -22), 224.0, 225.0, 1.75, 1.7500002, 2.0 ** -118, 0.0]
    w = torch.zeros(32 * len(top), device=DEV)
    w[::32] = torch.tensor(top)
    w[1::32] = w[::32] / 3
    h = torch.where(torch.rand((3, len(w)), device=DEV) < 0.5, -1.0, 1.0).to(torch.bfloat16)
    q, s, _ = ops.rms_norm_mx(h, w, eps=0.0)
    assert s[0].double().tolist() == [1.0, 2.0, 0.5, 1.0, 2.0 ** -8, 2.0 ** -7, 2.0 ** -126, 2.0 ** -127]
    check_mx(q, s, h, w, 0.0)
    assert not q[:, -32:].float().any()


def test_shapes_streams_and_refusals_of_the_torch_calls():
    x, r, w = draw((4, 6, 72), 41), draw((4, 6, 72), 42), weights(72, False)
    y, h = ops.rms_norm(x, w, r)
    assert y.shape == x.shape
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, h2 = ops.rms_norm(x, w, r)
        q, s, _ = ops.rms_norm_mx(x, w, r)
        dx, dw = ops.rms_norm_grad(y2, h2, w, r)
    side.synchronize()
    assert s.shape == (4, 6, 3) and torch.equal(y, y2) and torch.equal(h, h2) and all(torch.equal(a, b) for a, b in zip((dx, dw), ops.rms_norm_grad(y, h, w, r)))
    assert ops.rms_norm(x[:0], w)[0].shape == (0, 6, 72)
    assert not ops.rms_norm_grad(x[:0], x[:0], w)[1].any()
    one, _ = ops.rms_norm(x[0, 0], w)
    assert torch.equal(one, ops.rms_norm(x, w)[0][0, 0])
    for bad, match in ((lambda: ops.rms_norm(x.transpose(0, 1), w), "not contiguous"), (lambda: ops.rms_norm(x, w[:-1]), "entries for"),
                       (lambda: ops.rms_norm(x, w.half()), "float16"), (lambda: ops.rms_norm(x.float(), w), "float32"),
                       (lambda: ops.rms_norm(x, w, r[:2]), "shape"), (lambda: ops.rms_norm(x, w, sum_out=r), "residual"),
                       (lambda: ops.rms_norm_grad(x[:1], x, w), "shape"), (lambda: ops.rms_norm(x, w, out=y[:1]), "shape")):
        with pytest.raises(ValueError, match=match):
            bad()
    with pytest.raises(cast.CastError):
        ops.rms_norm(x, w, out=x)
    with pytest.raises(cast.CastError):
        ops.rms_norm(x, w, eps=-1.0)
    assert cast.cast_rms_norm(x, None, w.cpu(), False, y, None, 24, 72, 1e-6) == B.CAST_ERR_MEMORY
    rc, need = cast.cast_rms_norm_grad_workspace(24, 72)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert cast.cast_rms_norm_grad(x, r, w, False, None, y, dw, 24, 72, 1e-6, ws, need - 1) == B.CAST_ERR_PLAN


def test_offsets_beyond_32_bits():
    """More than 2^31 entries: the last rows are the first ones again."""
    dim = 4096
    tokens = (1 << 31) // dim + 9
    x = torch.zeros((tokens, dim), dtype=torch.bfloat16, device=DEV)
    w, part = weights(dim, False), draw((8, dim), 51)
    x[:8] = part
    x[-8:] = part
    y, _ = ops.rms_norm(x, w)
    assert torch.equal(y[:8], ops.rms_norm(part, w)[0]) and torch.equal(y[-8:], y[:8]) and not bool(y[8:-8].any())
    q, s, _ = ops.rms_norm_mx(x, w)
    assert torch.equal(q[-8:].view(torch.uint8), q[:8].view(torch.uint8)) and torch.equal(s[-8:].view(torch.uint8), s[:8].view(torch.uint8))
    del y, q
    dx, dw = ops.rms_norm_grad(x, x, w)
    small, small_w = ops.rms_norm_grad(part, part, w)
    assert torch.equal(dx[:8], small) and torch.equal(dx[-8:], small) and not bool(dx[8:-8].any())
    assert torch.allclose(dw, 2 * small_w, rtol=1e-5, atol=1e-5)


def test_captured_and_replayed():
    x, r, w, dy = draw((30, 768), 61), draw((30, 768), 62), weights(768, True), draw((30, 768), 63)
    def step():
        y, h = ops.rms_norm(x, w, r)
        return (y, h) + ops.rms_norm_grad(dy, h, w, dy) + ops.rms_norm_mx(x, w, r)[:2]
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    x.copy_(draw((30, 768), 64))
    dy.copy_(draw((30, 768), 65))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, step()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("tokens,dim,fp32", [(400, 4096, False), (2000, 128, True), (300, 5120, True), (200, 1001, False), (500, 96, False), (3000, 61, True)])
def test_8_bit_values_are_those_of_the_exact_norm(tokens, dim, fp32):
    """Values and scales within 4 units in the last place of a border are decided in fp64.  The fp32 evaluation's errors are sums of some tens of
    independent roundings of half a unit at most (the sum's count half), half a unit in the mean square: 4 are eight times that.  Below e4m3's normal numbers (2^-6 of the scale) a
    value may be one step off."""
    eps = 1e-5
    x, r, w = draw((tokens, dim), 71), draw((tokens, dim), 72, 2.0), weights(dim, fp32)
    q, s, h = ops.rms_norm_mx(x, w, r, eps)
    want = R.norm(h.double(), w.double(), float(torch.tensor(eps, dtype=torch.float32)))
    groups = (dim + 31) // 32
    top = torch.nn.functional.pad(want.abs(), (0, 32 * groups - dim)).view(tokens, groups, 32).amax(-1)
    fraction, exponent = torch.frexp(top / 448)
    least = torch.ldexp(torch.ones_like(top), exponent - (fraction == 0.5).int())
    assert torch.equal(s.double(), least)
    v = want / least.repeat_interleave(32, 1)[:, :dim]
    off = q.double() - R.to_e4m3(v)
    assert not bool(off[v.abs() >= 2.0 ** -6].any()) and float(off.abs().max()) <= 2.0 ** -9


@pytest.mark.parametrize("seed", range(40))
def test_sizes_and_places_drawn_at_random(seed):
    import random
    rng = random.Random(seed)
    dim = int(2.0 ** rng.uniform(0, 13.2))
    tokens = rng.randint(1, max(1, min(3000, 400000 // dim)))
    fp32, residual = rng.random() < 0.5, rng.random() < 0.5
    x, w = draw((tokens, dim), seed), weights(dim, fp32, seed)
    r = draw((tokens, dim), seed + 1, 2.0) if residual else None
    dh = draw((tokens, dim), seed + 2) if residual else None
    dy = draw((tokens, dim), seed + 3)
    bands = {}
    for name, t in (("x", x), ("w", w), ("r", r), ("dh", dh), ("dy", dy)):
        bands[name] = None if t is None else Banded(t.shape, t.dtype, rng.choice((0, 0, 1, 4, 8, rng.randint(0, 9))), t)
    at = lambda name: None if bands[name] is None else bands[name].t  # noqa: E731
    by, bh, bdx = (Banded(x.shape, x.dtype, rng.choice((0, 0, 1, 8, rng.randint(0, 9)))) for _ in range(3))
    eps, h = 1e-5, stored_sum(x, r)
    ops.rms_norm(at("x"), at("w"), at("r"), eps, out=by.t, sum_out=bh.t if residual else None)
    check_y(by.t, h, w, eps)
    assert not residual or torch.equal(bh.t, h)
    q, s, _ = ops.rms_norm_mx(at("x"), at("w"), at("r"), eps)
    check_mx(q, s, h, w, eps)
    bdh = Banded(x.shape, x.dtype, rng.randint(0, 9), h)
    dx, dw = ops.rms_norm_grad(at("dy"), bdh.t, at("w"), at("dh"), eps, out=bdx.t)
    check_grad(dx, dw, dy, h, w, dh, eps)
    assert all(b is None or b.intact() for b in list(bands.values()) + [by, bh, bdx, bdh])
    assert torch.equal(at("x"), x) and torch.equal(bdh.t, h)


def test_calls_on_two_streams_at_once():
    """Every call has a workspace and results of its own: what runs beside it does not show."""
    sets = [(draw((700, 1536), k), draw((700, 1536), k + 50), weights(1536, True, k)) for k in range(4)]
    alone = [ops.rms_norm_grad(dy, h, w) for dy, h, w in sets]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = [[] for _ in sets]
    for _ in range(20):
        for k, (stream, (dy, h, w)) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(stream):
                got[k].append(ops.rms_norm_grad(dy, h, w))
    torch.cuda.synchronize()
    for k, (dx, dw) in enumerate(alone):
        assert all(torch.equal(a, dx) and torch.equal(b, dw) for a, b in got[k])


def check_mx_exact(q, s, h, w, eps):
    """Scales are the least powers of two, and values from 2^-6 of the scale on the rounding, of the exact norm; below, one step off at most."""
    tokens, dim = h.shape
    want = R.norm(h.double(), w.double(), float(torch.tensor(eps, dtype=torch.float32)))
    groups = (dim + 31) // 32
    top = torch.nn.functional.pad(want.abs(), (0, 32 * groups - dim)).view(tokens, groups, 32).amax(-1)
    fraction, exponent = torch.frexp(top / 448)
    least = torch.ldexp(torch.ones_like(top), exponent - (fraction == 0.5).int())
    assert torch.equal(s.double(), least)
    v = want / least.repeat_interleave(32, 1)[:, :dim]
    off = q.double() - R.to_e4m3(v)
    wrong = (off != 0) & (v.abs() >= 2.0 ** -6)
    assert not bool(wrong.any()), f"{int(wrong.sum())} values"
    assert float(off.abs().max()) <= 2.0 ** -9


@pytest.mark.parametrize("dim", [64, 120, 776, 1000, 2048, 4096, 5120, 8192, 61, 1001, 5121])
def test_8_bit_values_are_exact_where_roundings_of_the_sum_point_one_way(dim):
    """One column in eight is a multiple of 1.0 and all others so small that every addition of their squares is rounded the same way, or one entry is far larger
    than what its thread adds behind it.  The fp32 part of the sum has three roundings at most, whatever the entries."""
    eps = 1e-5
    odd = torch.full((dim,), 2.0 ** -12 * (1 + 2.0 ** -7))
    odd[:max(dim // 4, 1):8] = 1.0
    gen = torch.Generator().manual_seed(dim)
    rows = [odd, odd.flip(0)]
    for k in range(14):
        signs = torch.where(torch.rand(dim, generator=gen) < 0.5, -1.0, 1.0)
        if k % 2:
            signs = signs * torch.randn(dim, generator=gen)
        signs[(k // 2) * 8 % dim] = 4096.0
        rows.append(signs)
    h = torch.stack(rows).to(torch.bfloat16).to(DEV)
    for seed in range(max(4, 60000 // dim)):
        w = weights(dim, True, 100 + seed)
        q, s, _ = ops.rms_norm_mx(h, w, None, eps)
        check_mx_exact(q, s, h, w, eps)


def test_calls_from_two_threads_at_once():
    """Widths that take one kernel with different amounts of shared memory, each from a thread of its own: no call is refused."""
    import threading
    tokens, calls = 8, 3000
    jobs = []
    for dim in (2560, 4096):
        dy, h, dh, w = draw((tokens, dim), dim), draw((tokens, dim), dim + 1), draw((tokens, dim), dim + 2), weights(dim, True)
        want = ops.rms_norm_grad(dy, h, w, dh)
        rc, need = cast.cast_rms_norm_grad_workspace(tokens, dim)
        cast.check(rc)
        got = torch.empty_like(h), torch.empty(dim, device=DEV), torch.empty(need, dtype=torch.uint8, device=DEV)
        jobs.append((dim, (dy, h, w, dh), want, got, need, torch.cuda.Stream()))
    torch.cuda.synchronize()
    refused = []

    def run(job):
        dim, (dy, h, w, dh), _, (dx, dw, ws), need, stream = job
        call = B.load_library().cast_rms_norm_grad
        args = (dy.data_ptr(), h.data_ptr(), w.data_ptr(), 1, dh.data_ptr(), dx.data_ptr(), dw.data_ptr(), tokens, dim, 1e-6, ws.data_ptr(), need, stream.cuda_stream)
        for _ in range(calls):
            rc = call(*args)
            if rc != B.CAST_OK:
                refused.append((dim, rc))
    threads = [threading.Thread(target=run, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not refused, (len(refused), refused[0])
    for _, _, want, got, _, _ in jobs:
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dim", [64, 61, 768, 2048, 4096, 4097, 8200])
@pytest.mark.parametrize("residual", [False, True])
def test_gradients_of_rows_and_results_near_the_ends_of_the_range(dim, residual):
    """Results in the range of bf16 from factors near its ends: rows below its normal numbers, whose factor 1 / rms is beyond fp32; rows near its
    largest, whose factor is below fp32's normal numbers; gradients whose products with the row are beyond fp32 although the row's squares are not."""
    gen = torch.Generator().manual_seed(dim)
    tokens, rows, grads = 12, [], []
    for size, grad in ((2.0 ** -127, 2.0 ** -40), (2.0 ** 124, 2.0 ** 100), (2.0 ** 40, 2.0 ** 95), (2.0 ** 49, 2.0 ** 110), (1.0, 1.0), (2.0 ** -60, 2.0 ** -60)):
        for _ in range(2):
            rows.append(torch.randn(dim, generator=gen, dtype=torch.float64).clamp(-3.9, 3.9) * size)
            grads.append(torch.randn(dim, generator=gen, dtype=torch.float64).clamp(-3.9, 3.9) * grad)
    h, dy = torch.stack(rows).to(torch.bfloat16).to(DEV), torch.stack(grads).to(torch.bfloat16).to(DEV)
    assert h.shape[0] == tokens and bool(h.isfinite().all()) and bool(dy.isfinite().all())
    w = weights(dim, True)
    for t in range(tokens):
        one, grad = h[t:t + 1].contiguous(), dy[t:t + 1].contiguous()
        want, want_w = R.norm_grad(grad.double(), one.double(), w.double(), None, 0.0)
        dh = (want * 0.5).to(torch.bfloat16) if residual else None
        assert bool((want.abs() < 2.0 ** 126).all())
        dx, dw = ops.rms_norm_grad(grad, one, w, dh, 0.0)
        check_grad(dx, dw, grad, one, w, dh, 0.0)
    dx, dw = ops.rms_norm_grad(dy, h, w, None, 0.0)
    check_grad(dx, dw, dy, h, w, None, 0.0)
