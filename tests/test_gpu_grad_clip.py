"""cast_grads_norm and cast_grads_clip against plain 64-bit evaluations.

A thread's sum of 32 squares has a chain of 12 links and is within 13 2^-24 of itself, the rest is fp64: the norm is within 7 2^-24 and its
rounding to fp32, NORM = 2^-20 is twice that.  A result is off by that, by the factor's rounding and the product's, and by its own rounding:
half a step of its type."""
import math

import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NORM = 2.0 ** -20
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}
F, H = torch.float32, torch.bfloat16


def arrays(counts, kinds, seed, std=1e-2, gap=0):
    """Tensors one behind the other in one buffer per type, `gap` entries apart, the gaps filled with NaN."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    flats = {}
    for kind in (F, H):
        total = sum(n + gap for n, k in zip(counts, kinds) if k == kind) + gap
        flats[kind] = [torch.full((total,), float("nan"), dtype=kind, device=DEV), gap]
    for n, k in zip(counts, kinds):
        flat, at = flats[k]
        t = flat[at:at + n]
        t.copy_(torch.randn(n, generator=gen, device=DEV) * std)
        flats[k][1] = at + n + gap
        out.append(t)
    return out, [flats[F][0], flats[H][0]]


def exact_norm(grads, scale):
    return abs(scale) * math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(norm, outs, before, max_norm, scale):
    want = exact_norm(before, scale)
    assert norm.dtype == torch.float32 and norm.shape == () and abs(float(norm) - want) <= NORM * want + 1e-44
    c = scale * min(1.0, max_norm / want if want else 1.0)
    for o, g in zip(outs, before):
        e = g.double().reshape(-1) * c
        err = (o.double().reshape(-1) - e).abs()
        assert bool((err <= (HALF[o.dtype] + NORM + 2.0 ** -22) * e.abs() + LEAST[o.dtype]).all())


SETS = [([1], "f"), ([7], "h"), ([8192], "f"), ([8193, 1, 8191], "fhf"), ([5] * 40, "fh" * 20), ([100000, 3, 70000, 16384], "hfhf"), ([4096] * 33, "f" * 33),
        ([33] * 1025, "h" * 1025), ([17, 9000] * 1100, "fh" * 1100), ([3000000, 12], "fh"), ([20000001], "h")]


@pytest.mark.parametrize("counts,kinds", SETS)
@pytest.mark.parametrize("gap", [0, 1, 64])
@pytest.mark.parametrize("max_norm,scale", [(0.5, 1.0), (1e9, 0.125), (0.25, -1.0 / 3.0)])
def test_clip(counts, kinds, gap, max_norm, scale):
    kinds = [F if k == "f" else H for k in kinds]
    grads, flats = arrays(counts, kinds, 1, gap=gap)
    before = [g.clone() for g in grads]
    whole = [f.clone() for f in flats]
    # to bf16 and fp32 places of their own
    for out_kinds in ([H] * len(kinds), [F if k == H else H for k in kinds]):
        outs, out_flats = arrays(counts, out_kinds, 2, gap=gap)
        nan = [f.isnan() for f in out_flats]
        s = ops.GradientSet(grads, outs)
        norm = s.clip(max_norm, scale)
        check(norm, outs, before, max_norm, scale)
        assert all(torch.equal(f.isnan(), n) for f, n in zip(out_flats, nan))            # nothing between the tensors
        assert all(torch.equal(f.view(torch.uint8), w.view(torch.uint8)) for f, w in zip(flats, whole))
        first = [o.clone() for o in outs]
        assert torch.equal(s.clip(max_norm, scale), norm) and all(torch.equal(a, b) for a, b in zip(first, outs))
        assert torch.equal(s.norm(scale), norm)
        s.close()
    # in place
    nan = [f.isnan() for f in flats]
    s = ops.GradientSet(grads)
    check(s.clip(max_norm, scale), grads, before, max_norm, scale)
    assert all(torch.equal(f.isnan(), n) for f, n in zip(flats, nan))


def test_what_needs_no_clipping_keeps_its_bits():
    grads, _ = arrays([9001, 77], [F, H], 3)
    before = [g.clone() for g in grads]
    s = ops.GradientSet(grads)
    norm = float(s.norm())
    s.clip(norm)
    s.clip(float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    outs = [torch.empty_like(g) for g in grads]
    ops.GradientSet(grads, outs).clip(norm)
    assert all(torch.equal(a, b) for a, b in zip(outs, before))


@pytest.mark.parametrize("size", [2.0 ** 70, 2.0 ** 120, 2.0 ** -70, 2.0 ** -120])
@pytest.mark.parametrize("kind", [F, H])
def test_squares_outside_the_range_of_fp32(size, kind):
    gen = torch.Generator(device=DEV).manual_seed(4)
    grads = [(torch.randn(n, generator=gen, device=DEV).clamp(-4, 4) * size).to(kind) for n in (20000, 5, 8192)]
    before = [g.clone() for g in grads]
    s = ops.GradientSet(grads)
    want = exact_norm(grads, 1.0)
    assert abs(float(s.norm()) - want) <= NORM * want if want < 3e38 else float(s.norm()) == float("inf")
    most = 1e-3 if size > 1 else want / 8
    most = float(torch.tensor(most, dtype=torch.float32))
    norm = s.clip(most)
    c = most / want
    for g, b in zip(grads, before):
        e = b.double() * c
        assert bool(((g.double() - e).abs() <= (HALF[kind] + NORM + 2.0 ** -22) * e.abs() + LEAST[kind]).all())
    assert float(norm) == float("inf") or abs(float(norm) - want) <= NORM * want


def test_zeros_nan_and_infinities():
    zeros = [torch.zeros(n, device=DEV) for n in (10000, 3)]
    s = ops.GradientSet(zeros)
    assert float(s.clip(0.0)) == 0.0 and not any(bool(z.any()) for z in zeros)
    grads, _ = arrays([9000, 100], [F, H], 5)
    outs = [torch.empty_like(g) for g in grads]
    s = ops.GradientSet(grads, outs)
    s.clip(0.0)
    assert not any(bool(o.any()) for o in outs)
    grads[1][3] = float("nan")
    assert math.isnan(float(s.clip(1.0))) and all(bool(o.isnan().all()) for o in outs)
    grads[1][3] = float("inf")
    assert float(s.clip(1.0)) == float("inf")
    assert math.isnan(float(outs[1][3])) and not bool(outs[0].any()) and int(outs[1].isnan().sum()) == 1


def test_a_set_for_norms_alone_and_the_same_tensor_twice():
    g = torch.full((5000,), 0.5, device=DEV)
    rc, handle = cast.cast_grads_create([B.make_grad(g, None, 5000, False, False)] * 2)
    cast.check(rc)
    rc, need = cast.cast_grads_workspace(handle)
    ws, norm = torch.empty(need + 64, dtype=torch.uint8, device=DEV), torch.zeros(1, device=DEV)
    ws[need:] = 77
    cast.check(cast.cast_grads_norm(handle, 2.0, norm, ws, need, torch.cuda.current_stream()))
    assert float(norm) == pytest.approx(100.0, rel=1e-6) and bool((ws[need:] == 77).all())
    assert cast.cast_grads_clip(handle, 1.0, 1.0, norm, ws, need) == B.CAST_ERR_NULL
    assert cast.cast_grads_norm(handle, 1.0, norm, ws, need - 1) == B.CAST_ERR_PLAN
    assert cast.cast_grads_norm(handle, float("nan"), norm, ws, need) == B.CAST_ERR_HYPER
    assert cast.cast_grads_norm(handle, 1.0, None, ws, need) == B.CAST_ERR_NULL
    assert cast.cast_grads_norm(handle, 1.0, ws, ws, need) == B.CAST_ERR_ALIAS
    assert cast.cast_grads_norm(handle, 1.0, norm.cpu(), ws, need) == B.CAST_ERR_MEMORY
    cast.check(cast.cast_grads_destroy(handle))
    assert cast.cast_grads_create([B.make_grad(g.cpu(), None, 5000, False, False)])[0] == B.CAST_ERR_MEMORY


def test_more_than_32_bits_of_entries():
    n = (1 << 32) + 8195
    g = torch.zeros(n, dtype=H, device=DEV)
    g[:3] = 2.0
    g[-4:] = 1.0
    s = ops.GradientSet([g])
    assert float(s.norm()) == 4.0
    s.clip(2.0)
    assert bool((g[:3] == 1.0).all()) and bool((g[-4:] == 0.5).all()) and not bool(g[3:-4].any())


def test_shapes_streams_capture_and_refusals():
    a, b, empty = torch.randn((30, 40), device=DEV), torch.randn(100, device=DEV).to(H), torch.empty(0, device=DEV)
    outs = [torch.empty((40, 30), dtype=H, device=DEV), torch.empty(100, device=DEV), empty]
    s = ops.GradientSet([a, b, empty], outs)
    norm = s.clip(1.0)
    kept = [o.clone() for o in outs]
    check(norm, outs[:2], [a, b], 1.0, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = s.clip(1.0)
    side.synchronize()
    assert torch.equal(there, norm) and all(torch.equal(x, y) for x, y in zip(kept, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.clip(1.0)
    a.mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    check(got, outs[:2], [a, b], 1.0, 1.0)
    assert float(ops.GradientSet([empty]).clip(1.0)) == 0.0
    for bad, match in ((lambda: ops.GradientSet([a.t()]), "not contiguous"), (lambda: ops.GradientSet([a.half()]), "float16"),
                       (lambda: ops.GradientSet([a], [b]), "entries"), (lambda: ops.GradientSet([a], []), "outs"), (lambda: ops.GradientSet([a, b.cpu()]), "CUDA")):
        with pytest.raises(ValueError, match=match):
            bad()
    with pytest.raises(cast.CastError):
        ops.GradientSet([a, a])
    with pytest.raises(cast.CastError):
        s.clip(-1.0)
    s.close()
    with pytest.raises(ValueError, match="closed"):
        s.norm()


def test_gradients_of_a_plan_are_clipped_in_place_ahead_of_its_step():
    from paper_2509_25996_b200 import runner
    state = runner.DeviceModelState([(96, 64), (32, 128)], seed=1, device=DEV)
    before = [m.g.clone() for m in state.mats]
    norm = exact_norm(before, 0.5)
    check(state.clip_gradients(norm / 4, scale=0.5), [m.g for m in state.mats], before, float(torch.tensor(norm / 4, dtype=torch.float32)), 0.5)
    again = [m.g.clone() for m in state.mats]
    assert float(state.clip_gradients(norm)) < norm / 3 and all(torch.equal(m.g, g) for m, g in zip(state.mats, again))
    state.step(runner.Hyper(), B.CAST_F_RESELECT)
    state.set_nm(1, 4)
    assert float(state.clip_gradients(norm)) < norm / 3
    state.close()


@pytest.mark.parametrize("n", [3, 50])
def test_norm_and_workspace_inside_the_tensors_are_refused(n):
    """The norm and the sums would be written over entries that other threads still read."""
    flat = torch.ones((2 * n, 4096), device=DEV)
    before = flat.clone()
    grads, outs = flat[:n], flat[n:]
    norm, apart = torch.zeros(64, device=DEV), torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    rc, handle = cast.cast_grads_create([B.make_grad(g[16:-16], o[16:-16], 4064, False, False) for g, o in zip(grads, outs)])
    cast.check(rc)
    rc, need = cast.cast_grads_workspace(handle)
    cast.check(rc)
    stream = torch.cuda.current_stream()

    def norm_call(place, ws):
        return cast.cast_grads_norm(handle, 1.0, place, ws, need, stream)

    def clip_call(place, ws):
        return cast.cast_grads_clip(handle, 1.0, 1.0, place, ws, need, stream)
    launched = cast.cast_kernel_launch_count()
    for call in (norm_call, clip_call):
        for t in (grads[0], grads[n // 2], grads[n - 1]):
            for at in (16, 2000, 4079):
                assert call(t[at:], apart) == B.CAST_ERR_ALIAS
            for at in (12, 1024, 4076):              # its end in the tensor, all of it (or its beginning), its beginning
                assert call(norm, t.data_ptr() + 4 * at) == B.CAST_ERR_ALIAS
    for t in (outs[0], outs[n - 1]):
        assert clip_call(t[16:], apart) == B.CAST_ERR_ALIAS and clip_call(t[4079:], apart) == B.CAST_ERR_ALIAS
        assert clip_call(norm, t[1024:]) == B.CAST_ERR_ALIAS
    assert cast.cast_kernel_launch_count() == launched and torch.equal(flat, before)
    # between the tensors, and a result's place for the norm alone
    want = math.sqrt(n * 4064)
    for place in (grads[0][15:], grads[1], grads[n - 1][4080:], outs[0][16:]):
        cast.check(norm_call(place, apart))
        assert abs(float(place[0]) - want) <= NORM * want
        place[0] = 1.0
    for place in (outs[0][15:], outs[n - 1][4080:]):
        cast.check(clip_call(place, apart))
        assert abs(float(place[0]) - want) <= NORM * want
    cast.check(cast.cast_grads_destroy(handle))


def test_gradients_of_a_plan_are_clipped_on_the_stream_of_its_step():
    """The clipping waits behind what its stream holds, like the step behind it; nothing of it is on the current stream."""
    from paper_2509_25996_b200 import runner
    state = runner.DeviceModelState([(96, 64), (32, 128)], seed=1, device=DEV)
    before = [m.g.clone() for m in state.mats]
    norm = exact_norm(before, 1.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for m, g in zip(state.mats, before):
            m.g.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)          # some 10 ms
            for m, g in zip(state.mats, before):
                m.g.copy_(g)
        got = state.clip_gradients(norm / 4, stream=stream)
        state.step(runner.Hyper(), B.CAST_F_RESELECT, stream=stream)
        side.synchronize()
        check(got, [m.g for m in state.mats], before, float(torch.tensor(norm / 4, dtype=torch.float32)), 1.0)
    state.close()
