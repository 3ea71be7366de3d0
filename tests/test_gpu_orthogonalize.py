"""cast_orthogonalize against the iteration in 64 bits.

Tolerance on |out - exact|_F / |exact|_F: the result is rounded to bf16 (2^-9 at most); in each step three operands are rounded to
fp16 (2^-12 each at most, random in sign) and enter with factors of up to |b| + 2 |c| ~ 9 against singular values near 1,
but only in directions that are not small, and partly undone by the steps that follow (the map is flat around 1): 1.2 2^-11 per step.
    2^-9 + 1.2 steps 2^-11       (4.9e-3 for five steps)
Single matrices of a few entries have no averaging of signs: 4 times that."""
import math

import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import gpu_util as U

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
QUINTIC = (3.4445, -4.7750, 2.0315)


def draw(n, rows, cols, seed, dtype=torch.float32, size=1e-3, rank=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.randn((n, rows, cols), generator=g, device=DEV)
    if rank:
        u = 0.02 * u + torch.randn((n, rows, rank), generator=g, device=DEV) @ torch.randn((n, rank, cols), generator=g, device=DEV)
    return [x.contiguous() for x in (u * size).to(dtype)]


def exact(u, coeffs, steps, eps=1e-7, scale=1.0):
    x = u.double()
    if u.shape[0] > u.shape[1]:
        x = x.T
    norm = torch.linalg.norm(x) + eps
    x = x / norm if float(norm) > 0 else x
    for k in range(steps):
        a, b, c = coeffs[3 * k:3 * k + 3] if len(coeffs) > 3 else coeffs
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return scale * (x.T if u.shape[0] > u.shape[1] else x)


def distance(got, want):
    return float(torch.linalg.norm(got.double() - want) / torch.linalg.norm(want))


def tolerance(steps, entries=1 << 30):
    return (2.0 ** -9 + 1.2 * steps * 2.0 ** -11) * (4 if entries < 4096 else 1)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 300), (64, 64), (65, 200), (200, 65), (127, 129), (128, 128), (256, 256), (257, 255), (300, 1000), (1000, 300),
          (768, 768), (768, 3000), (2000, 768), (1500, 1501)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shapes(rows, cols, dtype):
    u = draw(2, rows, cols, rows + cols, dtype)
    before = [x.clone() for x in u]
    guards = [U.Guarded(rows * cols, torch.bfloat16, DEV) for _ in u]
    rc, need = cast.cast_orthogonalize_workspace(2, rows, cols)
    cast.check(rc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)        # NaN patterns: nothing may be read before it is written
    cast.check(cast.cast_orthogonalize(u, dtype == torch.bfloat16, [g.view for g in guards], rows, cols, None, 5, 1e-7, 1.5, ws, need,
                                       torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert all(g.intact() for g in guards) and bool((ws[need:] == 255).all())
    assert cast.cast_product_failures() == (0, 0)
    assert all(torch.equal(a, b) for a, b in zip(u, before))
    for x, g in zip(u, guards):
        assert distance(g.view.reshape(rows, cols), exact(x, QUINTIC, 5, scale=1.5)) <= tolerance(5, rows * cols)


@pytest.mark.parametrize("n,rows,cols", [(1, 64, 5000), (1, 5000, 72), (3, 130, 8192), (1, 100, 6001), (2, 9000, 33), (1, 513, 7000), (66, 70, 4100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_and_narrow(n, rows, cols, dtype):
    """Few tiles with a long sum each: A is summed in splits.  (66: a full group and one of two, which takes other splits.)"""
    u = draw(n, rows, cols, rows, dtype)
    guards = [U.Guarded(rows * cols, torch.bfloat16, DEV) for _ in u]
    rc, need = cast.cast_orthogonalize_workspace(n, rows, cols)
    cast.check(rc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    cast.check(cast.cast_orthogonalize(u, dtype == torch.bfloat16, [g.view for g in guards], rows, cols, None, 5, 1e-7, 1.0, ws, need,
                                       torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert all(g.intact() for g in guards) and bool((ws[need:] == 255).all())
    for i in {0, n // 2, n - 1}:
        assert distance(guards[i].view.reshape(rows, cols), exact(u[i], QUINTIC, 5)) <= tolerance(5)
    assert torch.equal(guards[n - 1].view.reshape(rows, cols), ops.orthogonalize(u)[n - 1])


@pytest.mark.parametrize("rows,cols,rank", [(512, 512, 8), (400, 1200, 4), (1200, 400, 16), (1024, 1024, 1)])
def test_low_rank_updates(rows, cols, rank):
    """Spectra as momenta have them: few strong directions over weak ones, which the iteration amplifies."""
    for u in draw(2, rows, cols, rank, rank=rank):
        assert distance(ops.orthogonalize([u])[0], exact(u, QUINTIC, 5)) <= tolerance(5)


def test_singular_values_of_the_result():
    u = draw(1, 300, 700, 3)[0]
    s = torch.linalg.svdvals(ops.orthogonalize([u])[0].double())
    assert 0.65 < float(s.min()) and float(s.max()) < 1.25        # what the quintic maps (0.02, 1] to after five steps, and bf16


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_steps_and_coefficients(steps):
    schedule = [(3.0, -4.0, 1.9), (3.4445, -4.7750, 2.0315), (3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5)] + [(15 / 8, -10 / 8, 3 / 8)] * 3
    sigma = torch.linspace(0, 1, 10001, dtype=torch.float64)
    for a, b, c in schedule:                 # the documented condition on coefficients: singular values stay below 8
        sigma = sigma * (a + b * sigma ** 2 + c * sigma ** 4)
        assert float(sigma.abs().max()) < 8
    flat = [float(torch.tensor(v, dtype=torch.float32)) for t in schedule[:steps] for v in t]
    for rows, cols in ((200, 330), (330, 200)):
        u = draw(1, rows, cols, steps)[0]
        assert distance(ops.orthogonalize([u], steps=steps, coeffs=flat)[0], exact(u, flat, steps)) <= tolerance(steps)


def test_many_matrices_in_groups():
    """More matrices than one launch takes, and than the workspace holds at a time."""
    u = draw(70, 40, 56, 5)
    out = ops.orthogonalize(u)
    for i in (0, 1, 63, 64, 69):
        assert distance(out[i], exact(u[i], QUINTIC, 5)) <= tolerance(5, 0)
        assert torch.equal(out[i], ops.orthogonalize([u[i]])[0])
    u = draw(3, 4096, 11008, 6, torch.bfloat16)
    out = ops.orthogonalize(u)
    assert distance(out[2], exact(u[2], QUINTIC, 5)) <= tolerance(5)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e18, 3e37])
def test_magnitudes(size):
    u = draw(1, 200, 256, 7, size=1.0)[0] * size
    assert bool(torch.isfinite(u).all())
    assert distance(ops.orthogonalize([u], eps=0.0)[0], exact(u, QUINTIC, 5, eps=0.0)) <= tolerance(5)


def test_zero_and_single_entry():
    z = torch.zeros((100, 200), device=DEV)
    assert not ops.orthogonalize([z])[0].any()
    assert not ops.orthogonalize([z], eps=0.0)[0].any()
    one = z.clone()
    one[7, 9] = -3.0
    got = ops.orthogonalize([one])[0].double()
    want = exact(one, QUINTIC, 5)
    assert abs(float(got[7, 9] - want[7, 9])) < 1e-2
    got[7, 9] = 0.0
    assert not got.any()


@pytest.mark.parametrize("cols", [96, 77])
def test_off_alignment(cols):
    rows = 130
    u = draw(1, rows, cols, 8)[0]
    src = torch.empty(rows * cols + 1, device=DEV)
    src[1:] = u.reshape(-1)
    dst = U.Guarded(rows * cols + 3, torch.bfloat16, DEV)
    need = cast.cast_orthogonalize_workspace(1, rows, cols)[1]
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    cast.check(cast.cast_orthogonalize([src[1:]], False, [dst.view[3:]], rows, cols, None, 5, 1e-7, 1.0, ws, need, torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert dst.intact() and bool((dst.view[:3] == dst.canary).all())
    assert torch.equal(dst.view[3:].reshape(rows, cols), ops.orthogonalize([u])[0])


def test_repeatable_on_any_stream_and_in_a_graph():
    u = draw(2, 500, 300, 9)
    one = ops.orthogonalize(u)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        two = ops.orthogonalize(u)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        three = ops.orthogonalize(u)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, three))


def test_transposed_update_gives_the_transposed_result():
    u = draw(1, 384, 640, 10)[0]
    a, b = ops.orthogonalize([u])[0].double(), ops.orthogonalize([u.t().contiguous()])[0].double().T
    assert float(torch.linalg.norm(a - b) / torch.linalg.norm(a)) <= 2 * tolerance(5)


def test_refusals():
    u = draw(2, 64, 96, 11)
    outs = [torch.empty((64, 96), dtype=torch.bfloat16, device=DEV) for _ in u]
    need = cast.cast_orthogonalize_workspace(2, 64, 96)[1]
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    before = cast.cast_kernel_launch_count()
    args = (64, 96, None, 5, 1e-7, 1.0, ws, need)
    assert cast.cast_orthogonalize([u[0], u[1].cpu()], False, outs, *args) == B.CAST_ERR_MEMORY
    assert cast.cast_orthogonalize(u, False, [outs[0], u[1]], *args) == B.CAST_ERR_ALIAS
    assert cast.cast_orthogonalize(u, False, outs, 64, 96, None, 5, 1e-7, 1.0, ws, need - 1) == B.CAST_ERR_PLAN
    assert cast.cast_kernel_launch_count() == before
    with pytest.raises(ValueError, match="shape"):
        ops.orthogonalize([u[0], u[1][:32].contiguous()])
    with pytest.raises(ValueError, match="bfloat16|float32"):
        ops.orthogonalize([u[0], u[1].to(torch.bfloat16)])
    with pytest.raises(ValueError, match="coefficients"):
        ops.orthogonalize(u, coeffs=(1.0, 2.0))
    with pytest.raises(ValueError, match="not contiguous"):
        ops.orthogonalize([x.t() for x in u])


@pytest.mark.parametrize("n,rows,cols", [(1, 2048, 8192), (1, 8192, 2048), (3, 1500, 4100)])
def test_one_step_over_several_chunks(n, rows, cols):
    """A last step that still reads the second word, with more chunks per warp than its ring has slots and several tiles per
    CTA: every slot is written, read and loaded again."""
    u = draw(n, rows, cols, 21)
    out = ops.orthogonalize(u, steps=1)
    for x, o in zip(u, out):
        want = exact(x, QUINTIC, 1)
        assert distance(o, want) <= tolerance(1)
        # chunk by chunk, so that a wrong one is not averaged away; a chunk of 32 x 64 entries averages signs as well
        err = (o.double() - want).abs()
        assert float(err.max()) <= 4 * tolerance(1) * float(want.abs().max())
    assert all(torch.equal(a, b) for a, b in zip(out, ops.orthogonalize(u, steps=1)))


@pytest.mark.parametrize("rows,cols,rank", [(512, 512, 8), (768, 768, 8), (768, 3000, 8), (3000, 768, 8), (1500, 2000, 4), (768, 768, 0), (1024, 1536, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_noise_before_the_last_rounding(rows, cols, rank, dtype):
    """What the result's own rounding to bf16 leaves is known; the rest has to stay below it.  One fp16 word is rounded by
    2.1e-4 of itself (2^-11 at most, over all significands).  P's diagonal, alike in each of five steps: 1.05e-3; one word of X_4
    amplified by 3.44: 7.2e-4; A and the rest of P: 2^-11.  Together 1.4e-3, beside the rounding.  (One word of X_3 as well, amplified
    by 11.9, would be 2.5e-3.)"""
    for u in draw(2, rows, cols, 31 + rank, dtype, rank=rank):
        want = exact(u, QUINTIC, 5)
        rounding = distance(want.to(torch.bfloat16), want)
        assert distance(ops.orthogonalize([u])[0], want) <= math.hypot(rounding, 1.4e-3)


@pytest.mark.parametrize("n,rows,cols", [(1, 20000, 1), (3, 3000, 5), (2, 5000, 16), (2, 4000, 40), (5, 1 << 20, 16), (1, 3, 50), (66, 900, 63)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_shorter_than_a_line(n, rows, cols, dtype):
    u = draw(n, rows, cols, rows + cols, dtype)
    guards = [U.Guarded(rows * cols, torch.bfloat16, DEV) for _ in u]
    rc, need = cast.cast_orthogonalize_workspace(n, rows, cols)
    cast.check(rc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    cast.check(cast.cast_orthogonalize(u, dtype == torch.bfloat16, [g.view for g in guards], rows, cols, None, 5, 1e-7, 1.0, ws, need,
                                       torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert all(g.intact() for g in guards) and bool((ws[need:] == 255).all())
    for i in {0, n // 2, n - 1}:
        # few singular values do not average the signs of their errors
        assert distance(guards[i].view.reshape(rows, cols), exact(u[i], QUINTIC, 5)) <= tolerance(5, 0 if cols < 40 else 1 << 30)


@pytest.mark.parametrize("rows,cols", [(200, 330), (330, 200), (64, 5000), (1, 9)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_not_a_number_stays_in_its_matrix(rows, cols, value, dtype):
    """The norm of an update with an entry that is no number is none either, so no entry of its result is one; the other matrices of
    the call keep theirs."""
    u = draw(3, rows, cols, 41, dtype)
    clean = ops.orthogonalize(u)
    u[1][0, cols // 2] = value
    out = ops.orthogonalize(u)
    assert bool(out[1].isnan().all())
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])
