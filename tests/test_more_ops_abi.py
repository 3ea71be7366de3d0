"""Refusals of the norm, rotary and gradient-clipping entry points that need no GPU (fake, never-dereferenced addresses), and the
formulas that their GPU tests compare with, against automatic differentiation and differences."""
import math

import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import more_ops_reference as R

A1, A2, A3, A4, A5, A6, WS = (0x100000000 * k for k in range(1, 8))
NO_DEVICE = (B.CAST_ERR_CUDA, B.CAST_ERR_MEMORY)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def _nothing_launched():
    before = cast.cast_kernel_launch_count()
    yield
    assert cast.cast_kernel_launch_count() == before


NORM_REFUSALS = [
    (dict(x=None), B.CAST_ERR_NULL), (dict(weight=None), B.CAST_ERR_NULL), (dict(h=None), B.CAST_ERR_NULL), (dict(residual=None), B.CAST_ERR_NULL),
    (dict(tokens=0), B.CAST_ERR_SHAPE), (dict(tokens=1 << 31), B.CAST_ERR_SHAPE), (dict(dim=0), B.CAST_ERR_SHAPE), (dict(dim=32769), B.CAST_ERR_SHAPE),
    (dict(eps=-1e-9), B.CAST_ERR_HYPER), (dict(eps=NAN), B.CAST_ERR_HYPER), (dict(eps=INF), B.CAST_ERR_HYPER),
    (dict(x=A1 + 1), B.CAST_ERR_ALIGN), (dict(residual=A2 + 1), B.CAST_ERR_ALIGN), (dict(weight=A3 + 2), B.CAST_ERR_ALIGN), (dict(h=A5 + 1), B.CAST_ERR_ALIGN),
    (dict(h=A1 + 16), B.CAST_ERR_ALIAS), (dict(h=A3), B.CAST_ERR_ALIAS),
]


@pytest.mark.parametrize("over,status", NORM_REFUSALS + [
    (dict(y=None), B.CAST_ERR_NULL), (dict(y=A4 + 1), B.CAST_ERR_ALIGN), (dict(y=A1), B.CAST_ERR_ALIAS), (dict(y=A2 + 16), B.CAST_ERR_ALIAS),
    (dict(y=A5 + 32), B.CAST_ERR_ALIAS)])
def test_rms_norm(over, status):
    a = dict(x=A1, residual=A2, weight=A3, weight_fp32=True, y=A4, h=A5, tokens=4, dim=64, eps=1e-6)
    assert cast.cast_rms_norm(**a) in NO_DEVICE
    for alias in (dict(h=A1), dict(h=A2), dict(residual=None, h=None), dict(eps=0.0), dict(weight=A3 + 2, weight_fp32=False)):
        assert cast.cast_rms_norm(**{**a, **alias}) in NO_DEVICE
    a.update(over)
    assert cast.cast_rms_norm(**a) == status


@pytest.mark.parametrize("over,status", NORM_REFUSALS + [
    (dict(q=None), B.CAST_ERR_NULL), (dict(q_scales=None), B.CAST_ERR_NULL), (dict(q=A1 + 5), B.CAST_ERR_ALIAS), (dict(q_scales=A4 + 255), B.CAST_ERR_ALIAS),
    (dict(q_scales=A5), B.CAST_ERR_ALIAS)])
def test_rms_norm_mx(over, status):
    a = dict(x=A1, residual=A2, weight=A3, weight_fp32=True, q=A4, q_scales=A6, h=A5, tokens=4, dim=64, eps=1e-6)
    assert cast.cast_rms_norm_mx(**a) in NO_DEVICE
    assert cast.cast_rms_norm_mx(**{**a, "q": A4 + 1, "q_scales": A4 + 257}) in NO_DEVICE
    a.update(over)
    assert cast.cast_rms_norm_mx(**a) == status


@pytest.mark.parametrize("over,status", [
    (dict(grad_y=None), B.CAST_ERR_NULL), (dict(h=None), B.CAST_ERR_NULL), (dict(weight=None), B.CAST_ERR_NULL), (dict(grad_x=None), B.CAST_ERR_NULL),
    (dict(workspace=None), B.CAST_ERR_NULL), (dict(tokens=0), B.CAST_ERR_SHAPE), (dict(dim=32769), B.CAST_ERR_SHAPE), (dict(eps=NAN), B.CAST_ERR_HYPER),
    (dict(grad_y=A1 + 1), B.CAST_ERR_ALIGN), (dict(grad_weight=A6 + 2), B.CAST_ERR_ALIGN), (dict(workspace=WS + 8), B.CAST_ERR_ALIGN),
    (dict(grad_x=A1), B.CAST_ERR_ALIAS), (dict(grad_x=A2), B.CAST_ERR_ALIAS), (dict(grad_x=A4 + 16), B.CAST_ERR_ALIAS), (dict(grad_weight=A3), B.CAST_ERR_ALIAS),
    (dict(grad_weight=A5 + 64), B.CAST_ERR_ALIAS), (dict(workspace=A1), B.CAST_ERR_ALIAS),
])
def test_rms_norm_grad(over, status):
    a = dict(grad_y=A1, h=A2, weight=A3, weight_fp32=False, grad_h=A4, grad_x=A5, grad_weight=A6, tokens=4, dim=64, eps=1e-6, workspace=WS,
             workspace_bytes=1 << 24)
    assert cast.cast_rms_norm_grad(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_rms_norm_grad(**a) == status


def heads(**over):
    a = dict(x=A1, out=A2, heads=4, in_token_stride=1024, in_head_stride=64, out_token_stride=256, out_head_stride=64)
    a.update(over)
    return B.make_heads(**a)


ROTARY = dict(positions=A5, frequencies=A6, axes=WS, n_axes=2, pairs=32, adjacent=False, inverse=False, tokens=10, head_dim=64)


@pytest.mark.parametrize("over,status", [
    (dict(positions=None), B.CAST_ERR_NULL), (dict(frequencies=None), B.CAST_ERR_NULL), (dict(axes=None), B.CAST_ERR_SHAPE),
    (dict(tokens=0), B.CAST_ERR_SHAPE), (dict(pairs=0), B.CAST_ERR_SHAPE), (dict(pairs=33), B.CAST_ERR_SHAPE), (dict(pairs=513, head_dim=1026), B.CAST_ERR_SHAPE),
    (dict(head_dim=1025), B.CAST_ERR_SHAPE), (dict(n_axes=0), B.CAST_ERR_SHAPE), (dict(n_axes=65), B.CAST_ERR_SHAPE),
    (dict(positions=A5 + 2), B.CAST_ERR_ALIGN), (dict(frequencies=A6 + 4), B.CAST_ERR_ALIGN), (dict(axes=WS + 1), B.CAST_ERR_ALIGN),
    (dict(positions=A2 + 64), B.CAST_ERR_ALIAS), (dict(frequencies=A2), B.CAST_ERR_ALIAS), (dict(axes=A2), B.CAST_ERR_ALIAS),
    (dict(sets=[]), B.CAST_ERR_SHAPE), (dict(sets=[heads()] * 5), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(x=None)]), B.CAST_ERR_NULL), (dict(sets=[heads(out=None)]), B.CAST_ERR_NULL), (dict(sets=[heads(heads=0)]), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(heads=65537, out_head_stride=64, out_token_stride=1 << 23)]), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(x=A1 + 1)]), B.CAST_ERR_ALIGN), (dict(sets=[heads(out=A2 + 1)]), B.CAST_ERR_ALIGN),
    (dict(sets=[heads(in_token_stride=-64)]), B.CAST_ERR_SHAPE), (dict(sets=[heads(in_token_stride=1 << 50)]), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(out_head_stride=63)]), B.CAST_ERR_SHAPE), (dict(sets=[heads(out_token_stride=255)]), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(out_token_stride=0)]), B.CAST_ERR_SHAPE), (dict(sets=[heads(out_head_stride=639, out_token_stride=64)]), B.CAST_ERR_SHAPE),
    (dict(sets=[heads(out=A1 + 128)]), B.CAST_ERR_ALIAS), (dict(sets=[heads(out=A1)]), B.CAST_ERR_ALIAS),
    (dict(sets=[heads(), heads(x=A3, out=A2 + 128)]), B.CAST_ERR_ALIAS), (dict(sets=[heads(), heads(x=A2, out=A3)]), B.CAST_ERR_ALIAS),
    # side by side in rows of 320 entries: 4 heads of 64 leave room for one
    (dict(sets=[heads(out_token_stride=320), heads(x=A3, out=A2 + 512, heads=2, out_token_stride=320)]), B.CAST_ERR_ALIAS),
])
def test_rotary(over, status):
    a = dict(sets=[heads()], **ROTARY)
    assert cast.cast_rotary(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_rotary(**a) == status


@pytest.mark.parametrize("sets", [
    [heads(out=A1, out_token_stride=1024)],                                                             # in place
    [heads(out=A1, out_token_stride=1024), heads(x=A1 + 512, out=A1 + 512, out_token_stride=1024)],     # both in place in a fused array
    [heads(out_token_stride=320), heads(x=A3, out=A2 + 512, heads=1, out_token_stride=320)],            # results side by side
    [heads(out_head_stride=640, out_token_stride=64)],                                                  # heads first
    [heads(in_token_stride=0)], [heads(in_head_stride=0)],                                              # broadcast inputs
])
def test_rotary_arrangements_that_are_taken(sets):
    assert cast.cast_rotary(sets=sets, **ROTARY) in NO_DEVICE


def test_rotary_of_one_token_takes_any_token_stride():
    one = [heads(out=A1, in_token_stride=7, out_token_stride=0)]
    assert cast.cast_rotary(**{**ROTARY, "sets": one, "tokens": 1}) in NO_DEVICE


@pytest.mark.parametrize("grads,status", [
    ([], B.CAST_ERR_NULL), ([(None, A2, 10, 0, 0)], B.CAST_ERR_NULL), ([(A1, A2, 10, 0, 0), (A3, None, 10, 0, 0)], B.CAST_ERR_NULL),
    ([(A1, A2, 0, 0, 0)], B.CAST_ERR_SHAPE), ([(A1, A2, -5, 0, 0)], B.CAST_ERR_SHAPE), ([(A1, A2, (1 << 40) + 1, 0, 0)], B.CAST_ERR_SHAPE),
    ([(A1 + 2, A2, 10, 0, 0)], B.CAST_ERR_ALIGN), ([(A1, A2 + 2, 10, 0, 0)], B.CAST_ERR_ALIGN), ([(A1 + 1, A2, 10, 1, 0)], B.CAST_ERR_ALIGN),
    ([(A1, A1, 10, 0, 1)], B.CAST_ERR_ALIAS), ([(A1, A1 + 4, 10, 0, 0)], B.CAST_ERR_ALIAS), ([(A1, A2, 10, 0, 0), (A3, A2 + 36, 10, 0, 0)], B.CAST_ERR_ALIAS),
    ([(A1, A2, 10, 0, 0), (A2 + 16, A3, 10, 0, 0)], B.CAST_ERR_ALIAS), ([(A1, A1, 10, 0, 0), (A1, A1, 10, 0, 0)], B.CAST_ERR_ALIAS),
    ([(A1, A2, 10, 0, 0), (A1 + 20, A1 + 20, 3, 0, 0)], B.CAST_ERR_ALIAS),
])
def test_grads_create(grads, status):
    for taken in ([(A1, A1, 10, 0, 0)], [(A1, None, 10, 0, 0), (A1, None, 10, 0, 0)], [(A1, A2, 10, 0, 1), (A1, A2 + 20, 10, 0, 0)],
                  [(A1 + 2, A1 + 2, 10, 1, 1), (A1 + 22, A1 + 22, 10, 1, 1)]):
        rc, handle = cast.cast_grads_create([B.make_grad(*g) for g in taken])
        assert rc in NO_DEVICE and handle is None
    rc, handle = cast.cast_grads_create([B.make_grad(*g) for g in grads])
    assert rc == status and handle is None


def test_grads_calls_refuse_what_is_no_set():
    assert cast.cast_grads_destroy(None) == B.CAST_ERR_PLAN
    assert cast.cast_grads_workspace(None)[0] == B.CAST_ERR_PLAN
    assert cast.cast_grads_norm(None, 1.0, A1, A2, 100) == B.CAST_ERR_PLAN
    assert cast.cast_grads_clip(None, 1.0, 1.0, A1, A2, 100) == B.CAST_ERR_PLAN
    assert cast.cast_grads_clip(None, NAN, 1.0, A1, A2, 100) == B.CAST_ERR_HYPER
    assert cast.cast_grads_clip(None, -1.0, 1.0, A1, A2, 100) == B.CAST_ERR_HYPER


def test_workspace_sizes_refuse_bad_shapes():
    assert cast.cast_rms_norm_grad_workspace(0, 64)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_rms_norm_grad_workspace(5, 32769)[0] == B.CAST_ERR_SHAPE


def calls(x, w, pos):
    return (lambda: ops.rms_norm(x, w), lambda: ops.rms_norm_mx(x, w), lambda: ops.rms_norm_grad(x, x, w), lambda: ops.GradientSet([x]))


def test_torch_level_calls_refuse_host_tensors():
    x, w, pos = torch.zeros((4, 8), dtype=torch.bfloat16), torch.ones(8), torch.zeros(4, dtype=torch.int32)
    for call in calls(x, w, pos) + (lambda: ops.rotary(x[:, None], None, pos, None),):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="grads"):
        ops.GradientSet([])


def test_torch_level_calls_do_not_drop_a_graph():
    x, w, pos = torch.zeros((4, 8), dtype=torch.bfloat16, requires_grad=True), torch.ones(8), torch.zeros(4, dtype=torch.int32)
    for call in calls(x, w, pos):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
            call()


def test_spectrum():
    s = ops.RotarySpectrum.of(16, base=100.0, sections=[2, 0, 6], device="cpu")
    assert (s.pairs, s.n_axes) == (8, 3) and s.axes.tolist() == [0, 0, 2, 2, 2, 2, 2, 2]
    assert all(math.isclose(f, 100.0 ** (-i / 8)) for i, f in enumerate(s.frequencies.tolist()))
    s = ops.RotarySpectrum.of(12, base=100.0, sections=[2, 4], per_axis=True, adjacent=True, device="cpu")
    assert s.adjacent and all(math.isclose(f, 100.0 ** -p) for f, p in zip(s.frequencies.tolist(), (0, 0.5, 0, 0.25, 0.5, 0.75)))
    with pytest.raises(AttributeError):
        s.frequencies = torch.ones(2)
    for bad in (lambda: ops.RotarySpectrum.of(7, device="cpu"), lambda: ops.RotarySpectrum.of(8, sections=[3], device="cpu"),
                lambda: ops.RotarySpectrum.of(8, sections=[5, -1], device="cpu"), lambda: ops.RotarySpectrum([], device="cpu"),
                lambda: ops.RotarySpectrum([1.0], axes=[0, 1], device="cpu"), lambda: ops.RotarySpectrum([1.0], axes=[-1], device="cpu"),
                lambda: ops.RotarySpectrum([INF], device="cpu")):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------------------------------------ the formulas themselves

def test_norm_gradient_formula_against_autograd_and_differences():
    gen = torch.Generator().manual_seed(0)
    T, D, eps = 5, 7, 1e-3
    h, dy, dh = (torch.randn((T, D), generator=gen, dtype=torch.float64) for _ in range(3))
    w = torch.randn(D, generator=gen, dtype=torch.float64)
    dx, dw = R.norm_grad(dy, h, w, dh, eps)
    ha, wa = h.clone().requires_grad_(), w.clone().requires_grad_()
    loss = (R.norm(ha, wa, eps) * dy).sum() + (ha * dh).sum()
    loss.backward()
    assert torch.allclose(dx, ha.grad, rtol=1e-12, atol=1e-13) and torch.allclose(dw, wa.grad, rtol=1e-12, atol=1e-13)

    def value(h, w):
        return float((R.norm(h, w, eps) * dy).sum() + (h * dh).sum())
    step = 1e-5               # central differences: error step^2 ~ 1e-10 of third derivatives, rounding 1e-15 / step = 1e-10
    for i in range(T * D):
        e = torch.zeros(T * D, dtype=torch.float64)
        e[i] = step
        e = e.view(T, D)
        assert abs((value(h + e, w) - value(h - e, w)) / (2 * step) - float(dx.view(-1)[i])) < 1e-7
    for i in range(D):
        e = torch.zeros(D, dtype=torch.float64)
        e[i] = step
        assert abs((value(h, w + e) - value(h, w - e)) / (2 * step) - float(dw[i])) < 1e-7


def test_rotary_formula_is_a_rotation_whose_inverse_is_its_gradient():
    gen = torch.Generator().manual_seed(1)
    x, g = (torch.randn((6, 3, 20), generator=gen, dtype=torch.float64) for _ in range(2))
    positions = torch.randint(-1000, 1000, (2, 6), generator=gen).int()
    for adjacent in (False, True):
        args = (positions, [1.0, 0.3, 0.01, 0.5, 2.0, 0.7, 0.0, 1e-4], [0, 1, 0, 1, 1, 0, 0, 1], adjacent)
        xa = x.clone().requires_grad_()
        y = R.rotary(xa, *args, inverse=False)
        y.backward(g)
        assert torch.allclose(xa.grad, R.rotary(g, *args, inverse=True), atol=1e-13)
        assert torch.allclose(R.rotary(y.detach(), *args, inverse=True), x, atol=1e-12)
        assert torch.equal(y[..., 16:], x[..., 16:])


def test_reference_of_8_bit_values():
    """Every e4m3 value stands for itself, and what lies between two goes to the nearer one, a tie to the even one."""
    bits = torch.arange(0, 127, dtype=torch.uint8)
    grid = bits.view(torch.float8_e4m3fn).double()
    assert torch.equal(R.to_e4m3(grid), grid) and torch.equal(R.to_e4m3(-grid), -grid)
    mid = (grid[1:] + grid[:-1]) / 2
    assert torch.equal(R.to_e4m3(mid), torch.where(bits[:-1] % 2 == 0, grid[:-1], grid[1:]))
    assert torch.equal(R.to_e4m3(mid * (1 + 1e-9)), grid[1:]) and torch.equal(R.to_e4m3(mid * (1 - 1e-9)), grid[:-1])


def test_torch_level_calls_do_not_drop_a_tangent():
    from torch.autograd import forward_ad
    w, ids = torch.ones(8), torch.zeros(4, dtype=torch.int32)
    with forward_ad.dual_level():
        x = forward_ad.make_dual(torch.zeros((4, 8), dtype=torch.bfloat16), torch.ones((4, 8), dtype=torch.bfloat16))
        for call in calls(x, w, ids) + (lambda: ops.embed(x, ids), lambda: ops.linear_ce(x, x, ids), lambda: ops.orthogonalize([x])):
            with pytest.raises(ValueError, match="forward-mode tangent"):
                call()
        plain = forward_ad.unpack_dual(x).primal
        for call in calls(plain, w, ids):
            with pytest.raises(ValueError, match="CUDA tensor"):
                call()
