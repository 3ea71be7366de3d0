"""Refusals of the embedding, linear cross-entropy and orthogonalisation entry points that need no GPU: every check on
the host runs before the first CUDA call (fake, never-dereferenced addresses)."""
import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops

A1, A2, A3, A4, A5, A6, WS = (0x100000000 * k for k in range(1, 8))
NO_DEVICE = (B.CAST_ERR_CUDA, B.CAST_ERR_MEMORY)


@pytest.fixture(autouse=True)
def _nothing_launched():
    before = cast.cast_kernel_launch_count()
    yield
    assert cast.cast_kernel_launch_count() == before


@pytest.mark.parametrize("over,status", [
    (dict(table=None), B.CAST_ERR_NULL), (dict(ids=None), B.CAST_ERR_NULL), (dict(out=None), B.CAST_ERR_NULL),
    (dict(tokens=0), B.CAST_ERR_SHAPE), (dict(vocab=0), B.CAST_ERR_SHAPE), (dict(dim=0), B.CAST_ERR_SHAPE),
    (dict(tokens=1 << 31), B.CAST_ERR_SHAPE), (dict(vocab=0x7FFFFFFF), B.CAST_ERR_SHAPE),
    (dict(scale=float("nan")), B.CAST_ERR_HYPER),
    (dict(table=A1 + 1), B.CAST_ERR_ALIGN), (dict(ids=A2 + 2), B.CAST_ERR_ALIGN),
    (dict(out=A1 + 64), B.CAST_ERR_ALIAS), (dict(out=A2), B.CAST_ERR_ALIAS),
])
def test_embed(over, status):
    a = dict(table=A1, ids=A2, out=A3, tokens=4, vocab=100, dim=64, scale=1.0)
    assert cast.cast_embed(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_embed(**a) == status


@pytest.mark.parametrize("over,status", [
    (dict(grad_out=None), B.CAST_ERR_NULL), (dict(workspace=None), B.CAST_ERR_NULL),
    (dict(tokens=-1), B.CAST_ERR_SHAPE), (dict(dim=0), B.CAST_ERR_SHAPE),
    (dict(scale=float("inf")), B.CAST_ERR_HYPER),
    (dict(grad_table=A3 + 1), B.CAST_ERR_ALIGN), (dict(workspace=WS + 4), B.CAST_ERR_ALIGN),
    (dict(workspace_bytes=16), B.CAST_ERR_PLAN),
    (dict(grad_table=A1), B.CAST_ERR_ALIAS), (dict(workspace=A3 + 64), B.CAST_ERR_ALIAS), (dict(workspace=A1), B.CAST_ERR_ALIAS),
])
def test_embed_grad(over, status):
    rc, need = cast.cast_embed_grad_workspace(100, 64)
    assert rc == B.CAST_OK and need > 0
    a = dict(grad_out=A1, ids=A2, grad_table=A3, tokens=100, vocab=100, dim=64, scale=1.0, accumulate=False, workspace=WS, workspace_bytes=need)
    assert cast.cast_embed_grad(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_embed_grad(**a) == status


def test_workspace_sizes_refuse_bad_shapes():
    assert cast.cast_embed_grad_workspace(0, 64)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_embed_grad_workspace(1 << 30, 1 << 20)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_linear_ce_workspace(0, 100, 64)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_linear_ce_workspace(10, 100, 60)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_linear_ce_workspace(10, 100, 64, piece_tokens=-1)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_orthogonalize_workspace(0, 64, 64)[0] == B.CAST_ERR_SHAPE
    assert cast.cast_orthogonalize_workspace(1, 1 << 16, 1 << 16)[0] == B.CAST_ERR_SHAPE
    rc, one = cast.cast_orthogonalize_workspace(1, 64, 64)
    assert rc == B.CAST_OK
    assert cast.cast_orthogonalize_workspace(2, 64, 64)[1] > one
    # many large matrices share the memory of as many as make 64 M entries
    assert cast.cast_orthogonalize_workspace(100, 4096, 11008)[1] == cast.cast_orthogonalize_workspace(1, 4096, 11008)[1]


@pytest.mark.parametrize("over,status", [
    (dict(hidden=None), B.CAST_ERR_NULL), (dict(labels=None), B.CAST_ERR_NULL), (dict(loss=None), B.CAST_ERR_NULL),
    (dict(workspace=None), B.CAST_ERR_NULL),
    (dict(tokens=0), B.CAST_ERR_SHAPE), (dict(vocab=0), B.CAST_ERR_SHAPE), (dict(dim=60), B.CAST_ERR_SHAPE), (dict(piece_tokens=-5), B.CAST_ERR_SHAPE),
    (dict(grad_scale=float("nan")), B.CAST_ERR_HYPER),
    (dict(hidden=A1 + 2), B.CAST_ERR_ALIGN), (dict(grad_weight=A6 + 8), B.CAST_ERR_ALIGN), (dict(loss=A4 + 2), B.CAST_ERR_ALIGN),
])
def test_linear_ce(over, status):
    a = dict(hidden=A1, weight=A2, labels=A3, loss=A4, grad_hidden=A5, grad_weight=A6, tokens=4, vocab=100, dim=64, grad_scale=1.0,
             piece_tokens=0, workspace=WS, workspace_bytes=1 << 30)
    assert cast.cast_linear_ce(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_linear_ce(**a) == status


@pytest.mark.parametrize("over,status", [
    (dict(updates=None), B.CAST_ERR_NULL), (dict(outs=None), B.CAST_ERR_NULL), (dict(workspace=None), B.CAST_ERR_NULL),
    (dict(updates=[A1, None]), B.CAST_ERR_NULL), (dict(outs=[None, A4]), B.CAST_ERR_NULL),
    (dict(rows=0), B.CAST_ERR_SHAPE), (dict(rows=1 << 20, cols=1 << 12), B.CAST_ERR_SHAPE),
    (dict(steps=0), B.CAST_ERR_HYPER), (dict(steps=101), B.CAST_ERR_HYPER), (dict(eps=-1.0), B.CAST_ERR_HYPER), (dict(eps=float("nan")), B.CAST_ERR_HYPER),
    (dict(scale=float("inf")), B.CAST_ERR_HYPER), (dict(coeffs=[3.0, float("nan"), 2.0] * 5), B.CAST_ERR_HYPER),
    (dict(updates=[A1, A2 + 2]), B.CAST_ERR_ALIGN), (dict(outs=[A3 + 1, A4]), B.CAST_ERR_ALIGN), (dict(workspace=WS + 8), B.CAST_ERR_ALIGN),
    (dict(workspace_bytes=100), B.CAST_ERR_PLAN),
    (dict(outs=[A1 + 64, A4]), B.CAST_ERR_ALIAS), (dict(workspace=A4), B.CAST_ERR_ALIAS),
    (dict(outs=[A3, A1]), B.CAST_ERR_ALIAS), (dict(outs=[A3, A3 + 64]), B.CAST_ERR_ALIAS),
])
def test_orthogonalize(over, status):
    rc, need = cast.cast_orthogonalize_workspace(2, 64, 96)
    a = dict(updates=[A1, A2], updates_bf16=False, outs=[A3, A4], rows=64, cols=96, coeffs=None, steps=5, eps=1e-7, scale=1.0, workspace=WS,
             workspace_bytes=need)
    assert cast.cast_orthogonalize(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_orthogonalize(**a) == status


def test_product_failures():
    assert cast.cast_product_failures(3)[0] == B.CAST_ERR_HYPER
    assert cast.cast_product_failures(-1)[0] == B.CAST_ERR_HYPER


def test_torch_level_calls_refuse_host_tensors():
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ops.embed(x, ids), lambda: ops.embed_grad(x, ids, 10), lambda: ops.linear_ce(x, x, ids), lambda: ops.orthogonalize([x])):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    assert ops.orthogonalize([]) == []


@pytest.mark.parametrize("n,rows,cols", [(64, 1000000, 1), (16, 4000000, 1), (64, 65536, 16), (64, 1, 1000000), (1, 4000000, 1), (64, 300000, 65), (1000, 40, 7)])
def test_orthogonalize_workspace_of_narrow_matrices(n, rows, cols):
    """Four sets of 2-byte words over at most 64 M entries of padded rows, or one matrix of more; the squares, the norms and the
    sums of splits add less than that again."""
    rc, need = cast.cast_orthogonalize_workspace(n, rows, cols)
    padded = rows * (-(-cols // 8) * 8 if cols < 64 else -(-cols // 64) * 64)
    assert rc == B.CAST_OK and need <= 2 * 8 * max(64 << 20, padded)


@pytest.mark.parametrize("over", [dict(outs=[A3]), dict(outs=[A3, A4, A5]), dict(outs=[]), dict(coeffs=[3.0, -4.0, 2.0]), dict(coeffs=[1.0] * 16), dict(coeffs=[])])
def test_orthogonalize_sequences_of_another_length(over):
    a = dict(updates=[A1, A2], updates_bf16=False, outs=[A3, A4], rows=64, cols=96, coeffs=[1.0] * 15, steps=5, eps=1e-7, scale=1.0, workspace=WS,
             workspace_bytes=1 << 30)
    assert cast.cast_orthogonalize(**a) in NO_DEVICE
    a.update(over)
    assert cast.cast_orthogonalize(**a) == B.CAST_ERR_SHAPE


def test_torch_level_calls_do_not_drop_a_graph():
    """Tensors that require a gradient are refused while torch records a graph (and get as far as the next check when it does not)."""
    x = torch.zeros((4, 8), dtype=torch.bfloat16, requires_grad=True)
    plain = torch.zeros((4, 8), dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ops.embed(x, ids), lambda: ops.embed_grad(x, ids, 10), lambda: ops.linear_ce(x, plain, ids), lambda: ops.orthogonalize([x])):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
            call()
