"""Torch-level calls of the operators around the sparse step: token embedding and gradient, linear cross entropy,
orthogonalised updates.

Plumbing only, like `runner`: the functions check their tensors, allocate results and workspace with torch (on the
current stream, so the caching allocator keeps the workspace until the work is done) and make one call of the library.
They raise ValueError for tensors the library cannot take as they are (nothing is copied or converted behind the
caller's back) and CastError for a refused call.  The results carry no autograd graph: a tensor that requires a gradient is
refused while torch records one, not dropped from it silently.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch

from . import binding as B


def _need(t: torch.Tensor, name: str, dtype, dims: int, device=None) -> None:
    if isinstance(t, torch.Tensor) and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: requires a gradient, but results carry no autograd graph (call under torch.no_grad(), or pass it detached)")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed")
    if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise ValueError(f"{name}: {t.dtype} is not {dtype}")
    if t.dim() != dims:
        raise ValueError(f"{name}: {t.dim()} dimensions instead of {dims}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device} instead of {device}")


def _tokens(ids: torch.Tensor, name: str, device) -> int:
    _need(ids, name, torch.int32, ids.dim() if isinstance(ids, torch.Tensor) else 1, device)
    return ids.numel()


def _workspace(status_and_bytes, like: torch.Tensor) -> torch.Tensor:
    rc, n = status_and_bytes
    B.check(rc)
    return like.new_empty(n, dtype=torch.uint8)


# the current stream as the integer the library takes; the object that torch.cuda.current_stream() makes costs 3 us
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on(device: torch.device, call) -> None:
    """call(stream) with `device` current, and its current stream."""
    if device.index == torch.cuda.current_device():
        B.check(call(_raw_stream(device.index)))
    else:
        with torch.cuda.device(device):
            B.check(call(_raw_stream(device.index)))


def embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[ids] as bf16 [*ids.shape, dim]; zero rows for ids outside the table."""
    _need(table, "table", torch.bfloat16, 2)
    tokens = _tokens(ids, "ids", table.device)
    vocab, dim = table.shape
    shape = (*ids.shape, dim)
    if out is None:
        out = table.new_empty(shape)
    else:
        _need(out, "out", torch.bfloat16, len(shape), table.device)
        if tuple(out.shape) != shape:
            raise ValueError(f"out: shape {tuple(out.shape)} instead of {shape}")
    if tokens:
        _on(table.device, lambda stream: B.cast_embed(table.data_ptr(), ids.data_ptr(), out.data_ptr(), tokens, vocab, dim, scale, stream))
    return out


def embed_grad(grad_out: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, grad_table: Optional[torch.Tensor] = None,
               accumulate: bool = False) -> torch.Tensor:
    """Gradient of embed() with respect to the table, bf16 [vocab, dim]; with accumulate added to grad_table."""
    _need(grad_out, "grad_out", torch.bfloat16, ids.dim() + 1)
    dev, dim = grad_out.device, grad_out.shape[-1]
    tokens = _tokens(ids, "ids", dev)
    if grad_out.shape[:-1] != ids.shape:
        raise ValueError(f"grad_out: shape {tuple(grad_out.shape)} does not go with ids {tuple(ids.shape)}")
    if grad_table is None:
        if accumulate:
            raise ValueError("accumulate needs a grad_table")
        grad_table = grad_out.new_empty((vocab, dim))
    else:
        _need(grad_table, "grad_table", torch.bfloat16, 2, dev)
        if tuple(grad_table.shape) != (vocab, dim):
            raise ValueError(f"grad_table: shape {tuple(grad_table.shape)} instead of {(vocab, dim)}")
    if tokens == 0:
        return grad_table if accumulate else grad_table.zero_()
    ws = _workspace(B.cast_embed_grad_workspace(tokens, dim), grad_out)
    _on(dev, lambda stream: B.cast_embed_grad(grad_out.data_ptr(), ids.data_ptr(), grad_table.data_ptr(), tokens, vocab, dim, scale, accumulate,
                                              ws.data_ptr(), ws.numel(), stream))
    return grad_table


def linear_ce(hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, grad_scale: float = 1.0, hidden_grad: bool = True,
              weight_grad: bool = True, piece_tokens: int = 0
              ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(loss per token fp32, grad_hidden bf16 or None, grad_weight bf16 or None) of the softmax cross entropy of
    hidden @ weight.T; labels outside the vocabulary have no loss and no gradient."""
    _need(hidden, "hidden", torch.bfloat16, 2)
    dev = hidden.device
    _need(weight, "weight", torch.bfloat16, 2, dev)
    tokens, dim = hidden.shape
    vocab = weight.shape[0]
    if weight.shape[1] != dim:
        raise ValueError(f"weight: {weight.shape[1]} columns for hidden states of {dim}")
    if _tokens(labels, "labels", dev) != tokens or labels.dim() != 1:
        raise ValueError(f"labels: shape {tuple(labels.shape)} instead of {(tokens,)}")
    loss = hidden.new_empty(tokens, dtype=torch.float32)
    gh = torch.empty_like(hidden) if hidden_grad else None
    gw = torch.empty_like(weight) if weight_grad else None
    if tokens == 0:
        return loss, gh, gw.zero_() if gw is not None else None
    def call(stream):
        rc, need = B.cast_linear_ce_workspace(tokens, vocab, dim, piece_tokens, hidden_grad, weight_grad)      # depends on the device
        ws = _workspace((rc, need), hidden)
        return B.cast_linear_ce(hidden.data_ptr(), weight.data_ptr(), labels.data_ptr(), loss.data_ptr(), None if gh is None else gh.data_ptr(),
                                None if gw is None else gw.data_ptr(), tokens, vocab, dim, grad_scale, piece_tokens, ws.data_ptr(), need, stream)
    _on(dev, call)
    return loss, gh, gw


def orthogonalize(updates: Sequence[torch.Tensor], steps: int = 5, coeffs: Optional[Sequence[float]] = None, eps: float = 1e-7,
                  scale: float = 1.0, outs: Optional[Sequence[torch.Tensor]] = None) -> List[torch.Tensor]:
    """Newton-Schulz orthogonalisation of matrices of one shape and type (fp32 or bf16) as bf16 matrices.

    coeffs: (a, b, c) for every step, or 3 * steps numbers, or None for the library's quintic."""
    if len(updates) == 0:
        return []
    first = updates[0]
    _need(first, "updates[0]", (torch.float32, torch.bfloat16), 2)
    rows, cols = first.shape
    for i, u in enumerate(updates):
        _need(u, f"updates[{i}]", first.dtype, 2, first.device)
        if u.shape != first.shape:
            raise ValueError(f"updates[{i}]: shape {tuple(u.shape)} instead of {(rows, cols)}")
    if outs is None:
        outs = [first.new_empty((rows, cols), dtype=torch.bfloat16) for _ in updates]
    else:
        if len(outs) != len(updates):
            raise ValueError(f"{len(outs)} outs for {len(updates)} updates")
        for i, o in enumerate(outs):
            _need(o, f"outs[{i}]", torch.bfloat16, 2, first.device)
            if o.shape != first.shape:
                raise ValueError(f"outs[{i}]: shape {tuple(o.shape)} instead of {(rows, cols)}")
    if coeffs is not None:
        coeffs = list(coeffs)
        if len(coeffs) == 3:
            coeffs = coeffs * steps
        if len(coeffs) != 3 * steps:
            raise ValueError(f"{len(coeffs)} coefficients for {steps} steps")
    ws = _workspace(B.cast_orthogonalize_workspace(len(updates), rows, cols), first)
    _on(first.device, lambda stream: B.cast_orthogonalize([u.data_ptr() for u in updates], first.dtype == torch.bfloat16, [o.data_ptr() for o in outs],
                                                          rows, cols, coeffs, steps, eps, scale, ws.data_ptr(), ws.numel(), stream))
    return list(outs)
