"""Torch-level calls of the operators around the sparse step: token embedding and gradient, linear cross entropy,
orthogonalised updates, root-mean-square norm and gradient, rotary positions, gradient clipping.

Plumbing only, like `runner`: the functions check their tensors, allocate results and workspace with torch (on the
current stream, so the caching allocator keeps the workspace until the work is done) and make one call of the library.
They raise ValueError for tensors the library cannot take as they are (nothing is copied or converted behind the
caller's back) and CastError for a refused call.  The results carry no autograd graph: a tensor that requires a gradient is
refused while torch records one, and a dual tensor of forward-mode differentiation, not dropped from it silently.
"""
from __future__ import annotations

import functools
import math
import struct
from typing import List, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from . import binding as B


def _refuse_derivatives(t: torch.Tensor, name: str) -> None:
    """A tensor through which torch follows derivatives, which the results would drop."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: requires a gradient, but results carry no autograd graph (call under torch.no_grad(), or pass it detached)")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name}: has a forward-mode tangent, but results carry none (pass forward_ad.unpack_dual(...).primal)")


def _need(t: torch.Tensor, name: str, dtype, dims: int, device=None) -> None:
    if isinstance(t, torch.Tensor):
        _refuse_derivatives(t, name)
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


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(index: int, function, *args) -> None:
    """One call of the library, with device `index` current and its current stream as the last argument."""
    if index == _current_device():
        B.check(function(*args, _raw_stream(index)))
    else:
        with torch.cuda.device(index):
            B.check(function(*args, _raw_stream(index)))


def _taken(t, dtype, index: int) -> bool:
    """The usual case of what _need() asks for, decided in a microsecond less; where this is False, _need() says why or lets it pass."""
    return type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == index and t.is_contiguous() and not t.requires_grad and \
        forward_ad._current_level < 0


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


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


def _rows(x: torch.Tensor, weight: torch.Tensor, first: str, *others: Tuple[Optional[torch.Tensor], str]) -> Tuple[int, int, int]:
    """(tokens, dim, device index) of an array of rows, the weight of their columns and arrays of the same shape (or None)."""
    if not isinstance(x, torch.Tensor) or not _taken(x, torch.bfloat16, x.get_device()) or not x.is_cuda:
        _need(x, first, torch.bfloat16, x.dim() if isinstance(x, torch.Tensor) else 1)
    index, shape = x.get_device(), x.shape
    if not shape:
        raise ValueError(f"{first}: no columns")
    if not (_taken(weight, torch.bfloat16, index) or _taken(weight, torch.float32, index)) or weight.dim() != 1:
        _need(weight, "weight", (torch.float32, torch.bfloat16), 1, x.device)
    dim = shape[-1]
    if weight.numel() != dim:
        raise ValueError(f"weight: {weight.numel()} entries for {dim} columns")
    for t, name in others:
        if t is not None:
            if not _taken(t, torch.bfloat16, index):
                _need(t, name, torch.bfloat16, len(shape), x.device)
            if t.shape != shape:
                raise ValueError(f"{name}: shape {tuple(t.shape)} instead of {tuple(shape)}")
    return (x.numel() // dim if dim else 0), dim, index


def _bytes_on(device: torch.device, n: int) -> torch.Tensor:
    return torch.empty_strided((n,), (1,), dtype=torch.uint8, device=device)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, out: Optional[torch.Tensor] = None,
             sum_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(y, h): h = x + residual (x itself without a residual), y = weight h / sqrt(mean(h^2) + eps) over the last dimension, both
    bf16.  weight: bf16 or fp32.  sum_out may be residual (or x), which h then replaces."""
    tokens, dim, index = _rows(x, weight, "x", (residual, "residual"), (out, "out"), (sum_out, "sum_out"))
    if residual is None and sum_out is not None:
        raise ValueError("sum_out needs a residual")
    y = torch.empty_like(x) if out is None else out
    h = x if residual is None else torch.empty_like(x) if sum_out is None else sum_out
    if tokens:
        _call(index, B.load_library().cast_rms_norm, x.data_ptr(), _ptr(residual), weight.data_ptr(), weight.dtype is torch.float32, y.data_ptr(),
              None if residual is None else h.data_ptr(), tokens, dim, eps)
    return y, h


def rms_norm_mx(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                sum_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(q, scales, h): rms_norm with y as float8_e4m3fn values and a power of two (float8_e8m0fnu) for every 32 columns, row-major."""
    tokens, dim, index = _rows(x, weight, "x", (residual, "residual"), (sum_out, "sum_out"))
    if residual is None and sum_out is not None:
        raise ValueError("sum_out needs a residual")
    q = torch.empty_like(x, dtype=torch.float8_e4m3fn)
    scales = x.new_empty((*x.shape[:-1], (dim + 31) // 32), dtype=torch.float8_e8m0fnu)
    h = x if residual is None else torch.empty_like(x) if sum_out is None else sum_out
    if tokens:
        _call(index, B.load_library().cast_rms_norm_mx, x.data_ptr(), _ptr(residual), weight.data_ptr(), weight.dtype is torch.float32, q.data_ptr(),
              scales.data_ptr(), None if residual is None else h.data_ptr(), tokens, dim, eps)
    return q, scales, h


@functools.lru_cache(maxsize=1024)
def _rms_norm_grad_bytes(tokens: int, dim: int, device_index: int) -> int:
    with torch.cuda.device(device_index):
        rc, n = B.cast_rms_norm_grad_workspace(tokens, dim)
    B.check(rc)
    return n


def rms_norm_grad(grad_y: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, grad_h: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  weight_grad: bool = True, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(grad_x bf16, grad_weight fp32 or None) of rms_norm from the h it returned.  grad_h: the gradient that reaches h from what
    comes after on the residual stream; grad_x is then the gradient of x and of residual.  out may be grad_h."""
    tokens, dim, index = _rows(h, weight, "h", (grad_y, "grad_y"), (grad_h, "grad_h"), (out, "out"))
    if grad_y is None:
        raise ValueError("grad_y: a CUDA tensor is needed")
    gx = torch.empty_like(h) if out is None else out
    gw = torch.empty_like(weight, dtype=torch.float32) if weight_grad else None
    if tokens == 0:
        return gx, gw.zero_() if gw is not None else None
    n = _rms_norm_grad_bytes(tokens, dim, index) if weight_grad else 0
    ws = _bytes_on(h.device, n) if weight_grad else None
    _call(index, B.load_library().cast_rms_norm_grad, grad_y.data_ptr(), h.data_ptr(), weight.data_ptr(), weight.dtype is torch.float32, _ptr(grad_h),
          gx.data_ptr(), _ptr(gw), tokens, dim, eps, _ptr(ws), n)
    return gx, gw


class RotarySpectrum:
    """Which columns of a head turn together, how fast, and with which axis of the positions.

    frequencies: radians per position of every pair of columns.  axes: the axis of every pair (None: all on axis 0).
    adjacent: pairs are columns (2i, 2i + 1) instead of (i, i + pairs)."""

    def __init__(self, frequencies: Sequence[float], axes: Optional[Sequence[int]] = None, adjacent: bool = False, device=None):
        frequencies = [float(f) for f in frequencies]
        axes = [0] * len(frequencies) if axes is None else [int(a) for a in axes]
        if not frequencies or len(axes) != len(frequencies):
            raise ValueError(f"{len(axes)} axes for {len(frequencies)} frequencies")
        if not all(math.isfinite(f) for f in frequencies):
            raise ValueError("frequencies: not all finite")
        if min(axes) < 0:
            raise ValueError("axes: negative")
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.pairs, self.n_axes, self.adjacent = len(frequencies), max(axes) + 1, bool(adjacent)
        self._frequencies = torch.tensor(frequencies, dtype=torch.float64, device=device)
        self._axes = torch.tensor(axes, dtype=torch.int32, device=device)

    @property
    def frequencies(self) -> torch.Tensor:
        """fp64 [pairs] on the device; its entries may be changed, the tensor stays."""
        return self._frequencies

    @property
    def axes(self) -> torch.Tensor:
        """int32 [pairs] on the device, as frequencies; a pair of an axis that the positions do not have does not turn."""
        return self._axes

    @classmethod
    def of(cls, dims: int, base: float = 10000.0, sections: Optional[Sequence[int]] = None, per_axis: bool = False, adjacent: bool = False,
           device=None) -> "RotarySpectrum":
        """The usual spectrum of `dims` turning columns: base^(-2i / dims) for pair i.  sections: how many consecutive pairs
        belong to each axis; per_axis: every axis has the spectrum of its own columns instead of its part of the whole one."""
        if dims < 2 or dims % 2:
            raise ValueError(f"{dims} columns do not make pairs")
        sections = [dims // 2] if sections is None else [int(n) for n in sections]
        if sum(sections) != dims // 2 or min(sections) < 0:
            raise ValueError(f"sections {sections} of {dims // 2} pairs")
        frequencies: List[float] = []
        axes: List[int] = []
        for axis, n in enumerate(sections):
            frequencies += [base ** -(j / n if per_axis else (len(axes) + j) / (dims // 2)) for j in range(n)]
            axes += [axis] * n
        return cls(frequencies, axes, adjacent, device)


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, spectrum: RotarySpectrum, inverse: bool = False,
           out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Turns the heads of q and k (bf16 [tokens, heads, head_dim], any strides with contiguous columns; k may be None) by the
    positions, int32 [axes, tokens] or [tokens].  inverse: the other way, which takes gradients back.  out: where the results go (q and k
    themselves, or arrays of any strides); new contiguous arrays without."""
    if not isinstance(positions, torch.Tensor) or positions.dim() not in (1, 2) or not _taken(positions, torch.int32, positions.get_device()) or not positions.is_cuda:
        _need(positions, "positions", torch.int32, positions.dim() if isinstance(positions, torch.Tensor) and positions.dim() in (1, 2) else 2)
    dev, index = positions.device, positions.get_device()
    n_axes, tokens = (1, positions.shape[0]) if positions.dim() == 1 else positions.shape
    if n_axes < spectrum.n_axes:
        raise ValueError(f"positions: {n_axes} axes for a spectrum of {spectrum.n_axes}")
    if spectrum.frequencies.get_device() != index:
        raise ValueError(f"spectrum: on {spectrum.frequencies.device} instead of {dev}")
    if k is None and out is not None and out[1] is not None:
        raise ValueError("out[1]: there is no k")
    head_dim = q.shape[-1] if isinstance(q, torch.Tensor) and q.dim() else 0
    sets, n_sets = b"", 0
    results: List[Optional[torch.Tensor]] = [None, None]
    for i in (0, 1) if k is not None else (0,):
        x = k if i else q
        heads, from_token, from_head = _need_heads(x, "k" if i else "q", index, tokens, None, head_dim)
        if out is None:
            to_token, to_head = heads * head_dim, head_dim
            o = torch.empty_strided((tokens, heads, head_dim), (to_token, to_head, 1), dtype=torch.bfloat16, device=dev)
        else:
            o = out[i]
            _, to_token, to_head = _need_heads(o, f"out[{i}]", index, tokens, heads, head_dim)
        results[i] = o
        if heads:
            sets += struct.pack("7q", x.data_ptr(), o.data_ptr(), heads, from_token, from_head, to_token, to_head)      # a cast_heads_t
            n_sets += 1
    if 2 * spectrum.pairs > head_dim:
        raise ValueError(f"spectrum: {2 * spectrum.pairs} columns of heads of {head_dim}")
    if tokens and n_sets:
        _call(index, B.load_library().cast_rotary, sets, n_sets, positions.data_ptr(), spectrum.frequencies.data_ptr(), spectrum.axes.data_ptr(), n_axes,
              spectrum.pairs, spectrum.adjacent, inverse, tokens, head_dim)
    return results[0], results[1]


def _need_heads(t: torch.Tensor, name: str, index: int, tokens: int, heads: Optional[int], head_dim: int) -> Tuple[int, int, int]:
    """(heads, token stride, head stride) of an array of heads."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed")
    _refuse_derivatives(t, name)
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name}: {t.dtype} is not {torch.bfloat16}")
    if t.get_device() != index:
        raise ValueError(f"{name}: on {t.device} instead of cuda:{index}")
    shape = t.shape
    if len(shape) != 3 or shape[0] != tokens or shape[2] != head_dim or heads not in (None, shape[1]):
        raise ValueError(f"{name}: shape {tuple(shape)} instead of {(tokens, 'heads' if heads is None else heads, head_dim)}")
    token_stride, head_stride, column_stride = t.stride()
    if column_stride != 1 and head_dim > 1:
        raise ValueError(f"{name}: the columns of a head are not contiguous")
    return shape[1], token_stride, head_stride


class GradientSet:
    """The gradients of a model as one set, for their global norm and clipping.

    grads: contiguous fp32 or bf16 tensors of one device.  outs: where the clipped gradients go, fp32 or bf16, one of the same number
    of entries for each, e.g. the bf16 gradients that a step takes behind ones accumulated in fp32.  Without outs clip() works in place.
    The tensors are kept alive and keep their places."""

    def __init__(self, grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None):
        self._handle = None
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if len(grads) == 0 or len(outs) != len(grads):
            raise ValueError(f"{len(outs)} outs for {len(grads)} grads")
        kinds = (torch.float32, torch.bfloat16)
        _need(grads[0], "grads[0]", kinds, grads[0].dim() if isinstance(grads[0], torch.Tensor) else 1)
        self.device = grads[0].device
        rows = []
        for i, (g, o) in enumerate(zip(grads, outs)):
            _need(g, f"grads[{i}]", kinds, g.dim() if isinstance(g, torch.Tensor) else 1, self.device)
            _need(o, f"outs[{i}]", kinds, o.dim() if isinstance(o, torch.Tensor) else 1, self.device)
            if o.numel() != g.numel():
                raise ValueError(f"outs[{i}]: {o.numel()} entries instead of {g.numel()}")
            if g.numel():
                rows.append(B.cast_grad_t(g.data_ptr(), o.data_ptr(), g.numel(), g.dtype == torch.bfloat16, o.dtype == torch.bfloat16))
        self.grads, self.outs = grads, outs
        self._empty = not rows
        if rows:
            with torch.cuda.device(self.device):
                rc, self._handle = B.cast_grads_create(rows)
                B.check(rc)
                rc, self._bytes = B.cast_grads_workspace(self._handle)
                B.check(rc)

    def _run(self, function, *args) -> torch.Tensor:
        if self._handle is None:
            if not self._empty:
                raise ValueError("the set is closed")
            return torch.zeros((), dtype=torch.float32, device=self.device)
        norm = torch.empty_strided((), (), dtype=torch.float32, device=self.device)
        ws = _bytes_on(self.device, self._bytes)
        _call(self.device.index, function, self._handle, *args, norm.data_ptr(), ws.data_ptr(), self._bytes)
        return norm

    def norm(self, scale: float = 1.0) -> torch.Tensor:
        """The norm of scale times all gradients, fp32 on the device."""
        return self._run(B.load_library().cast_grads_norm, scale)

    def clip(self, max_norm: float, scale: float = 1.0) -> torch.Tensor:
        """outs = grads * scale * min(1, max_norm / norm); returns the norm (of scale times all gradients, before clipping)."""
        return self._run(B.load_library().cast_grads_clip, max_norm, scale)

    def close(self) -> None:
        if self._handle is not None:
            handle, self._handle = self._handle, None
            B.check(B.cast_grads_destroy(handle))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
