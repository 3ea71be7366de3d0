"""Plain 64-bit evaluations of the norm, the rotary positions and the 8-bit rounding, for tests."""
import torch


def norm(h, w, eps):
    return w * h / (h.square().mean(-1, keepdim=True) + eps).sqrt()


def norm_grad(dy, h, w, dh, eps):
    r = 1.0 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    n, g = h * r, w * dy
    dx = r * (g - n * (g * n).mean(-1, keepdim=True))
    return dx if dh is None else dx + dh, (dy * n).reshape(-1, h.shape[-1]).sum(0)


def rotary(x, positions, frequencies, axes, adjacent, inverse):
    """x fp64 [tokens, heads, dim]; positions [axes, tokens]."""
    f = torch.tensor(frequencies, dtype=torch.float64, device=x.device)
    at = torch.tensor(axes, dtype=torch.long, device=x.device)
    angle = (positions.double()[at] * f[:, None]).T[:, None, :]
    c, s = angle.cos(), angle.sin() * (-1.0 if inverse else 1.0)
    p = len(frequencies)
    a, b = (x[..., 0:2 * p:2], x[..., 1:2 * p:2]) if adjacent else (x[..., :p], x[..., p:2 * p])
    u, v = a * c - b * s, a * s + b * c
    front = torch.stack((u, v), -1).flatten(-2) if adjacent else torch.cat((u, v), -1)
    return torch.cat((front, x[..., 2 * p:]), -1)


def to_e4m3(v):
    """Nearest e4m3 value (ties to even) of |v| <= 448, as fp64."""
    size = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -30))).clamp(min=-6)
    size = torch.where(v.abs() >= torch.exp2(size + 1), size + 1, size)
    size = torch.where((v.abs() < torch.exp2(size)) & (size > -6), size - 1, size)
    step = torch.exp2(size - 3)
    return torch.round(v / step) * step
