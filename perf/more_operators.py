"""Measured cases of the operators that stand between the matrices of a trained language model and before the optimizer
step: the root-mean-square norm with the residual's addition (bf16 or 8-bit output) and its gradient, rotary positions
with one or several axes, and the global gradient norm with clipping.

Each case is a plain dict; `prepare` draws its inputs on the GPU from a seed, `run` makes one pass: with `own` false in
elementary torch operations in fp32, with `own` true through the library.  `exact` evaluates the definitions in fp64.

Definitions (T tokens, D columns):

  rms_norm       h = x + residual, rounded to bf16 (h = x without a residual); y = weight h / sqrt(mean(h^2) + eps).
                 out "mx": per 32 columns of a row (the last group may be shorter) scale = the least power of two with
                 max|y| <= 448 scale, 2^-127 for a group of zeros; q = y / scale, rounded to e4m3
  rms_norm_grad  with r = 1 / sqrt(mean(h^2) + eps), g = weight grad_y, n = h r:
                 grad_x = r (g - n mean(g n)) + grad_h,   grad_weight = sum over the tokens of grad_y n
  rotary         pair i of every head of token t turns by the angle frequency[i] * positions[axis of i][t]:
                 (a, b) -> (a cos - b sin, a sin + b cos), the other way round for the gradient (inverse).  The pair is
                 (i, i + dims / 2) or, adjacent, (2 i, 2 i + 1); columns from `dims` on stay as they are
  clip           norm = scale sqrt(sum of all squares); out = grad scale min(1, max_norm / norm)
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-5

LARGEST_NORM = 16384 * 4096            # tokens x columns
LARGEST_ROTARY = 16384 * 64 * 128      # tokens x heads x columns
LARGEST_CLIP = 200_000_000             # parameters of a drawn set of gradients


def listed():
    return [
        # one decoding step of eight sequences: latency
        dict(name="norm-decode", op="rms_norm", tokens=8, dim=4096, residual=True, weight="bf16", out="bf16"),
        # a training micro-batch through the norm before a block of a 7B-sized model
        dict(name="norm-batch", op="rms_norm", tokens=16384, dim=4096, residual=True, weight="bf16", out="bf16"),
        # the same at 13B size, for block-scaled 8-bit products; a ragged number of tokens
        dict(name="norm-mx-d5120", op="rms_norm", tokens=8190, dim=5120, residual=True, weight="fp32", out="mx"),
        # one micro-batch of a small decoder, backward
        dict(name="norm-grad-d768", op="rms_norm_grad", tokens=1000, dim=768, residual=True, weight="fp32"),
        # the training micro-batch, backward; the gradient that comes down the residual stream is added
        dict(name="norm-grad-batch", op="rms_norm_grad", tokens=16384, dim=4096, residual=True, weight="bf16"),
        # one decoding step far into long contexts, eight key heads
        dict(name="rotary-decode", op="rotary", tokens=8, heads=32, key_heads=8, head_dim=128, dims=128, sections="64", base=500000.0,
             per_axis=False, adjacent=False, inverse=False, far=1 << 20),
        # a training micro-batch, queries and keys inside the output of one fused projection
        dict(name="rotary-batch", op="rotary", tokens=16384, heads=32, key_heads=32, head_dim=128, dims=128, sections="64", base=10000.0,
             per_axis=False, adjacent=False, inverse=False, far=4096),
        # gradients of video tokens: (time, height, width), every axis with frequencies of its own, adjacent pairs
        dict(name="rotary-video-grad", op="rotary", tokens=8190, heads=24, key_heads=24, head_dim=128, dims=128, sections="16,24,24", base=10000.0,
             per_axis=True, adjacent=True, inverse=True, far=512),
        # gradients of one feed-forward matrix that is tuned alone: latency
        dict(name="clip-one-matrix", op="clip", layers=1, matrices="2048x768", vocab=0, dim=768, vectors=1, grad="fp32", out="bf16", align=64,
             scale=0.25, max_norm=1.0),
        # a whole small decoder with its table and norms, gradients accumulated in fp32 over eight micro-batches
        dict(name="clip-d768", op="clip", layers=12, matrices="768x768,768x768,768x768,768x768,768x2304,2304x768", vocab=50257, dim=768, vectors=2,
             grad="fp32", out="bf16", align=64, scale=0.125, max_norm=1.0),
        # eight layers (a pipeline stage) of a 7B-sized model, the same way: far more than the caches hold
        dict(name="clip-7b-stage", op="clip", layers=8, matrices="4096x4096,4096x4096,4096x4096,4096x4096,11008x4096,11008x4096,4096x11008", vocab=0,
             dim=4096, vectors=2, grad="fp32", out="bf16", align=64, scale=0.125, max_norm=1.0),
        # half of the layers of a 7B-sized model and its table, bf16 gradients from a backward pass into the optimizer's buffer
        dict(name="clip-7b-half", op="clip", layers=16, matrices="4096x4096,4096x4096,4096x4096,4096x4096,11008x4096,11008x4096,4096x11008", vocab=32000,
             dim=4096, vectors=2, grad="bf16", out="bf16", align=64, scale=1.0, max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rms_norm", "rms_norm", "rms_norm_grad", "rms_norm_grad", "rotary", "rotary", "clip"))
    if op in ("rms_norm", "rms_norm_grad"):
        dim = _log_int(rng, 64, 8192)
        if rng.random() < 0.75:
            dim = dim // 8 * 8
        tokens = _log_int(rng, 1, min(262144, LARGEST_NORM // dim))
        case = dict(op=op, tokens=tokens, dim=dim, residual=rng.random() < 0.6, weight=rng.choice(("bf16", "fp32")))
        if op == "rms_norm":
            case["out"] = rng.choice(("bf16", "bf16", "mx"))
        return case
    if op == "rotary":
        head_dim = rng.choice((64, 80, 96, 128, 192, 256))
        dims = head_dim if rng.random() < 0.7 else rng.randrange(8, head_dim + 1, 2)
        heads = _log_int(rng, 1, 64)
        key_heads = rng.randint(0, heads)
        axes = rng.choice((1, 1, 2, 3)) if dims >= 12 else 1
        cuts = sorted(rng.sample(range(1, dims // 2), axes - 1)) if axes > 1 else []
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [dims // 2]))
        tokens = _log_int(rng, 1, min(16384, LARGEST_ROTARY // ((heads + key_heads) * head_dim)))
        return dict(op=op, tokens=tokens, heads=heads, key_heads=key_heads, head_dim=head_dim, dims=dims, sections=sections,
                    base=rng.choice((10000.0, 500000.0, 1000000.0)), per_axis=rng.random() < 0.4, adjacent=rng.random() < 0.4,
                    inverse=rng.random() < 0.4, far=_log_int(rng, 64, 1 << 20))
    dim = _log_int(rng, 32, 4096)
    ffn = _log_int(rng, 32, 11008)
    matrices = ",".join(rng.choice(("%dx%d" % (dim, dim), "%dx%d" % (ffn, dim), "%dx%d" % (dim, ffn))) for _ in range(rng.randint(1, 7)))
    vocab = rng.choice((0, _log_int(rng, 100, 50257)))
    one = sum(math.prod(map(int, m.split("x"))) for m in matrices.split(","))
    vocab = min(vocab, LARGEST_CLIP // (2 * dim))
    layers = _log_int(rng, 1, max(1, min(48, (LARGEST_CLIP - vocab * dim) // one)))
    grad = rng.choice(("fp32", "fp32", "bf16"))
    return dict(op=op, layers=layers, matrices=matrices, vocab=vocab, dim=dim, vectors=rng.randint(0, 2), grad=grad,
                out=rng.choice(("bf16", "bf16", grad)), align=rng.choice((64, 64, 1)), scale=rng.choice((1.0, 0.125, 1.0 / 3.0)),
                max_norm=rng.choice((1.0, 0.1, 1e4)))


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _counts(case):
    """Entries of every matrix and of every vector (norm weights) of the set."""
    per_layer = [math.prod(map(int, m.split("x"))) for m in case["matrices"].split(",")]
    return per_layer * case["layers"] + ([case["vocab"] * case["dim"]] if case["vocab"] else []), [case["dim"]] * (case["vectors"] * case["layers"])


def _places(counts, align):
    """Where each tensor begins in one flat buffer, and the buffer's length."""
    at, places = 0, []
    for n in counts:
        places.append(at)
        at += -(-n // align) * align
    return places, at


def _frequencies(case):
    """(frequency in radians per position, axis) of every pair."""
    sections = [int(s) for s in case["sections"].split(",")]
    pairs, out = sum(sections), []
    for axis, n in enumerate(sections):
        for j in range(n):
            share = j / n if case["per_axis"] else len(out) / pairs
            out.append((case["base"] ** -share, axis))
    return out


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    if op in ("rms_norm", "rms_norm_grad"):
        T, D = case["tokens"], case["dim"]
        weight = (1.0 + 0.2 * _randn(g, D)).to(_type(case["weight"]))
        # a residual stream: tokens of different size, a few columns far larger than the others
        size = torch.exp(0.5 * _randn(g, T, 1)) * torch.where(torch.rand(D, generator=g, device=DEVICE) < 0.004, 20.0, 1.0)
        stream = (_randn(g, T, D) * size).to(torch.bfloat16)
        other = (_randn(g, T, D) * (0.5 if op == "rms_norm" else 1e-3)).to(torch.bfloat16)
        if op == "rms_norm":
            return dict(case=case, weight=weight, x=other if case["residual"] else stream, residual=stream if case["residual"] else None)
        grad_h = (_randn(g, T, D) * 1e-3).to(torch.bfloat16) if case["residual"] else None
        return dict(case=case, weight=weight, h=stream, grad_y=other, grad_h=grad_h)
    if op == "rotary":
        T, H, K, D = case["tokens"], case["heads"], case["key_heads"], case["head_dim"]
        fused = _randn(g, T, (H + 2 * K) * D).to(torch.bfloat16)
        q = fused[:, :H * D].view(T, H, D)
        k = fused[:, H * D:(H + K) * D].view(T, K, D) if K else None
        axes = len(case["sections"].split(","))
        positions = torch.randint(0, case["far"], (axes, T), generator=g, device=DEVICE, dtype=torch.int32)
        frequencies, axis = zip(*_frequencies(case))
        state = dict(case=case, q=q, k=k, positions=positions, axis=torch.tensor(axis, device=DEVICE),
                     frequencies=torch.tensor(frequencies, dtype=torch.float64, device=DEVICE)[:, None])
        if own:
            from paper_2509_25996_b200 import ops
            state["spectrum"] = ops.RotarySpectrum(frequencies, axes=axis, adjacent=case["adjacent"])
        return state
    matrices, vectors = _counts(case)
    state = dict(case=case)
    grads, outs = [], []
    for key, counts, kind in (("m", matrices, case["grad"]), ("v", vectors, "fp32")):
        places, total = _places(counts, case["align"])
        flat = torch.zeros(total, dtype=_type(kind), device=DEVICE)
        # every tensor's gradients are of a size of their own
        sizes = (1e-3 * torch.exp(torch.randn(len(counts), generator=g, device=DEVICE))).tolist()
        for at, n, size in zip(places, counts, sizes):
            part = flat[at:at + n]
            for b in range(0, n, 1 << 27):
                part[b:b + (1 << 27)].copy_(_randn(g, min(n - b, 1 << 27)).mul_(size))
            grads.append(part)
        state[key] = flat
        flat = torch.zeros(total, dtype=_type(case["out"] if key == "m" else kind), device=DEVICE)
        state["out_" + key] = flat
        outs += [flat[at:at + n] for at, n in zip(places, counts)]
    if own:
        from paper_2509_25996_b200 import ops
        state["set"] = ops.GradientSet(grads, outs)
    return state


def _run_own(s):
    from paper_2509_25996_b200 import ops
    case, op = s["case"], s["case"]["op"]
    if op == "rms_norm":
        call = ops.rms_norm if case["out"] == "bf16" else ops.rms_norm_mx
        got = call(s["x"], s["weight"], s["residual"], eps=EPS)
        return got if case["residual"] else got[:-1]
    if op == "rms_norm_grad":
        return ops.rms_norm_grad(s["grad_y"], s["h"], s["weight"], s["grad_h"], eps=EPS)
    if op == "rotary":
        q, k = ops.rotary(s["q"], s["k"], s["positions"], s["spectrum"], inverse=case["inverse"])
        return [q] if k is None else [q, k]
    return [s["set"].clip(case["max_norm"], scale=case["scale"]), s["out_m"], s["out_v"]]


def _turned(x, cos, sin, dims, adjacent):
    x = x.float()
    a, b = (x[..., 0:dims:2], x[..., 1:dims:2]) if adjacent else (x[..., :dims // 2], x[..., dims // 2:dims])
    c, d = a * cos - b * sin, a * sin + b * cos
    front = torch.stack((c, d), -1).flatten(-2) if adjacent else torch.cat((c, d), -1)
    return torch.cat((front, x[..., dims:]), -1).to(torch.bfloat16)


def _to_mx(y):
    """(e4m3 values, their scales) of fp32 rows in groups of 32 columns."""
    T, D = y.shape
    groups = -(-D // 32)
    y = torch.nn.functional.pad(y, (0, groups * 32 - D)).view(T, groups, 32)
    fraction, exponent = torch.frexp(y.abs().amax(-1, keepdim=True) / 448.0)
    exponent = torch.where(fraction == 0.0, -127, exponent - (fraction == 0.5).int()).clamp(min=-127)
    scale = torch.ldexp(torch.ones_like(fraction), exponent)
    q = (y / scale).view(T, groups * 32)[:, :D].to(torch.float8_e4m3fn)
    return q, scale.view(T, groups).to(torch.float8_e8m0fnu)


def run(s):
    if own:
        return _run_own(s)
    case, op = s["case"], s["case"]["op"]
    if op == "rms_norm":
        h, out = s["x"], []
        if case["residual"]:
            h = (h.float() + s["residual"].float()).to(torch.bfloat16)
            out = [h]
        x = h.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["weight"].float()
        return ([y.to(torch.bfloat16)] if case["out"] == "bf16" else list(_to_mx(y))) + out
    if op == "rms_norm_grad":
        x, dy = s["h"].float(), s["grad_y"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n, g = x * r, dy * s["weight"].float()
        dx = r * (g - n * (g * n).mean(-1, keepdim=True))
        if case["residual"]:
            dx = dx + s["grad_h"].float()
        return [dx.to(torch.bfloat16), (dy * n).sum(0)]
    if op == "rotary":
        angle = (s["positions"][s["axis"]].double() * s["frequencies"]).T[:, None, :]
        cos, sin = angle.cos().float(), angle.sin().float()
        if case["inverse"]:
            sin = -sin
        return [_turned(x, cos, sin, case["dims"], case["adjacent"]) for x in (s["q"], s["k"]) if x is not None]
    m, v = s["m"], s["v"]
    total = (m.float().square().sum(dtype=torch.float64) + v.square().sum(dtype=torch.float64)).sqrt() * case["scale"]
    factor = (case["scale"] * (case["max_norm"] / total).clamp(max=1.0)).float()
    return [total.float(), (m.float() * factor).to(_type(case["out"])), v * factor]


def work(case):
    op = case["op"]
    if op == "clip":
        matrices, vectors = (sum(c) for c in _counts(case))
        size = {"fp32": 4, "bf16": 2}
        return dict(bytes=(size[case["grad"]] + size[case["out"]]) * matrices + 8 * vectors, flops=3 * (matrices + vectors))
    if op == "rotary":
        n = case["tokens"] * (case["heads"] + case["key_heads"]) * case["head_dim"]
        return dict(bytes=4 * n + 4 * case["tokens"] * len(case["sections"].split(",")), flops=3 * n)
    T, D = case["tokens"], case["dim"]
    weight = D * (4 if case["weight"] == "fp32" else 2)
    if op == "rms_norm":
        out = 2 * T * D if case["out"] == "bf16" else T * D + T * -(-D // 32)
        return dict(bytes=T * D * (6 if case["residual"] else 2) + out + weight, flops=(6 if case["residual"] else 5) * T * D)
    return dict(bytes=T * D * (8 if case["residual"] else 6) + weight + 4 * D, flops=12 * T * D)


def exact(case, seed):
    """The definitions in fp64."""
    s, op = prepare(case, seed), case["op"]
    if op == "rms_norm":
        x, stored = s["x"].double(), []
        if case["residual"]:
            x = (x + s["residual"].double()).to(torch.bfloat16).double()
            stored = [x]
        y = s["weight"].double() * x / (torch.linalg.vector_norm(x, dim=1, keepdim=True).square() / case["dim"] + EPS).sqrt()
        if case["out"] == "bf16":
            return [y] + stored
        q, scales = torch.empty_like(y), []
        for c in range(0, case["dim"], 32):
            part = y[:, c:c + 32]
            top = part.abs().max(1, keepdim=True).values
            k = torch.ceil(torch.log2(top / 448.0)).clamp(-127, 127)
            k = k - ((448.0 * torch.exp2(k - 1)) >= top).double()        # log2 is rounded: the least power that still holds
            k = torch.where(448.0 * torch.exp2(k) < top, k + 1, k).clamp(min=-127)
            value = part * torch.exp2(-k)
            size = torch.floor(torch.log2(value.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
            step = torch.exp2(size - 3)
            q[:, c:c + 32] = torch.round(value / step) * step
            scales.append(torch.exp2(k))
        return [q, torch.cat(scales, 1)] + stored
    if op == "rms_norm_grad":
        D = case["dim"]
        x, dy, w = s["h"].double(), s["grad_y"].double(), s["weight"].double()
        ms = torch.einsum("td,td->t", x, x)[:, None] / D + EPS
        inner = torch.einsum("td,td,d->t", x, dy, w)[:, None] / D
        dx = (dy * w - x * (inner / ms)) / ms.sqrt()
        if case["residual"]:
            dx = dx + s["grad_h"].double()
        return [dx, torch.einsum("td,td->d", dy, x / ms.sqrt())]
    if op == "rotary":
        out = []
        for x in (s["q"], s["k"]):
            if x is None:
                continue
            y = x.double()
            half = case["dims"] // 2
            for i, (f, axis) in enumerate(_frequencies(case)):
                turn = torch.polar(torch.ones(case["tokens"], dtype=torch.float64, device=x.device),
                                   s["positions"][axis].double() * (-f if case["inverse"] else f))
                a, b = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + half)
                z = torch.complex(x[..., a].double(), x[..., b].double()) * turn[:, None]
                y[..., a], y[..., b] = z.real, z.imag
            out.append(y)
        return out
    square = sum(torch.linalg.vector_norm(part.double()).square()
                 for flat in (s["m"], s["v"]) for part in flat.split(1 << 27))
    norm = case["scale"] * square.sqrt()
    factor = case["scale"] * min(1.0, case["max_norm"] / float(norm))
    return [norm, s["m"].double() * factor, s["v"].double() * factor]
