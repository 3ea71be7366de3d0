"""Measured cases of the language-model operators around the sparse training step: the token embedding and its
gradient, the softmax cross entropy of a linear head without stored logits, and the Newton-Schulz orthogonalisation
of an update.

Each case is a plain dict; `prepare` draws its inputs on the GPU from a seed, `run` makes one pass: with `own` false in
elementary fp32 torch operations, with `own` true through the library.  `exact` evaluates the definitions in fp64.

Definitions (T tokens, V vocabulary rows, D columns; an id or label outside [0, V) means "none"):

  embed        out[t] = scale * table[ids[t]], a zero row for no id
  embed_grad   grad_table[v] = scale * sum over {t: ids[t] = v} of grad_out[t]
  linear_ce    l = hidden weight^T, p = softmax of each row; loss[t] = logsumexp(l[t]) - l[t, label], 0 for no label;
               dl = grad_scale (p - onehot(label)), a zero row for no label; grad_hidden = dl weight,
               grad_weight = dl^T hidden
  orthogonalize  X = U / (|U|_F + eps); `steps` times X <- a X + (b A + c A A) X with A = X X^T (for more rows than
               columns X <- a X + X (b A + c A A) with A = X^T X); out = scale * X
"""
import math

import torch

own = False

A, B, C = 3.4445, -4.7750, 2.0315      # quintic of the Newton-Schulz iteration
STEPS, EPS = 5, 1e-7

LARGEST_CE = 8192 * 128256 * 4096      # tokens x vocabulary x width of the largest listed loss
LARGEST_ORTHO = 4096 * 4096 * 11008    # min(rows, cols)^2 x max(rows, cols) x matrices of the largest listed update


def listed():
    return [
        # a short continuation being scored while training on it: hardly more than reading and writing the head
        dict(name="loss-few-tokens", op="linear_ce", tokens=48, vocab=32000, dim=768, grads="both"),
        # a small decoder with a vocabulary that is no multiple of anything, batch of a ragged number of tokens
        dict(name="loss-d768-odd", op="linear_ce", tokens=1000, vocab=50257, dim=768, grads="both"),
        # one micro-batch of two sequences of 2048 through the head of a 7B-sized model
        dict(name="loss-d4096", op="linear_ce", tokens=4096, vocab=32000, dim=4096, grads="both"),
        # the same width with a large vocabulary: stored logits and their gradient would be gigabytes
        dict(name="loss-large-vocab", op="linear_ce", tokens=8192, vocab=128256, dim=4096, grads="both"),
        # perplexity of an evaluation chunk (one token short of 2048: the targets are shifted), no gradients
        dict(name="loss-eval-d5120", op="linear_ce", tokens=2047, vocab=32000, dim=5120, grads="none"),
        # one square attention projection of a small decoder: latency of a chain of dependent products
        dict(name="ortho-d768", op="orthogonalize", count=1, rows=768, cols=768, dtype="fp32"),
        # the twelve equal feed-forward matrices of the d=768 decoder in one call, bf16 updates, more rows than columns
        dict(name="ortho-d768-stack", op="orthogonalize", count=12, rows=3072, cols=768, dtype="bf16"),
        # one down projection of a 7B-sized model
        dict(name="ortho-4096x11008", op="orthogonalize", count=1, rows=4096, cols=11008, dtype="fp32"),
        # one decoding step of eight sequences
        dict(name="embed-decode", op="embed", tokens=8, vocab=32000, dim=4096, scale=1.0),
        # a training micro-batch, embeddings scaled by the root of the width
        dict(name="embed-batch", op="embed", tokens=16384, vocab=32000, dim=4096, scale=64.0),
        # gradient of a small decoder's table: mostly rows without a token
        dict(name="embed-grad-d768", op="embed_grad", tokens=1000, vocab=50257, dim=768, scale=1.0),
        # gradient of a training micro-batch: token frequencies fall like 1/rank, a few rows take hundreds of tokens
        dict(name="embed-grad-d4096", op="embed_grad", tokens=16384, vocab=32000, dim=4096, scale=64.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("linear_ce", "linear_ce", "orthogonalize", "orthogonalize", "embed", "embed_grad"))
    if op == "linear_ce":
        dim = 8 * _log_int(rng, 8, 640)
        vocab = _log_int(rng, 1000, 128256)
        tokens = _log_int(rng, 1, max(1, min(8192, LARGEST_CE // (dim * vocab))))
        return dict(op=op, tokens=tokens, vocab=vocab, dim=dim, grads=rng.choice(("both", "both", "both", "none", "hidden", "weight")))
    if op == "orthogonalize":
        rows, cols = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
        one = min(rows, cols) ** 2 * max(rows, cols)
        if one > LARGEST_ORTHO:
            rows = cols = 4096
            one = 4096 ** 3
        count = _log_int(rng, 1, max(1, min(16, LARGEST_ORTHO // one)))
        return dict(op=op, count=count, rows=rows, cols=cols, dtype=rng.choice(("fp32", "bf16")))
    tokens, vocab = _log_int(rng, 1, 16384), _log_int(rng, 1000, 32000)
    dim = _log_int(rng, 64, 4096)
    if rng.random() < 0.75:
        dim = dim // 8 * 8
    return dict(op=op, tokens=tokens, vocab=vocab, dim=dim, scale=rng.choice((1.0, 0.7071, 16.0)))


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _token_ids(g, tokens, vocab, none_share):
    """Ids whose frequencies fall like 1/rank, hot ranks spread over the table, a share of them -1 (padding)."""
    u = torch.rand(tokens, generator=g, device="cuda")
    rank = (torch.exp(u * math.log(vocab)) - 1).long().clamp_(0, vocab - 1)
    stride = next(s for s in (7919, 7907, 7901) if math.gcd(s, vocab) == 1)
    ids = (rank * stride + 11) % vocab
    none = torch.rand(tokens, generator=g, device="cuda") < none_share
    return torch.where(none, -1, ids).to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "embed" or op == "embed_grad":
        ids = _token_ids(g, case["tokens"], case["vocab"], 0.02)
        shape = (case["vocab"] if op == "embed" else case["tokens"], case["dim"])
        x = (_randn(g, *shape) * (0.02 if op == "embed" else 1e-3)).to(torch.bfloat16)
        return dict(case=case, ids=ids, x=x)
    if op == "linear_ce":
        T, V, D = case["tokens"], case["vocab"], case["dim"]
        weight = (_randn(g, V, D) * 0.02).to(torch.bfloat16)
        labels = _token_ids(g, T, V, 0.03)
        # normalised hidden states, partly aligned with their label's row: label probabilities from chance to near one
        lift = torch.rand((T, 1), generator=g, device="cuda") * (12.0 / (0.02 * math.sqrt(D)))
        toward = weight[labels.clamp(min=0).long()].float() / (0.02 * math.sqrt(D))
        hidden = (_randn(g, T, D) + lift * toward).to(torch.bfloat16)
        return dict(case=case, hidden=hidden, weight=weight, labels=labels, grad_scale=1.0 / T)
    # a momentum: a decaying spectrum of 24 directions over a floor of noise
    n, r, c = case["count"], case["rows"], case["cols"]
    rank = 24
    strength = 8.0 * 0.8 ** torch.arange(rank, device="cuda", dtype=torch.float32)
    u = _randn(g, n, r, c)
    u += (_randn(g, n, r, rank) * strength) @ _randn(g, n, rank, c) / math.sqrt(min(r, c))
    u = (u * 1e-4).to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16)
    return dict(case=case, updates=[m.clone() for m in u], scale=math.sqrt(max(1.0, r / c)))


def _run_own(s):
    from paper_2509_25996_b200 import ops
    case, op = s["case"], s["case"]["op"]
    if op == "embed":
        return ops.embed(s["x"], s["ids"], scale=case["scale"])
    if op == "embed_grad":
        return ops.embed_grad(s["x"], s["ids"], case["vocab"], scale=case["scale"])
    if op == "linear_ce":
        loss, gh, gw = ops.linear_ce(s["hidden"], s["weight"], s["labels"], grad_scale=s["grad_scale"],
                                     hidden_grad=case["grads"] in ("both", "hidden"), weight_grad=case["grads"] in ("both", "weight"))
        return [x for x in (loss, gh, gw) if x is not None]
    return ops.orthogonalize(s["updates"], steps=STEPS, coeffs=(A, B, C), eps=EPS, scale=s["scale"])


def run(s):
    if own:
        return _run_own(s)
    case, op = s["case"], s["case"]["op"]
    if op == "embed":
        valid = ((s["ids"] >= 0) & (s["ids"] < case["vocab"]))[:, None]
        rows = s["x"][s["ids"].clamp(0, case["vocab"] - 1)].float() * case["scale"]
        return torch.where(valid, rows, 0.0).to(torch.bfloat16)
    if op == "embed_grad":
        valid = ((s["ids"] >= 0) & (s["ids"] < case["vocab"]))[:, None]
        rows = torch.where(valid, s["x"].float() * case["scale"], 0.0)
        table = torch.zeros((case["vocab"], case["dim"]), device="cuda")
        return table.index_add_(0, s["ids"].clamp(0, case["vocab"] - 1), rows).to(torch.bfloat16)
    if op == "linear_ce":
        h, w, labels = s["hidden"].float(), s["weight"].float(), s["labels"]
        valid = (labels >= 0) & (labels < case["vocab"])
        at = labels.clamp(0, case["vocab"] - 1).long()[:, None]
        logits = h @ w.T
        target = logits.gather(1, at)
        top = logits.amax(1, keepdim=True)
        p = logits.sub_(top).exp_()
        total = p.sum(1, keepdim=True)
        out = [torch.where(valid, (total.log() + top - target)[:, 0], 0.0)]
        if case["grads"] == "none":
            return out
        factor = torch.where(valid, s["grad_scale"], 0.0)[:, None]
        dl = p.mul_(factor / total)
        dl.scatter_add_(1, at, -factor)
        if case["grads"] != "weight":
            out.append((dl @ w).to(torch.bfloat16))
        if case["grads"] != "hidden":
            out.append((dl.T @ h).to(torch.bfloat16))
        return out
    x = torch.stack(s["updates"]).float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    wide = case["rows"] <= case["cols"]
    for _ in range(STEPS):
        a = x @ x.mT if wide else x.mT @ x
        p = B * a + C * (a @ a)
        x = A * x + (p @ x if wide else x @ p)
    return list((s["scale"] * x).to(torch.bfloat16))


def work(case):
    op = case["op"]
    if op == "orthogonalize":
        m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        each = m * n * ((4 if case["dtype"] == "fp32" else 2) + 2)
        # A and A A are symmetric: half of their products need computing
        return dict(bytes=case["count"] * each, flops=case["count"] * STEPS * (m * m * n + m * m * m + 2 * m * m * n))
    T, V, D = case["tokens"], case["vocab"], case["dim"]
    if op == "embed":
        return dict(bytes=2 * min(T, V) * D + 2 * T * D + 4 * T, flops=T * D)
    if op == "embed_grad":
        return dict(bytes=2 * T * D + 4 * T + 2 * V * D, flops=T * D)
    gh, gw = case["grads"] in ("both", "hidden"), case["grads"] in ("both", "weight")
    return dict(bytes=2 * (T + V) * D + 8 * T + 2 * T * D * gh + 2 * V * D * gw, flops=2 * T * V * D * (1 + gh + gw))


def exact(case, seed):
    """The definitions in fp64, matrix by matrix and label by label."""
    s, op, V = prepare(case, seed), case["op"], case.get("vocab")
    if op == "embed" or op == "embed_grad":
        keep = torch.nonzero((s["ids"] >= 0) & (s["ids"] < V))[:, 0]
        ids = s["ids"][keep].long()
        if op == "embed":
            out = torch.zeros((case["tokens"], case["dim"]), dtype=torch.float64, device="cuda")
            out[keep] = s["x"].double()[ids] * case["scale"]
            return out
        order = torch.argsort(ids, stable=True)
        rows = s["x"].double()[keep[order]] * case["scale"]
        sums = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)]) if len(ids) else torch.zeros((1, case["dim"]), dtype=torch.float64, device="cuda")
        ends = torch.searchsorted(ids[order], torch.arange(V + 1, device="cuda"))
        return sums[ends[1:]] - sums[ends[:-1]]
    if op == "linear_ce":
        h, w = s["hidden"].double(), s["weight"].double()
        keep = torch.nonzero((s["labels"] >= 0) & (s["labels"] < V))[:, 0]
        label = s["labels"][keep].long()
        logits = h[keep] @ w.T
        lse = torch.logsumexp(logits, 1)
        loss = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
        loss[keep] = lse - logits[torch.arange(len(keep), device="cuda"), label]
        out = [loss]
        if case["grads"] == "none":
            return out
        d = torch.exp(logits - lse[:, None])
        del logits
        d[torch.arange(len(keep), device="cuda"), label] -= 1
        d *= s["grad_scale"]
        if case["grads"] != "weight":
            gh = torch.zeros_like(h)
            gh[keep] = d @ w
            out.append(gh)
        if case["grads"] != "hidden":
            out.append(d.T @ h[keep])
        return out
    out = []
    for u in s["updates"]:
        x = u.double() if case["rows"] <= case["cols"] else u.double().T
        x = x / (torch.linalg.norm(x) + EPS)
        for _ in range(STEPS):
            gram = x @ x.T
            x = A * x + (B * gram + C * gram @ gram) @ x
        out.append(s["scale"] * (x if case["rows"] <= case["cols"] else x.T))
    return out
