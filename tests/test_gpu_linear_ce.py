"""cast_linear_ce against a plain 64-bit evaluation on the same bf16 inputs.

Tolerances.  With A_i = max_j sum_k |h_ik w_jk|: a logit is a sum of exact products in fp32, taken 16 at a time, so its error
is at most (dim/16 + 4) 2^-23 A_i; the exponent's argument adds 2^-22 of the largest |logit|, the row sums (128 terms in
sequence, then a tree) 160 2^-24, ex2 2^-22:
    eps_i   = 2 (dim/16 + 4) 2^-23 A_i + 2^-21 max|l_i| + 1.2e-5           (relative error of 1 + S and of S)
    loss    |cuda - exact| <= eps_i
    dH      <= 2^-8 |exact| + s sum_{j != label} p_ij |w_jk| (2^-8 + eps_i + vocab 2^-27) + s (1 - p_label) |w_label,k| (eps_i + 2^-22)
    dW      <= 2^-8 |exact| + s sum_{i: label != j} p_ij |h_ik| (3 2^-8 + eps_i + tokens 2^-27)
                            + s sum_{i: label = j} (1 - p_ij) |h_ik| (eps_i + tokens 2^-23)
(operands of the backward products are rounded to bf16, 2^-9 each; results are rounded to bf16, dW of a row with labels twice)."""
import math

import pytest
import torch

import paper_2509_25996_b200 as cast
from paper_2509_25996_b200 import binding as B
from paper_2509_25996_b200 import ops
import gpu_util as U

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def draw(tokens, vocab, dim, seed, lift=6.0):
    """Hidden states partly aligned with the label's row: target probabilities from chance to near one."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (torch.randn((vocab, dim), generator=g, device=DEV) / math.sqrt(dim)).to(torch.bfloat16)
    y = torch.randint(0, vocab, (tokens,), generator=g, device=DEV).int()
    h = torch.randn((tokens, dim), generator=g, device=DEV) + torch.rand((tokens, 1), generator=g, device=DEV) * lift * w[y.long()].float()
    return h.to(torch.bfloat16), w, y


def exact(h, w, y, s):
    h, w = h.double(), w.double()
    vocab, dim = w.shape
    tokens = h.shape[0]
    rows = torch.nonzero((y >= 0) & (y < vocab))[:, 0]
    label = y[rows].long()
    hr = h[rows]
    l = hr @ w.T
    lse = torch.logsumexp(l, 1)
    at = torch.arange(len(rows), device=DEV)
    loss, eps = torch.zeros(tokens, dtype=torch.float64, device=DEV), torch.zeros(tokens, dtype=torch.float64, device=DEV)
    others = torch.exp(l - l[at, label][:, None])
    others[at, label] = 0.0
    loss[rows] = torch.log1p(others.sum(1))             # = lse - l_label, without its cancellation
    size = (hr.abs() @ w.abs().T).amax(1)
    e = 2 * (dim / 16 + 4) * 2.0 ** -23 * size + 2.0 ** -21 * l.abs().amax(1) + 1.2e-5
    eps[rows] = e
    p = torch.exp(l - lse[:, None])
    p[at, label] = 0.0                                  # the other columns
    rest = p.sum(1)                                     # 1 - p_label, without its cancellation
    s = abs(s), (1.0 if s >= 0 else -1.0)
    gh, bh = torch.zeros_like(h), torch.zeros_like(h)
    gh[rows] = s[0] * s[1] * (p @ w - rest[:, None] * w[label])
    bh[rows] = s[0] * ((p * (2.0 ** -8 + e[:, None] + vocab * 2.0 ** -27)) @ w.abs() + (rest * (e + 2.0 ** -22))[:, None] * w[label].abs())
    gw = s[0] * s[1] * (p.T @ hr).index_add_(0, label, -rest[:, None] * hr)
    bw = s[0] * ((p * (3 * 2.0 ** -8 + e[:, None] + tokens * 2.0 ** -27)).T @ hr.abs()).index_add_(
        0, label, (rest * (e + tokens * 2.0 ** -23))[:, None] * hr.abs())
    return (loss, eps), (gh, 2.0 ** -8 * gh.abs() + bh + 1e-37), (gw, 2.0 ** -8 * gw.abs() + bw + 1e-37)


def run(h, w, y, s, want_h=True, want_w=True, piece=0):
    (tokens, dim), vocab = h.shape, w.shape[0]
    gl, gh, gw = (U.Guarded(n, t, DEV) for n, t in ((tokens, torch.float32), (tokens * dim, torch.bfloat16), (vocab * dim, torch.bfloat16)))
    rc, need = cast.cast_linear_ce_workspace(tokens, vocab, dim, piece, want_h, want_w)
    cast.check(rc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)        # NaN patterns: nothing may be read before it is written
    cast.check(cast.cast_linear_ce(h, w, y, gl.view, gh.view if want_h else None, gw.view if want_w else None, tokens, vocab, dim, s, piece,
                                   ws, need, torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert gl.intact() and gh.intact() and gw.intact() and bool((ws[need:] == 255).all())
    assert cast.cast_product_failures() == (0, 0)
    return gl.view, gh.view.reshape(tokens, dim), gw.view.reshape(vocab, dim)


def close(got, pair, what):
    want, bound = pair
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), f"{what}: worst {float((err / bound).nan_to_num(nan=math.inf).max()):.3g} x the bound"


def check(h, w, y, s, label="", **kw):
    loss, gh, gw = run(h, w, y, s, **kw)
    l, a, b = exact(h, w, y, s)
    close(loss, l, f"{label} loss")
    if kw.get("want_h", True):
        close(gh, a, f"{label} dH")
    if kw.get("want_w", True):
        close(gw, b, f"{label} dW")
    return loss, gh, gw


SHAPES = [(1, 1, 8), (1, 2, 8), (1, 1000, 64), (2, 63, 16), (17, 130, 72), (64, 256, 64), (127, 1003, 264), (128, 5000, 768), (129, 257, 256),
          (200, 32000, 128), (257, 513, 520), (512, 4096, 512), (1000, 50257, 96), (1, 32000, 4096)]


@pytest.mark.parametrize("tokens,vocab,dim", SHAPES)
def test_shapes(tokens, vocab, dim):
    h, w, y = draw(tokens, vocab, dim, tokens + vocab)
    check(h, w, y, 1.0 / tokens, f"{tokens}x{vocab}x{dim}")


@pytest.mark.parametrize("tokens,piece", [(700, 256), (700, 100), (513, 256), (300, 129), (5, 1), (1024, 512)])
def test_pieces_of_tokens(tokens, piece):
    h, w, y = draw(tokens, 1500, 136, tokens)
    y[3 % tokens] = -1
    loss, gh, gw = check(h, w, y, 0.5, f"{tokens} in pieces of {piece}", piece=piece)
    whole = run(h, w, y, 0.5)
    close(gw, (whole[2].double(), 2 * exact(h, w, y, 0.5)[2][1]), "pieces against whole")


@pytest.mark.parametrize("tokens", [40, 300])
def test_single_results_are_those_of_the_full_call(tokens):
    h, w, y = draw(tokens, 900, 128, 5)
    loss, gh, gw = run(h, w, y, -2.0)
    check(h, w, y, -2.0, "negative scale")
    only, _, _ = run(h, w, y, -2.0, want_h=False, want_w=False)
    assert torch.equal(only, loss)
    l2, h2, _ = run(h, w, y, -2.0, want_w=False)
    assert torch.equal(l2, loss) and torch.equal(h2, gh)
    l3, _, w3 = run(h, w, y, -2.0, want_h=False)
    assert torch.equal(l3, loss) and torch.equal(w3, gw)


@pytest.mark.parametrize("tokens", [100, 400])
def test_tokens_without_a_label(tokens):
    h, w, y = draw(tokens, 600, 64, 7)
    y[::3] = -1
    y[1] = 600
    y[2] = 2 ** 31 - 1
    y[tokens - 1] = -2 ** 31
    loss, gh, gw = check(h, w, y, 1.0, "some without a label")
    none = (y < 0) | (y >= 600)
    assert not loss[none].any() and not gh[none].any()
    # what those tokens hold does not matter
    h2 = h.clone()
    h2[none] = float("nan")
    h2[none.nonzero()[0, 0]] = float("inf")
    again = run(h2, w, y, 1.0)
    assert all(torch.equal(a, b) for a, b in zip((loss, gh, gw), again))
    # none at all
    loss, gh, gw = run(h, w, torch.full_like(y, -100), 1.0)
    assert not loss.any() and not gh.any() and not gw.any()


def test_equal_labels_and_confident_tokens():
    """All tokens on one label (one long sum), and targets so likely that 1 - p underflows a subtraction in fp32."""
    h, w, y = draw(500, 700, 256, 8, lift=60.0)
    y[:] = 123
    h[:250] = (torch.randn((250, 256), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) * 0.2 + 45.0 * w[123].float()).to(torch.bfloat16)
    loss, _, _ = check(h, w, y, 1.0, "one label")
    assert float(loss[:250].max()) < 1e-4
    ref = exact(h, w, y, 1.0)[0][0][:250]
    assert float(((loss[:250].double() - ref).abs() / ref).max()) < 1e-2        # small losses keep their leading digits


@pytest.mark.parametrize("gap", [30.0, 39.0, 45.0, 80.0, 200.0])
@pytest.mark.parametrize("tokens", [20, 300])
def test_improbable_targets(gap, tokens):
    """Other logits far above the target's: beyond e^40 the row is brought to another reference."""
    vocab, dim = 1300, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    w = (torch.randn((vocab, dim), generator=g, device=DEV) / 8).to(torch.bfloat16)
    y = torch.randint(0, vocab, (tokens,), generator=g, device=DEV).int()
    h = torch.randn((tokens, dim), generator=g, device=DEV).to(torch.bfloat16)
    # one column pushes a single other logit up by about `gap` for every second token
    w[:, 0] = 0.0
    w[777, 0] = 1.0
    h[:, 0] = 0.0
    h[::2, 0] = gap
    y[y == 777] = 5
    check(h, w, y, 1.0 / tokens, f"gap {gap}")
    check(h, w, y, 1.0 / tokens, f"gap {gap} in pieces", piece=max(1, tokens // 3))


def test_extreme_values():
    """Large logits of both signs; a vocabulary whose other rows are all far below the target."""
    h, w, y = draw(150, 300, 64, 12)
    check((h.float() * 30).to(torch.bfloat16), w, y, 1.0, "logits of hundreds")
    w2 = w.clone()
    w2[:] = -50.0
    w2[y[0].long()] = 50.0
    h2 = torch.ones_like(h)
    loss, gh, gw = run(h2, w2, torch.full_like(y, int(y[0])), 1.0)
    assert not loss.any() and not gh.any() and not gw.any()


def test_gradients_against_differences():
    """Central differences of the kernel's own loss along directions that keep the inputs exact in bf16.  The third
    derivative of logsumexp along u is at most range(u)^3; the losses carry eps each."""
    tokens, vocab, dim = 60, 200, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    w = (torch.randint(-8, 9, (vocab, dim), generator=g, device=DEV) / 16).to(torch.bfloat16)
    h = (torch.randint(-8, 9, (tokens, dim), generator=g, device=DEV) / 16).to(torch.bfloat16)
    y = torch.randint(0, vocab, (tokens,), generator=g, device=DEV).int()
    y[5] = -1
    _, gh, gw = run(h, w, y, 1.0)
    step = 1.0 / 64
    dh = (torch.randint(0, 2, (tokens, dim), generator=g, device=DEV) * 2 - 1).to(torch.bfloat16)
    dw = (torch.randint(0, 2, (vocab, dim), generator=g, device=DEV) * 2 - 1).to(torch.bfloat16)
    (_, eps), _, _ = exact(h, w, y, 1.0)
    for name, moved, inner, span in (
            ("hidden", lambda t: run((h + t * dh), w, y, 1.0, False, False)[0], float((gh.double() * dh.double()).sum()), dh.double() @ w.double().T),
            ("weight", lambda t: run(h, (w + t * dw), y, 1.0, False, False)[0], float((gw.double() * dw.double()).sum()), h.double() @ dw.double().T)):
        up, down = moved(step), moved(-step)
        slope = float((up.double() - down.double()).sum()) / (2 * step)
        width = (span.amax(1) - span.amin(1))
        tol = float((2 * eps).sum()) / (2 * step) + step ** 2 / 6 * float((width ** 3).sum()) + 2.0 ** -8 * float(
            ((gh.double() if name == "hidden" else gw.double()).abs()).sum())
        assert abs(slope - inner) <= tol, (name, slope, inner, tol)
        assert tol < 0.5 * abs(float(((gh if name == "hidden" else gw).double().abs()).sum()))        # the bound says something


def test_more_exponentials_than_32_bits_address():
    """One piece whose exponentials are more than 2^31: the last tokens' results against the same tokens on their own."""
    tokens, vocab, dim = 17000, 128256, 64
    h, w, y = draw(tokens, vocab, dim, 21)
    loss, gh, gw = run(h, w, y, 1.0, piece=tokens)
    tail = slice(tokens - 300, tokens)
    (l, eps), (a, ba), _ = exact(h[tail], w, y[tail], 1.0)
    close(loss[tail], (l, eps), "loss")
    close(gh[tail], (a, ba), "dH")
    cols = torch.randint(0, vocab, (64,), device=DEV)
    part, size = torch.zeros((64, dim), dtype=torch.float64, device=DEV), torch.zeros((64, dim), dtype=torch.float64, device=DEV)
    for t0 in range(0, tokens, 2000):
        hd = h[t0:t0 + 2000].double()
        logits = hd @ w.double().T
        p = torch.exp(logits[:, cols] - torch.logsumexp(logits, 1, keepdim=True))
        hot = (y[t0:t0 + 2000, None] == cols[None]).double()
        part += (p - hot).T @ hd
        size += (p + hot).T @ hd.abs()
    err = (gw[cols].double() - part).abs()
    assert bool((err <= 2.0 ** -8 * part.abs() + size * (4 * 2.0 ** -8 + tokens * 2.0 ** -23)).all())


def test_repeatable_on_any_stream():
    h, w, y = draw(700, 3000, 200, 30)
    one = ops.linear_ce(h, w, y, 0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        two = ops.linear_ce(h, w, y, 0.1)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    loss, gh, gw = ops.linear_ce(h[:0], w, y[:0])
    assert loss.numel() == 0 and gh.shape == (0, 200) and not gw.any()


def test_graph_capture():
    h, w, y = draw(100, 900, 64, 31)
    want = ops.linear_ce(h, w, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.linear_ce(h, w, y)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals():
    h, w, y = draw(10, 50, 64, 32)
    loss, gh, gw = torch.empty(10, device=DEV), torch.empty_like(h), torch.empty_like(w)
    need = cast.cast_linear_ce_workspace(10, 50, 64)[1]
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    before = cast.cast_kernel_launch_count()

    def call(**over):
        a = dict(hidden=h, weight=w, labels=y, loss=loss, grad_hidden=gh, grad_weight=gw, tokens=10, vocab=50, dim=64, grad_scale=1.0, piece_tokens=0,
                 workspace=ws, workspace_bytes=need)
        a.update(over)
        return cast.cast_linear_ce(**a)
    assert call(workspace_bytes=need - 1) == B.CAST_ERR_PLAN
    assert call(grad_hidden=h) == B.CAST_ERR_ALIAS
    assert call(grad_weight=gh) == B.CAST_ERR_ALIAS
    assert call(loss=ws) == B.CAST_ERR_ALIAS
    assert call(labels=y.cpu()) == B.CAST_ERR_MEMORY
    assert cast.cast_kernel_launch_count() == before
    with pytest.raises(ValueError, match="columns"):
        ops.linear_ce(h, w[:, :32].contiguous(), y)
    with pytest.raises(ValueError, match="not contiguous"):
        ops.linear_ce(h, w[:, :32], y)
    with pytest.raises(ValueError, match="labels"):
        ops.linear_ce(h, w, y[:5])
    with pytest.raises(cast.CastError):
        ops.linear_ce(h[:, :60].contiguous(), w[:, :60].contiguous(), y)


def test_a_counted_failure_stops_further_calls():
    """What a product that gives up a wait does to the calls after it, with the count set on the host."""
    h, w, y = draw(10, 50, 64, 33)
    want = ops.linear_ce(h, w, y)
    assert cast.cast_product_failures(1) == (0, 0)
    try:
        with pytest.raises(cast.CastError) as e:
            ops.linear_ce(h, w, y)
        assert e.value.status == B.CAST_ERR_STAGING
        with pytest.raises(cast.CastError):
            ops.orthogonalize([torch.ones((8, 8), device=DEV)])
    finally:
        assert cast.cast_product_failures(2) == (0, 1)
    assert all(torch.equal(a, b) for a, b in zip(want, ops.linear_ce(h, w, y)))


@pytest.mark.parametrize("captured", [False, True])
def test_work_behind_a_call_without_any_label(captured):
    """A copy of grad_weight on the same stream, directly behind a call none of whose tokens has a label, sees the finished
    product: zeros everywhere.  (200 tokens into 100000 x 2048: the product stores 410 MB.)"""
    tokens, vocab, dim = 200, 100000, 2048
    h, w, y = draw(tokens, vocab, dim, 41)
    y.fill_(-1)
    gw = torch.empty_like(w)
    seen = torch.empty_like(w)
    loss = torch.empty(tokens, device=DEV)
    need = cast.cast_linear_ce_workspace(tokens, vocab, dim, 0, False, True)[1]
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def enqueue():
        gw.fill_(7.0)
        cast.check(cast.cast_linear_ce(h, w, y, loss, None, gw, tokens, vocab, dim, 1.0, 0, ws, need, torch.cuda.current_stream()))
        seen.copy_(gw)
    if captured:
        run(h[:2], w[:4], y[:2], 1.0)              # what a first call allocates
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            enqueue()
    for _ in range(5):
        seen.fill_(3.0)
        if captured:
            graph.replay()
        else:
            enqueue()
        torch.cuda.synchronize()
        assert not seen.any() and not loss.any()


@pytest.mark.parametrize("tokens,vocab,dim,piece", [(4096, 512, 256, 0), (200, 300, 256, 0), (700, 3000, 136, 300), (3000, 40, 64, 0), (900, 70, 72, 400)])
@pytest.mark.parametrize("mean", [0.5, 1.0])
def test_rows_whose_terms_cancel(tokens, vocab, dim, piece, mean):
    """A calibrated head: labels drawn from the model's own probabilities, hidden states with a common mean, one label that is
    frequent.  The two parts of its row of dW nearly cancel, so neither may be rounded before their difference is.  Per row j, in norm:
    the result's rounding, 2^-8 |exact|; the operands' (two of at most 2^-8, independent from token to token, six deviations:
    6 sqrt(2/3) < 5), 5 2^-8 sqrt(sum p_ij^2 |h_i|^2); and the relative error eps_i of the probabilities."""
    g = torch.Generator(device=DEV).manual_seed(tokens + dim)
    mu = torch.randn(dim, generator=g, device=DEV) * mean
    w = torch.randn((vocab, dim), generator=g, device=DEV) * 0.02
    w[7] += 6.0 * mu / mu.square().sum()
    w = w.to(torch.bfloat16)
    h = (torch.randn((tokens, dim), generator=g, device=DEV) + mu).to(torch.bfloat16)
    p = torch.softmax(h.double() @ w.double().T, 1)
    u = torch.rand((tokens, 1), generator=g, device=DEV).double()
    y = (p.cumsum(1) < u).sum(1).clamp(max=vocab - 1).int()
    _, _, gw = check(h, w, y, 1.0, "calibrated head", piece=piece)
    (_, eps), _, (want, _) = exact(h, w, y, 1.0)
    size = h.double().norm(dim=1)
    hot = torch.nn.functional.one_hot(y.long(), vocab).double()
    q = p * (1 - hot)
    bound = 2.0 ** -8 * want.norm(dim=1) + 5 * 2.0 ** -8 * (q.square().T @ size.square()).sqrt() + (q + (1 - p) * hot).T @ ((eps + 2.0 ** -22) * size)
    err = (gw.double() - want).norm(dim=1)
    assert bool((err <= bound).all()), f"worst {float((err / bound).max()):.3g} x the bound, row {int((err / bound).argmax())}"


@pytest.mark.parametrize("dim", [768, 4096, 16384])
def test_logits_whose_sums_are_exact(dim):
    """Sparse small integers: every partial sum of a logit is exact in fp32, on whichever unit, so the first term of eps_i falls
    away and the loss is within 2^-21 max|l_i| + 1.2e-5."""
    tokens, vocab = 300, 1000
    g = torch.Generator(device=DEV).manual_seed(dim)
    h, w = torch.zeros((tokens, dim), device=DEV), torch.zeros((vocab, dim), device=DEV)
    cols = torch.randperm(dim, generator=g, device=DEV)[:16]
    h[:, cols] = torch.randint(0, 3, (tokens, 16), generator=g, device=DEV).float()
    w[:, cols] = torch.randint(-1, 3, (vocab, 16), generator=g, device=DEV).float()
    h, w = h.to(torch.bfloat16), w.to(torch.bfloat16)
    y = torch.randint(0, vocab, (tokens,), generator=g, device=DEV).int()
    loss, _, _ = run(h, w, y, 1.0, want_h=False, want_w=False)
    (want, _), _, _ = exact(h, w, y, 1.0)
    top = (h.double() @ w.double().T).abs().amax(1)
    assert float(top.max()) > 25.0
    err = (loss.double() - want).abs() / (2.0 ** -21 * top + 1.2e-5)
    assert float(err.max()) <= 1.0, f"worst {float(err.max()):.3g} x the bound"


@pytest.mark.parametrize("tokens", [60, 500])
def test_long_sums_do_not_shrink(tokens):
    """A unit that truncates where it adds 16 products to a sum loses at most 2^-24 of it per addition on the mean.  Sums in runs of
    1024 take 64 of them, 2^-18 of a logit, whatever the depth (16384 in one run: 2^-14); d loss = -shrink sum_{j != label} p_ij l_ij.
    The rest of the loss is rounded to nearest: its mean error over the tokens is below 2^-20."""
    vocab, dim = 2000, 16384
    h, w, y = draw(tokens, vocab, dim, 51, lift=4.0)
    h = (h.float() * 3).to(torch.bfloat16)                # other logits of up to ten or so
    loss, _, _ = run(h, w, y, 1.0, want_h=False, want_w=False)
    (want, _), _, _ = exact(h, w, y, 1.0)
    l = h.double() @ w.double().T
    p = torch.softmax(l, 1)
    p[torch.arange(tokens, device=DEV), y.long()] = 0.0
    error, bound = abs(float((loss.double() - want).mean())), 2.0 ** -18 * float((p * l.abs()).sum(1).mean()) + 2.0 ** -20
    assert error <= bound, (error, bound)


@pytest.mark.parametrize("tokens,piece", [(40, 0), (300, 0), (300, 130)])
@pytest.mark.parametrize("feature", [1.0, 2.0])
def test_labels_on_a_masked_row(tokens, piece, feature):
    """A row of the head that is masked with the type's lowest value: its logits are -3.4e38, or -inf in fp32.  It changes nothing for
    the other labels, and a token whose label it is has that loss and the gradient of a target without probability."""
    h, w, y = draw(tokens, 900, 64, 61)
    masked, low = 123, float(torch.finfo(torch.bfloat16).min)
    w[masked] = 0.0
    w[masked, 0] = low
    h[:, 0] = feature
    y[y == masked] = 5
    y[::3] = masked
    loss, gh, gw = run(h, w, y, 1.0, piece=piece)
    l = h.double() @ w.double().T
    at = torch.arange(tokens, device=DEV)
    want = (torch.logsumexp(l, 1) - l[at, y.long()]).float()
    on = y == masked
    assert torch.equal(torch.isinf(loss), torch.isinf(want)) and bool((loss[on] > 3e38).all())
    keep = torch.ones(900, dtype=torch.bool, device=DEV)
    keep[masked] = False
    # the rest: as if that row were not there
    y2 = y - (y > masked).int()
    y2[on] = -1
    close(loss[~on], tuple(t[~on] for t in exact(h, w[keep], y2, 1.0)[0]), "loss of the others")
    d = torch.softmax(l, 1)
    d[at, y.long()] -= 1.0
    for got, ref, size in ((gh, d @ w.double(), d.abs() @ w.double().abs()), (gw, d.T @ h.double(), d.abs().T @ h.double().abs())):
        assert bool(torch.isfinite(got).all())
        assert bool(((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 4 * 2.0 ** -8 * size).all())


@pytest.mark.parametrize("tokens", [40, 300])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_not_a_number_stays_with_its_token(tokens, value):
    """An entry of a labelled hidden state that is no number: that token's loss and gradient are none either, nor is dW, to which it
    belongs; the other tokens' losses and gradients are what they were."""
    h, w, y = draw(tokens, 700, 64, 62)
    clean = run(h, w, y, 1.0)
    h[7, 3] = value
    loss, gh, gw = run(h, w, y, 1.0)
    rest = torch.arange(tokens, device=DEV) != 7
    assert torch.equal(loss[rest], clean[0][rest]) and torch.equal(gh[rest], clean[1][rest])
    assert not math.isfinite(float(loss[7])) and bool(gh[7].isnan().all()) and bool(gw[:, 3].isnan().all())
    # an entry of the head: every token's
    h, w, y = draw(tokens, 700, 64, 63)
    w[650, 5] = value
    loss, gh, gw = run(h, w, y, 1.0)
    ref = torch.nn.functional.cross_entropy(h.double() @ w.double().T, y.long(), reduction="none")
    assert torch.equal(loss.isfinite(), ref.isfinite())
    assert bool(gh[:, 5].isnan().all())


def test_a_masked_row_of_infinities():
    """-inf as the logit of a row that is nobody's label: the losses are those without it."""
    h, w, y = draw(200, 500, 64, 64)
    h[:, 0] = h[:, 0].abs() + 0.125
    y[y == 77] = 5
    w[77] = 0.0
    w[77, 0] = -float("inf")
    loss, _, gw = run(h, w, y, 1.0, want_h=False)
    keep = torch.arange(500, device=DEV) != 77
    y2 = y - (y > 77).int()
    ref = exact(h, w[keep], y2, 1.0)
    close(loss, ref[0], "loss")
    close(gw[keep], ref[2], "dW")
    assert not gw[77].any()


def test_calls_from_several_threads():
    """Each thread on a stream of its own, with its own workspace: the results are those of calls one after the other."""
    import threading
    inputs = [draw(tokens, 700, 96, 70 + tokens) for tokens in (60, 300, 90, 500)]
    updates = [torch.randn((200, 96 + 8 * i), generator=torch.Generator(device=DEV).manual_seed(i), device=DEV) for i in range(4)]
    want = [(ops.linear_ce(*x), ops.orthogonalize([u])[0]) for x, u in zip(inputs, updates)]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                got = ops.linear_ce(*inputs[i]), ops.orthogonalize([updates[i]])[0]
                torch.cuda.current_stream().synchronize()
                if not (all(torch.equal(a, b) for a, b in zip(got[0], want[i][0])) and torch.equal(got[1], want[i][1])):
                    wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not wrong and not any(t.is_alive() for t in threads)
