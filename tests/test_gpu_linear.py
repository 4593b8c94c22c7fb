"""A worker's layers on the GPU against plain implementations in 64 bits.

Tolerances, from the arithmetic (u = half a step of the 16-bit type, relative: bf16 2^-8, fp16 2^-11):
  sums               exact products; the tensor core truncates what it adds, at most 4e-9 of the terms' magnitudes per
                     term (measured for these kernels' products: 1e-9 to 2.8e-9), and the fp32 result, a bias and
                     sums of parts round: sum_k |a| |b| (4e-9 K + 2^-21) =: D(K)
  log probabilities  z is off by at most D(hidden), so lse by at most that; the softmax's own arithmetic (z - m rounded,
                     the exponent's product, exponentials to 2^-22, sums in parts) less than 1e-5 as for
                     gar_token_logprobs
  gradients          dz = a (d - p) is rounded to 16 bits and p off by its exponent's error: u |dz| + |a| p (D + 1e-5);
                     that through the products, their own D, and the result's rounding
  checkpoints        a code is off by half a step, and where the value next to the half step is off, by what that makes"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -25}                    # absolute, among the subnormals


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as entry
    entry.build()
    import paper_1905_04374_b200 as p
    return p


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).to(DTYPES[dtype])


def strided(x, pad, shift):
    """The same matrix as a view into a wider buffer: row stride cols + pad, first element shifted."""
    rows, cols = x.shape
    wide = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=x.dtype, device=x.device)
    view = wide[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def close(got, want, tol, what=""):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(inf, torch.isinf(got)) and torch.equal(got[inf], want[inf]), what
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine] - (tol if not torch.is_tensor(tol) else tol.expand_as(want)[fine])
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {float(off.max()):.3e} over the bound"


def short(k):
    """What a sum of k terms may be off by, relative to the terms' magnitudes."""
    return 4e-9 * k + 2.0 ** -21


# ---- log probabilities ------------------------------------------------------------------------
def head(rows, hidden, vocab, dtype, bias, seed=0):
    x = normal((rows, hidden), dtype, 11 * vocab + rows + seed)
    w = normal((vocab, hidden), dtype, 7 * hidden + 1 + seed, 2.0 / math.sqrt(hidden))
    b = normal((vocab,), dtype, 5 + seed) if bias else None
    t = torch.randint(-1, vocab, (rows,), generator=gen(vocab + seed), device=DEV)
    return x, w, b, t


def scores_64(x, w, b, t):
    """log probabilities, lse, all p, and D of each row's logits."""
    z = x.double() @ w.double().t()
    mag = x.double().abs() @ w.double().abs().t()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs().nan_to_num(0.0, 0.0, 0.0)
    bad = torch.isnan(z).any(1) | (z == math.inf).any(1)
    lse = torch.where(bad, math.nan, torch.logsumexp(z, 1))
    has = t >= 0
    inside = has & (t < z.shape[1])
    picked = z.gather(1, torch.where(inside, t, 0)[:, None])[:, 0] - lse
    picked = torch.where(lse == -math.inf, lse, picked)
    logprobs = torch.where(has, torch.where(inside, picked, math.nan), 0.0)
    return logprobs, lse, torch.exp(z - lse[:, None]), mag.nan_to_num(0.0, 0.0, 0.0).amax(1) * short(x.shape[1])


def check_scores(pkg, x, w, b, t, **kw):
    r = pkg.gar_linear_logprobs(x, w, t, bias=b, **kw)
    torch.cuda.synchronize()
    logprobs, lse, _, d = scores_64(x, w, b, t)
    tol = 2 * d + 1e-5 + 2.0 ** -22 * lse.abs().nan_to_num(0.0, 0.0, 0.0)
    close(r.lse, lse, tol, "lse")
    close(r.logprobs, logprobs, tol + 2.0 ** -22 * logprobs.abs().nan_to_num(0.0, 0.0, 0.0), "logprobs")
    return r


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,hidden,vocab,bias", [(1, 1, 1, False), (1, 64, 2, True), (3, 8, 10, False), (5, 63, 255, True), (128, 64, 256, False),
                                                    (129, 65, 257, True), (257, 128, 513, False), (300, 500, 1000, True), (513, 1000, 777, False),
                                                    (4, 2048, 40001, False), (1, 4096, 32, False), (8, 136, 5001, True), (9, 1000, 300, False),
                                                    (16, 264, 20000, True), (16, 3000, 70, True), (5, 8000, 100, False), (2000, 32, 5000, True), (700, 192, 20000, False)])
def test_scores(pkg, dtype, rows, hidden, vocab, bias):
    check_scores(pkg, *head(rows, hidden, vocab, dtype, bias))


@pytest.mark.parametrize("rows,vocab", [(40, 31 + 74 * k) for k in (31, 63, 95, 127, 159, 191, 223, 255)] + [(300, 37 * k + 1) for k in (63, 127, 191, 255)])
def test_scores_of_every_tile_width(pkg, rows, vocab):
    """Vocabularies that one round of tiles of 32, 64, .. 256 columns covers, forward and backward."""
    x, w, b, t = head(rows, 128, vocab, "bf16", True, 9)
    check_scores(pkg, x, w, b, t)
    a = -torch.rand(rows, generator=gen(1), device=DEV)
    check_head_gradient(pkg, x, w, b, t, a, 2, "f32")


def test_scores_without_targets(pkg):
    """lse alone; and the gradient from what gar_token_logprobs saved of the same logits, or without the lower part of lse."""
    for rows in (3, 300):
        x, w, b, t = head(rows, 64, 500, "bf16", True, 8)
        t = t.clamp_min(0)
        r = pkg.gar_linear_logprobs(x, w, bias=b)
        full = pkg.gar_linear_logprobs(x, w, t, bias=b)
        assert r.logprobs is None and torch.equal(r.lse, full.lse) and torch.equal(r.lse_lo, full.lse_lo)
        a = torch.ones(rows, device=DEV)
        check_head_gradient(pkg, x, w, b, t, a, 1, "f32", saved=r)
        check_head_gradient(pkg, x, w, b, t, a, 1, "f32", saved=r._replace(lse_lo=None))
        logits = (x.float() @ w.float().t() + b.float())
        check_head_gradient(pkg, x, w, b, t, a, 1, "f32", saved=pkg.gar_token_logprobs(logits, t))


def test_scores_in_runs_of_rows(pkg):
    """So many rows and columns that the rows are gone through in runs."""
    rows, hidden, vocab = 8400, 16, 131000
    x, w, b, t = head(rows, hidden, vocab, "bf16", True, 2)
    r = pkg.gar_linear_logprobs(x, w, t, bias=b)
    for r0 in range(0, rows, 1200):
        at = slice(r0, r0 + 1200)
        logprobs, lse, _, d = scores_64(x[at], w, b, t[at])
        close(r.lse[at], lse, 2 * d + 2e-5, "lse")
        close(r.logprobs[at], logprobs, 2 * d + 2e-5, "logprobs")


@pytest.mark.parametrize("pad,shift", [(0, 1), (8, 0), (3, 5), (8, 8)])
def test_scores_strides(pkg, pad, shift):
    x, w, b, t = head(70, 136, 300, "bf16", True)
    want = check_scores(pkg, x, w, b, t)
    got = check_scores(pkg, strided(x, pad, shift), strided(w, pad + 1, shift), torch.cat([b[:1], b])[1:], t)
    for p, q in zip(want, got):
        assert torch.equal(p, q)


def test_scores_hard_rows(pkg):
    """Masks, infinities and NaN: of a column, of a row, of everything."""
    rows, hidden, vocab = 40, 64, 700
    x, w, b, t = head(rows, hidden, vocab, "bf16", True)
    t[:4] = torch.tensor([-5, vocab, vocab + 7, 1 << 40], device=DEV)
    b[500:] = -math.inf
    b[100:120] = torch.finfo(torch.bfloat16).min
    t[5], t[6] = 600, 110                                    # masked targets
    x[7, 3], x[8, 3] = math.nan, math.inf                    # z NaN, or +-inf throughout
    r = pkg.gar_linear_logprobs(x, w, t, bias=b)
    logprobs, lse, _, d = scores_64(x, w, b, t)
    tol = 2 * d + 1e-5 + 2.0 ** -21 * logprobs.abs().nan_to_num(0.0, 0.0, 0.0)
    close(r.lse, lse, 2 * d + 2e-5, "lse")
    close(r.logprobs, logprobs, tol, "logprobs")
    # every column masked: by -inf, and by the lowest value, where lse needs its lower part
    b.fill_(-math.inf)
    r = pkg.gar_linear_logprobs(x[10:], w, t[10:], bias=b)
    assert bool((r.lse == -math.inf).all()) and bool((r.logprobs[t[10:] >= 0] == -math.inf).all()) and bool((r.lse_lo == 0).all())
    b.fill_(torch.finfo(torch.bfloat16).min)
    r = pkg.gar_linear_logprobs(x[10:], w, t[10:], bias=b)
    live = t[10:] >= 0
    # x w^T is lost next to the lowest value: all columns are equal
    close(r.logprobs[live], torch.full_like(r.logprobs[live], -math.log(vocab)), 1e-5, "lowest value")
    close(r.lse_lo, torch.full_like(r.lse_lo, math.log(vocab)), 1e-5, "lse_lo")


def check_head_gradient(pkg, x, w, b, t, a, workers, grads_dtype, weight_at=0, bias=False, dx=True, grads=None, workspace=None, stream=None, saved=None):
    dtype = {torch.bfloat16: "bf16", torch.float16: "f16"}[x.dtype]
    rows, hidden = x.shape
    vocab, u = w.shape[0], HALF[dtype]
    r = saved or pkg.gar_linear_logprobs(x, w, t, bias=b)
    bias_at = weight_at + vocab * hidden + 3 if bias else None
    if grads is None:
        grads = torch.full((workers, weight_at + vocab * hidden + (3 + vocab if bias else 0) + 5), 7.0, dtype=DTYPES[grads_dtype], device=DEV)
    got = pkg.gar_linear_logprobs_backward(x, w, r, t, a, bias=b, grads=grads, weight_offset=weight_at, bias_offset=bias_at, dx=dx, workspace=workspace,
                                           stream=stream)
    torch.cuda.synchronize()
    _, lse, p, d = scores_64(x, w, b, t)
    coef = torch.where(t >= 0, a.double(), 0.0)
    live = (coef != 0) & (lse != -math.inf)
    coef = torch.where(live, coef, 0.0)
    p = torch.where(live[:, None], p, 0.0)
    hot = torch.zeros_like(p).scatter_(1, t.clamp(0, vocab - 1)[:, None], live.double()[:, None])
    dz = coef[:, None] * (hot - p)
    # (an underflow of dz is 2^-25 of 2^-14 of the largest coefficient in fp16)
    off = u * dz.abs() + coef.abs()[:, None] * p * (2 * d[:, None] + 2e-5) + TINY[dtype] * 2.0 ** -14 * coef.abs().max()
    wa, xa = w.double().abs(), torch.where(live[:, None], x.double(), 0.0).abs()
    if got is not None:
        want = dz @ w.double()
        close(got, want, off @ wa + short(min(vocab, 32768)) * (dz.abs() @ wa) + u * want.abs() + TINY[dtype], "dx")
    tokens = rows // workers
    ug = HALF[grads_dtype]
    for k in range(workers):
        at = slice(k * tokens, (k + 1) * tokens)
        xs = torch.where(live[at, None], x[at].double(), 0.0)
        want = dz[at].t() @ xs
        tol = off[at].t() @ xa[at] + short(tokens) * (dz[at].abs().t() @ xa[at])
        mine = grads[k, weight_at:weight_at + vocab * hidden].view(vocab, hidden)
        close(mine, want, tol + ug * want.abs() + TINY[grads_dtype], f"weights of worker {k}")
        if bias:
            want = dz[at].sum(0)
            close(grads[k, bias_at:bias_at + vocab], want, off[at].sum(0) + short(tokens) * dz[at].abs().sum(0) + ug * want.abs() + TINY[grads_dtype], "bias")
            assert bool((grads[k, bias_at - 3:bias_at] == 7).all())
        assert bool((grads[k, :weight_at] == 7).all()) and bool((grads[k, -5:] == 7).all())
    return got, grads


@pytest.mark.parametrize("dtype,grads", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("workers,tokens,hidden,vocab,bias", [(1, 1, 1, 1, True), (1, 3, 8, 10, False), (2, 64, 64, 256, True), (3, 100, 65, 257, True),
                                                              (5, 33, 500, 100, False), (1, 700, 130, 999, True), (2, 300, 64, 20000, False),
                                                              (16, 5, 96, 600, True), (1, 2048, 256, 512, False)])
def test_head_gradient(pkg, dtype, grads, workers, tokens, hidden, vocab, bias):
    x, w, b, t = head(workers * tokens, hidden, vocab, dtype, bias, 3)
    a = -torch.rand(workers * tokens, generator=gen(1), device=DEV) / tokens
    a[tokens // 2] = 0.0
    check_head_gradient(pkg, x, w, b, t, a, workers, grads, weight_at=2, bias=bias)


@pytest.mark.parametrize("grads,tokens,hidden,shift", [("f32", 600, 65, 1), ("f32", 800, 64, 0), ("f32", 300, 64, 3), ("bf16", 2049, 64, 0),
                                                       ("bf16", 700, 66, 1), ("bf16", 64, 1030, 0)])
def test_head_gradient_results_that_start_anywhere(pkg, grads, tokens, hidden, shift):
    """Blocks whose rows lie on 16 bytes and anywhere, sums of one accumulator and of more."""
    x, w, b, t = head(2 * tokens, hidden, 400, "bf16", True, 6)
    a = -torch.rand(2 * tokens, generator=gen(7), device=DEV) / tokens
    check_head_gradient(pkg, x, w, b, t, a, 2, grads, weight_at=shift, bias=True)


def test_small_gradients_in_binary16(pkg):
    """Coefficients of 2^-20 and rows that differ by 2^12 among them: dz would underflow without its power of two."""
    x, w, b, t = head(200, 64, 3000, "f16", False, 5)
    a = torch.full((200,), 2.0 ** -20, device=DEV)
    a[::2] *= 2.0 ** -12
    # the results themselves are far below binary16's subnormals but for fp32 blocks
    check_head_gradient(pkg, x, w, b, t, a, 1, "f32", dx=False)
    check_head_gradient(pkg, x, w, b, t, a * 2.0 ** 60, 1, "f32", dx=False)


def test_head_gradient_in_pieces(pkg):
    """So many rows that a piece of the vocabulary is narrow, and a vocabulary of several of the widest."""
    for workers, tokens, hidden, vocab in ((2, 9000, 32, 5000), (1, 40, 64, 40000)):
        x, w, b, t = head(workers * tokens, hidden, vocab, "bf16", True, 4)
        a = torch.rand(workers * tokens, generator=gen(2), device=DEV) - 0.5
        check_head_gradient(pkg, x, w, b, t, a, workers, "f32", bias=True)


@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 5), (8, 8)])
def test_head_gradient_strides(pkg, pad, shift):
    x, w, b, t = head(120, 72, 300, "bf16", True, 5)
    a = -torch.rand(120, generator=gen(3), device=DEV)
    dx0, g0 = check_head_gradient(pkg, x, w, b, t, a, 3, "f32", bias=True)
    out = strided(torch.zeros_like(x), pad, shift)
    dx1, g1 = check_head_gradient(pkg, strided(x, pad, shift), strided(w, pad, shift), b, t, a, 3, "f32", bias=True, dx=out)
    assert dx1.data_ptr() == out.data_ptr() and torch.equal(dx0, dx1) and torch.equal(g0, g1)
    # rows behind the last column are the caller's
    if pad:
        assert bool(torch.isnan(out.as_strided((120, pad), (72 + pad, 1), out.storage_offset() + 72)[:-1]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_head_gradient_hard_rows(pkg, dtype):
    """Rows without a target hold NaN, a worker has a target outside the vocabulary, another a NaN, a third is masked."""
    rows, hidden, vocab, workers = 120, 64, 300, 4
    x, w, b, t = head(rows, hidden, vocab, dtype, True, 6)
    b[200:] = -math.inf
    t = t % 200
    a = -torch.rand(rows, generator=gen(4), device=DEV) - 0.1
    t[0], x[0], x[1] = -100, math.nan, math.inf
    a[1] = 0.0                                               # counts as little as a row without a target
    dx, grads = check_head_gradient(pkg, x, w, b, t, a, workers, "f32", bias=True)
    assert bool((dx[:2] == 0).all())
    t[40], x[70, 5] = vocab, math.nan
    r = pkg.gar_linear_logprobs(x, w, t, bias=b)
    bad = torch.empty_like(grads).fill_(7.0)
    dx2 = pkg.gar_linear_logprobs_backward(x, w, r, t, a, bias=b, grads=bad, bias_offset=vocab * hidden + 3)
    for k in (0, 3):
        assert torch.equal(bad[k], grads[k])                 # the others' bits are as before
    for k in (1, 2):
        assert bool(torch.isnan(bad[k, :vocab * hidden]).any())
    assert bool(torch.isnan(dx2[[40, 70]]).all())
    keep = [i for i in range(rows) if i not in (40, 70)]
    assert torch.equal(dx2[keep], dx[keep])
    # masked throughout: gradient 0 whatever comes in
    b.fill_(-math.inf)
    a[3], t[4] = math.inf, vocab + 1
    r = pkg.gar_linear_logprobs(x[2:70], w, t[2:70], bias=b)
    g = torch.full((1, vocab * hidden), 7.0, device=DEV)
    dx = pkg.gar_linear_logprobs_backward(x[2:70], w, r, t[2:70], a[2:70], bias=b, grads=g)
    assert bool((dx == 0).all()) and bool((g == 0).all())
    # all columns equal the lowest value: p = 1 / vocab each, by the lower part of lse
    if dtype == "bf16":
        b.fill_(torch.finfo(torch.bfloat16).min)
        r = pkg.gar_linear_logprobs(x[5:40], w, t[5:40], bias=b)
        dx = pkg.gar_linear_logprobs_backward(x[5:40], w, r, t[5:40], torch.ones(35, device=DEV), bias=b)
        want = w.double()[t[5:40]] - w.double().mean(0)
        close(dx, want, (w.double().abs()[t[5:40]] + w.double().abs().mean(0)) * (2 * HALF[dtype] + 1e-4), "lowest value")


def test_head_gradient_against_differences(pkg):
    """d sum_i a_i logprob_i along random directions of x and W, by central differences in 64 bits of the forward formula."""
    x, w, b, t = head(90, 48, 130, "bf16", True, 7)
    t = t.clamp_min(0)
    a = torch.randn(90, generator=gen(5), device=DEV)
    r = pkg.gar_linear_logprobs(x, w, t, bias=b)
    grads = torch.empty(1, 130 * 48, device=DEV)
    dx = pkg.gar_linear_logprobs_backward(x, w, r, t, a, bias=b, grads=grads)
    vx, vw = (torch.randn(s.shape, generator=gen(6), device=DEV, dtype=torch.float64) for s in (x, w))

    def value(step):
        z = (x.double() + step * vx) @ (w.double() + step * vw).t() + b.double()
        return float((a.double() * torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]).sum())

    h = 1e-5
    want = (value(h) - value(-h)) / (2 * h)
    got = float((dx.double() * vx).sum() + (grads[0].double().view(130, 48) * vw).sum())
    # 90 x 48 and 130 x 48 products of random signs, each off by 2^-8 or so of itself; h^2 and 1e-16 / h are far below
    scale = math.sqrt(float((dx.double() * vx).square().sum() + (grads[0].double().view(130, 48) * vw).square().sum()))
    assert abs(got - want) <= 4 * 2.0 ** -7 * scale


# ---- the gated block ------------------------------------------------------------------------
def act_64(name, x):
    if name == "relu":
        return torch.relu(x), (x > 0).double()
    if name == "silu":
        g = torch.sigmoid(x)
        return x * g, g * (1 + x * (1 - g))
    if name == "identity":
        return x, torch.ones_like(x)
    cdf = 0.5 * torch.special.erfc(-x / math.sqrt(2))
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def block(rows, hidden, inner, dtype, bias, seed=0):
    x = normal((rows, hidden), dtype, 3 * rows + inner + seed)
    wg, wu = (normal((inner, hidden), dtype, 17 * hidden + k + seed, 1.5 / math.sqrt(hidden)) for k in (0, 1))
    bg, bu = (normal((inner,), dtype, 29 + k + seed) if bias else None for k in (0, 1))
    return x, wg, wu, bg, bu


def projections_64(x, w, b):
    z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    return z, mag * short(x.shape[1])


def check_codes(ck, want, off, u):
    """Codes and scales of a checkpoint against the values it stands for, each known to `off`."""
    rows, cols = want.shape
    pad = -cols % ck.group
    v = torch.nn.functional.pad(want, (0, pad)).unflatten(1, (-1, ck.group))
    o = torch.nn.functional.pad(off, (0, pad)).unflatten(1, (-1, ck.group))
    top, slack = v.abs().amax(2), o.amax(2)
    close(ck.scales, top / 127, slack / 127 + 2.0 ** -23 * top, "scales")
    q = torch.nn.functional.pad(ck.q[:, :cols].double(), (0, pad)).unflatten(1, (-1, ck.group))
    step = (top / 127).clamp_min(1e-300)[:, :, None]
    assert float(((q - v / step).abs() - 0.5 - (2 * slack[:, :, None] / step) - 1e-4).max()) <= 0
    restored = q * ck.scales.double()[:, :, None]
    return restored.flatten(1)[:, :cols]


def check_gated(pkg, act, x, wg, wu, bg, bu, **kw):
    dtype = {torch.bfloat16: "bf16", torch.float16: "f16"}[x.dtype]
    r = pkg.gar_gated_linear_forward(act, x, wg, wu, bg, bu, **kw)
    torch.cuda.synchronize()
    g, og = projections_64(x, wg, bg)
    u, ou = projections_64(x, wu, bu)
    value, slope = act_64(act, g)
    want = value * u
    # |act'| <= 1.13; the activation's own arithmetic is 2e-6 of |g|
    tol = 1.13 * og * u.abs() + value.abs() * ou + og * ou * 1.13 + 4e-6 * g.abs() * u.abs()
    close(r.y, want, tol * 1.01 + HALF[dtype] * want.abs() + TINY[dtype], "y")
    if r.x is not None:
        check_codes(r.x, g, og, HALF[dtype])
        check_codes(r.up, u, ou, HALF[dtype])
    if r.out is not None:
        again = pkg.gar_checkpoint_pack(r.y, r.out.group)
        cols = wg.shape[0]
        assert torch.equal(again.q[:, :cols], r.out.q[:, :cols]) and torch.equal(again.scales, r.out.scales)
    return r


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act,rows,hidden,inner,bias,group", [("silu", 1, 1, 1, True, 32), ("gelu", 3, 8, 10, False, 64), ("relu", 128, 64, 128, False, 128),
                                                              ("silu", 129, 65, 129, True, 128), ("identity", 40, 200, 31, True, 32),
                                                              ("gelu", 300, 500, 800, True, 32), ("silu", 513, 130, 2050, False, 64),
                                                              ("relu", 1, 2048, 257, True, 64), ("gelu", 1000, 96, 1000, False, 128)])
def test_gated(pkg, dtype, act, rows, hidden, inner, bias, group):
    parts = block(rows, hidden, inner, dtype, bias)
    r = check_gated(pkg, act, *parts, group=group, save_output=True)
    bare = check_gated(pkg, act, *parts, save_input=False)   # (a few rows go through a kernel of their own)
    assert (rows <= 16 or torch.equal(bare.y, r.y)) and bare.x is None and bare.up is None and bare.out is None


@pytest.mark.parametrize("act,rows,hidden,inner,bias", [("silu", 1, 4096, 1000, False), ("gelu", 8, 1000, 333, True), ("relu", 9, 264, 64, True),
                                                        ("identity", 16, 3000, 9, False), ("silu", 16, 520, 5000, True), ("gelu", 17, 520, 500, True)])
def test_gated_few_rows(pkg, act, rows, hidden, inner, bias):
    for dtype in ("bf16", "f16"):
        x, wg, wu, bg, bu = block(rows, hidden, inner, dtype, bias)
        want = check_gated(pkg, act, x, wg, wu, bg, bu, save_input=False).y
        y = strided(torch.zeros_like(want), 3, 1)
        got = check_gated(pkg, act, strided(x, 5, 3), strided(wg, 8, 0), wu, bg, bu, save_input=False, y=y).y
        assert torch.equal(got, want)


@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 5), (8, 8)])
def test_gated_strides(pkg, pad, shift):
    x, wg, wu, bg, bu = block(70, 72, 200, "bf16", True)
    want = check_gated(pkg, "silu", x, wg, wu, bg, bu)
    y = strided(torch.zeros(70, 200, dtype=torch.bfloat16, device=DEV), pad, shift)
    got = check_gated(pkg, "silu", strided(x, pad, shift), strided(wg, pad, shift), strided(wu, pad + 2, shift), bg, bu, y=y)
    assert got.y.data_ptr() == y.data_ptr() and torch.equal(got.y, want.y) and torch.equal(got.x.scales, want.x.scales)
    if pad:
        assert bool(torch.isnan(y.as_strided((69, pad), (200 + pad, 1), y.storage_offset() + 200)).all())


def test_gated_non_finite(pkg):
    """A NaN or an infinity in a row stays in that row: its groups are restored as NaN, the others as before."""
    x, wg, wu, bg, bu = block(40, 64, 200, "bf16", True)
    want = pkg.gar_gated_linear_forward("silu", x, wg, wu, bg, bu, group=64)
    bg[130] = math.inf
    x[7, 3] = math.nan
    got = pkg.gar_gated_linear_forward("silu", x, wg, wu, bg, bu, group=64)
    rows = [i for i in range(40) if i != 7]
    cols = [i for i in range(200) if i != 130]
    assert torch.equal(got.y[rows][:, cols], want.y[rows][:, cols]) and bool(torch.isnan(got.y[7]).all())
    assert bool(torch.isnan(got.x.scales[:, 2]).all()) and bool(torch.isnan(got.x.scales[7]).all())
    assert torch.equal(got.x.scales[rows][:, [0, 1, 3]], want.x.scales[rows][:, [0, 1, 3]])
    assert torch.equal(got.up.scales[rows], want.up.scales[rows])
    assert bool(torch.isnan(pkg.gar_checkpoint_unpack(got.x)[:, 128:192]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act,rows,hidden,inner,group", [("silu", 1, 1, 1, 32), ("gelu", 130, 72, 100, 64), ("relu", 300, 257, 513, 128),
                                                         ("silu", 64, 64, 4000, 32), ("gelu", 1000, 500, 128, 64)])
def test_gated_backward(pkg, dtype, act, rows, hidden, inner, group):
    x, wg, wu, bg, bu = block(rows, hidden, inner, dtype, True, 1)
    u = HALF[dtype]
    f = pkg.gar_gated_linear_forward(act, x, wg, wu, bg, bu, group=group)
    dy = normal((rows, inner), dtype, 8, 0.1)
    r = pkg.gar_gated_linear_backward(act, dy, f.x, f.up, wg, wu)
    torch.cuda.synchronize()
    want = pkg.gar_activation_backward(act, dy, f.x, f.up)
    assert torch.equal(r.dgate, want.dx) and torch.equal(r.dup, want.dup)
    dg, du, g, v = r.dgate.double(), r.dup.double(), wg.double(), wu.double()
    dx = dg @ g + du @ v
    close(r.dx, dx, short(2 * inner) * (dg.abs() @ g.abs() + du.abs() @ v.abs()) + u * dx.abs() + TINY[dtype], "dx")
    # in place, into the caller's tensors, without dx
    own = strided(torch.zeros(rows, hidden, dtype=dy.dtype, device=DEV), 3, 1)
    buf = dy.clone()
    s = pkg.gar_gated_linear_backward(act, buf, f.x, f.up, wg, wu, dx=own, dgate=buf)
    assert s.dgate.data_ptr() == buf.data_ptr() and torch.equal(buf, r.dgate) and torch.equal(own, r.dx)
    assert pkg.gar_gated_linear_backward(act, dy, f.x, f.up, wg, wu, dx=False).dx is None


def test_gated_backward_against_differences(pkg):
    """Along random directions of x, Wg and Wu, by central differences in 64 bits of the forward formula.  A restored value is off by
    half a 254th of its group's largest magnitude (3 standard deviations) at most, 0.7 % of a standard deviation
    in the mean: dgate and dup by 1.2 % of their own in the mean with both inputs and their rounding, independently of
    one another, and x' by 0.7 %; six standard deviations of what that makes of the sum."""
    x, wg, wu, bg, bu = block(60, 40, 96, "bf16", True, 2)
    dy = normal((60, 96), "bf16", 9)
    ck = pkg.gar_checkpoint_pack(x, 32)
    f = pkg.gar_gated_linear_forward("silu", x, wg, wu, bg, bu, group=32)
    r = pkg.gar_gated_linear_backward("silu", dy, f.x, f.up, wg, wu)
    grads = torch.empty(2, 1, 96 * 40, device=DEV)
    pkg.gar_linear_weight_grad(r.dgate.view(1, 60, 96), ck, grads[0])
    pkg.gar_linear_weight_grad(r.dup.view(1, 60, 96), ck, grads[1])
    v = [torch.randn(s.shape, generator=gen(12 + i), device=DEV, dtype=torch.float64) for i, s in enumerate((x, wg, wu))]

    def value(step):
        xs, gs, us = (p.double() + step * q for p, q in zip((x, wg, wu), v))
        return float((dy.double() * act_64("silu", xs @ gs.t() + bg.double())[0] * (xs @ us.t() + bu.double())).sum())

    h = 1e-5
    want = (value(h) - value(-h)) / (2 * h)
    got = sum(float((p.double().view(q.shape) * q).sum()) for p, q in ((r.dx, v[0]), (grads[0], v[1]), (grads[1], v[2])))
    tol = 0.0
    for d, w, q in ((r.dgate.double(), wg.double(), v[1]), (r.dup.double(), wu.double(), v[2])):
        along = v[0] @ w.t() + x.double() @ q.t()            # what a change of d makes of the sum
        tol += 6 * (0.012 * float(d.square().mean().sqrt() * along.norm()) + 0.007 * float((d @ q).norm()))
    assert abs(got - want) <= tol


# ---- dropout ----------------------------------------------------------------------------------
def philox(block, offset, seed):
    """Philox 4x32-10 in Python's whole numbers, from the paper's definition."""
    c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, cols, seed, offset, p):
    limit, per = round(p * 65536), -(-cols // 8)
    out = np.zeros((rows, per * 8), dtype=bool)
    for r in range(rows):
        for b in range(per):
            words = philox(r * per + b, offset, seed)
            out[r, 8 * b:8 * b + 8] = [((words[j // 2] >> 16 * (j % 2)) & 0xFFFF) >= limit for j in range(8)]
    return torch.from_numpy(out[:, :cols].copy()).to(DEV)


def test_generator_known_values():
    """The published vectors of Philox 4x32-10 (all zeros; all ones)."""
    assert philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox(2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,p,residual", [(1, 1, 0.5, False), (7, 8, 0.1, True), (33, 65, 0.3, True), (5, 1001, 0.25, False), (64, 128, 0.9, True)])
def test_dropout(pkg, dtype, rows, cols, p, residual):
    x, r = normal((rows, cols), dtype, 1), normal((rows, cols), dtype, 2) if residual else None
    seed, offset = 0xDEADBEEF12345678, 2 ** 40 + 3
    keep = kept(rows, cols, seed, offset, p)
    x[~keep] = math.nan                                      # a dropped element counts as 0 whatever it holds
    y = pkg.gar_dropout(x, p, seed, offset, residual=r)
    scale = 65536 / (65536 - round(p * 65536))
    want = torch.where(keep, x.double() * scale, 0.0)
    mag = want.abs()
    if residual:
        want, mag = want + r.double(), mag + r.double().abs()
    close(y, want, 2.0 ** -22 * mag + HALF[dtype] * want.abs() + TINY[dtype])
    # any strides, in place, a counter on the device
    for pad, shift in ((0, 1), (1, 0), (8, 8)):
        got = pkg.gar_dropout(strided(x, pad, shift), p, seed, offset, residual=None if r is None else strided(r, pad, shift))
        assert torch.equal(got, y)
    counter = torch.tensor([5], device=DEV)
    buf = x.clone()
    assert pkg.gar_dropout(buf, p, seed, offset - 5, residual=r, y=buf, counter=counter) is buf and torch.equal(buf, y)
    if residual:
        buf = r.clone()
        assert torch.equal(pkg.gar_dropout(x, p, seed, offset, residual=buf, y=buf), y)


def test_dropout_edges(pkg):
    x = normal((40, 200), "bf16", 3)
    assert torch.equal(pkg.gar_dropout(x, 0.0, 1), x)
    assert bool((pkg.gar_dropout(x * math.nan, 1.0, 1) == 0).all())
    assert pkg.gar_dropout(x[:0], 0.5, 1).shape == (0, 200)
    a, b, c = pkg.gar_dropout(x, 0.5, 1, 0), pkg.gar_dropout(x, 0.5, 1, 1), pkg.gar_dropout(x, 0.5, 2, 0)
    assert not torch.equal(a, b) and not torch.equal(a, c) and not torch.equal(b, c)
    assert torch.equal(pkg.gar_dropout(x, 0.5, 2 ** 64 - 1, 2 ** 64 - 1), pkg.gar_dropout(x, 0.5, 2 ** 64 - 1, 2 ** 64 - 2, counter=torch.ones(1, dtype=torch.int64, device=DEV)))


def test_dropout_probability(pkg):
    """2^24 elements, p = 0.1: the dropped share is within five standard deviations, in every column's half too."""
    x = torch.ones(4096, 4096, device=DEV)
    dropped = pkg.gar_dropout(x, 0.1, 77) == 0
    p = round(0.1 * 65536) / 65536
    assert abs(float(dropped.double().mean()) - p) <= 5 * math.sqrt(p * (1 - p) / 2 ** 24)
    per = dropped.view(4096, 512, 8).double().mean((0, 1))
    assert float((per - p).abs().max()) <= 5 * math.sqrt(p * (1 - p) / 2 ** 21)
    both = (dropped[:, 1:] & dropped[:, :-1]).double().mean()
    assert abs(float(both) - p * p) <= 6 * math.sqrt(p * p / 2 ** 24)
