"""Faults of a worker's layers that were mended, one test or more for each."""
import math

import pytest
import torch

from tests.test_gpu_linear import DEV, DTYPES, HALF, TINY, check_head_gradient, close, gen, head, normal, scores_64, short

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as entry
    entry.build()
    import paper_1905_04374_b200 as p
    return p


# ---- binary16 gradients of workers whose coefficients differ ----------------------------------------
@pytest.mark.parametrize("workers,tokens,hidden,vocab,grads", [(2, 40, 64, 300, "f32"), (3, 33, 65, 257, "f16"), (2, 20, 64, 40000, "f32"), (3, 900, 64, 300, "f32"),
                                                               (2, 2100, 72, 500, "f16"), (2, 9000, 32, 5000, "f32"), (2, 1, 8, 10, "f32")])
def test_a_large_coefficient_stays_with_its_worker(pkg, workers, tokens, hidden, vocab, grads):
    """One worker's coefficients 2^40 (and 2^100) times the others': the others' bits are as without, and its own are the same times that
    power of two."""
    x, w, b, t = head(workers * tokens, hidden, vocab, "f16", True, 21)
    t = t.clamp_min(0)
    a = -(torch.rand(workers * tokens, generator=gen(8), device=DEV) + 0.5) / tokens
    bias_at = vocab * hidden + 3
    want_dx, want = check_head_gradient(pkg, x, w, b, t, a, workers, grads, bias=True)
    saved = pkg.gar_linear_logprobs(x, w, t, bias=b)
    at = slice((workers - 1) * tokens, workers * tokens)
    for power in (2.0 ** 40, 2.0 ** 100):
        big = a.clone()
        big[at] *= power
        got = torch.full_like(want, 7.0)
        dx = pkg.gar_linear_logprobs_backward(x, w, saved, t, big, bias=b, grads=got, bias_offset=bias_at)
        assert torch.equal(got[:-1], want[:-1]) and torch.equal(dx[:at.start], want_dx[:at.start])
        if grads == "f32":
            own = [c for c in range(want.shape[1]) if c < vocab * hidden or bias_at <= c < bias_at + vocab]
            assert torch.equal(got[-1, own], want[-1, own] * power)


@pytest.mark.parametrize("rows,hidden,vocab", [(40, 64, 300), (33, 65, 257), (20, 64, 40000), (9000, 32, 5000)])
def test_a_large_coefficient_stays_with_its_row(pkg, rows, hidden, vocab):
    """Without weight gradients nothing adds rows up: the gradient at a row's hidden state goes by its own coefficient alone."""
    x, w, b, t = head(rows, hidden, vocab, "f16", True, 24)
    t = t.clamp_min(0)
    a = -(torch.rand(rows, generator=gen(8), device=DEV) + 0.5)
    saved = pkg.gar_linear_logprobs(x, w, t, bias=b)
    want = pkg.gar_linear_logprobs_backward(x, w, saved, t, a, bias=b)
    check_head_gradient(pkg, x, w, b, t, a, 1, "f32", saved=saved)
    some = torch.arange(rows, device=DEV) % 3 == 0
    for power in (2.0 ** 40, 2.0 ** -20, 2.0 ** 6):
        dx = pkg.gar_linear_logprobs_backward(x, w, saved, t, torch.where(some, a * power, a), bias=b)
        assert torch.equal(dx[~some], want[~some])
    # a power of two of a row's coefficient is one of its gradient, but for what binary16 rounds off its subnormals
    off = 2.0 ** -25 * 64 * (want[some].double().abs() < 2.0 ** -14)
    close(dx[some], want[some].double() * 64, off, "scaled rows")


# ---- so many columns that a group of row tiles times them passes 32 bits ------------------------------
def test_scores_of_two_to_the_thirty_columns(pkg):
    """17 rows with one step of the contraction, 2^22 column tiles and more.  Logits 0 but for some columns."""
    rows, vocab = 17, (1 << 30) + 300
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    w = torch.zeros(vocab, 8, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 255, 256, (1 << 29) + 77, (1 << 30) - 1, 1 << 30, vocab - 2, vocab - 1], device=DEV)
    w[at, 0] = -torch.arange(1, 9, device=DEV).bfloat16()
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = torch.linspace(0.25, 1.25, rows, device=DEV).bfloat16()
    t = torch.cat([at, at[:4] + 9, at[:5]])
    r = pkg.gar_linear_logprobs(x, w, t)
    z = -x[:, :1].double() * torch.arange(1, 9, device=DEV)
    lse = torch.log((vocab - 8) + torch.exp(z).sum(1))
    picked = torch.cat([z.diagonal(), torch.zeros(4, dtype=torch.float64, device=DEV), z[12:, :5].diagonal()])
    # whole numbers of columns but for eight: the sums are exact to a few roundings
    close(r.lse, lse, 1e-5, "lse")
    close(r.logprobs, picked - lse, 1e-5, "logprobs")


# ---- rows masked throughout ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_masked_row_counts_for_nothing(pkg, dtype):
    """A row whose logits are all -inf (an infinity in x before a column of negative weights) has gradient 0: neither its coefficient nor
    what it holds reaches the other rows of its worker."""
    rows, hidden, vocab = 50, 64, 256
    x, w, _, t = head(rows, hidden, vocab, dtype, False, 22)
    t = t.clamp_min(0)
    w[:, 5] = -w[:, 5].abs() - 0.25
    a = -torch.rand(rows, generator=gen(9), device=DEV) - 0.5
    a[7] = 0.0
    want_dx, want = check_head_gradient(pkg, x, w, None, t, a, 1, "f32")
    x[7, 5], a[7] = math.inf, 2.0 ** 60
    saved = pkg.gar_linear_logprobs(x, w, t)
    assert float(saved.lse[7]) == -math.inf and float(saved.logprobs[7]) == -math.inf
    got = torch.empty_like(want).fill_(7.0)
    dx = pkg.gar_linear_logprobs_backward(x, w, saved, t, a, grads=got)
    assert torch.equal(got, want) and torch.equal(dx, want_dx)
    t[7] = vocab + 3                                         # not even a target outside the vocabulary
    dx = pkg.gar_linear_logprobs_backward(x, w, saved, t, a, grads=got)
    assert torch.equal(got, want) and torch.equal(dx, want_dx)


# ---- infinities next to columns that do not exist ----------------------------------------------------
@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("vocab", [1, 31, 200, 256, 999])
def test_a_row_of_minus_infinity_at_every_width(pkg, rows, vocab):
    """All of a row's logits are -inf: so are lse and log probability, whether or not the last tile of columns is full."""
    x, w, b, t = head(rows, 72, vocab, "bf16", True, 23)
    t = t.clamp_min(0)
    w[:, 5] = -w[:, 5].abs() - 0.25
    x[1, 5] = math.inf
    r = pkg.gar_linear_logprobs(x, w, t, bias=b)
    logprobs, lse, _, d = scores_64(x, w, b, t)
    assert float(lse[1]) == -math.inf and float(logprobs[1]) == -math.inf
    close(r.lse, lse, 2 * d + 2e-5, "lse")
    close(r.logprobs, logprobs, 2 * d + 2e-5, "logprobs")


# ---- sums of any operands --------------------------------------------------------------------------
def chunk_of(k):
    """Terms that go into one accumulator."""
    return k if k <= 640 else 512


def sums_off(k, rows):
    """Of the terms' magnitudes M, at most.  A product is cut to a multiple of 2^-25 (mma.sync, up to 16 rows: 2^-24) of the largest magnitude
    among the accumulator and the 16 products of its instruction, which is below M; so is the accumulator, and their sum to 24 bits, 2^-23 of M
    at most.  That is (17 unit + 2^-23) M for 16 terms.  The chunks' sums are added with half a unit of 24 bits each."""
    unit = 2.0 ** -24 if rows <= 16 else 2.0 ** -25
    return chunk_of(k) * (17 / 16 * unit + 2.0 ** -27) + 2.0 ** -24 * (-(-k // chunk_of(k)) + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_an_addition_keeps(pkg, dtype):
    """The unit of the bound above: terms of 2^-25 (2^-24) next to 1 are added whole, in the same instruction and behind it."""
    for rows, unit in ((4, 24), (40, 25)):
        for first in (1, 16):
            n = 2 ** (unit - 23)                             # together one unit of fp32's last place next to 1
            w, x = torch.zeros(1, 64, dtype=DTYPES[dtype], device=DEV), torch.zeros(rows, 64, dtype=DTYPES[dtype], device=DEV)
            w[:, 0], x[:, 0] = 1.0, 1.0
            w[:, first:first + n], x[:, first:first + n] = 2.0 ** -13, 2.0 ** (13 - unit)
            assert bool((pkg.gar_linear_logprobs(x, w).lse == 1 + 2.0 ** -23).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [4, 12, 40, 600])
@pytest.mark.parametrize("hidden", [4096, 6144])
def test_logits_that_are_exact(pkg, dtype, rows, hidden):
    """Hidden states with one element other than 0: the logits are single products, which fp32 holds.  lse and log probabilities are
    off by the softmax's own arithmetic and their rounding only (2^-22 of lse, 1e-5)."""
    vocab = 600
    w = normal((vocab, hidden), dtype, 31, 1.0)
    x = torch.zeros(rows, hidden, dtype=DTYPES[dtype], device=DEV)
    at = torch.randint(0, hidden, (rows,), generator=gen(32), device=DEV)
    x[torch.arange(rows, device=DEV), at] = 256.0
    t = torch.randint(0, vocab, (rows,), generator=gen(33), device=DEV)
    r = pkg.gar_linear_logprobs(x, w, t)
    logprobs, lse, _, _ = scores_64(x, w, None, t)
    # z up to some 800: of it 4e-6, as a factor for what other sums lose would make, is 3e-3
    assert float(lse.abs().min()) > 500
    close(r.lse, lse, 1e-5 + 2.0 ** -22 * lse.abs(), "lse")
    close(r.logprobs, logprobs, 1e-5 + 2.0 ** -22 * (lse.abs() + logprobs.abs()), "logprobs")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,hidden,vocab", [(4, 4096, 500), (4, 6200, 500), (16, 3000, 70), (40, 520, 300), (40, 640, 300), (40, 641, 300), (40, 768, 300), (40, 4096, 500), (40, 16384, 500), (300, 4096, 10),
                                               (2000, 1500, 5000), (600, 16384, 1200)])
@pytest.mark.parametrize("signs", ["one", "random"])
def test_logits_of_long_sums(pkg, dtype, rows, hidden, vocab, signs):
    """Terms of one sign, where the tensor core loses most, and of random signs."""
    g = gen(hidden + rows)
    x, w = torch.randn(rows, hidden, generator=g, device=DEV), torch.randn(vocab, hidden, generator=g, device=DEV)
    if signs == "one":
        x, w = x.abs() + 0.5, (w.abs() + 0.5) * (20.0 / hidden)
    else:
        w *= 3.0 / math.sqrt(hidden)
    x, w = x.to(DTYPES[dtype]), w.to(DTYPES[dtype])
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    r = pkg.gar_linear_logprobs(x, w, t)
    z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    off = mag * sums_off(hidden, rows)
    # lse moves by the mean of the logits' errors under p, a log probability by its own logit's besides
    mean, picked = (p * off).sum(1), off.gather(1, t[:, None])[:, 0]
    logprobs = z.gather(1, t[:, None])[:, 0] - lse
    close(r.lse, lse, 1.01 * mean + 1e-5 + 2.0 ** -22 * lse.abs(), "lse")
    close(r.logprobs, logprobs, 1.01 * (mean + picked) + 1e-5 + 2.0 ** -22 * (lse.abs() + logprobs.abs()), "logprobs")
    if signs == "random" and vocab >= 300:
        # The rows' mean, which leaves the loss of the sums alone: 1e-9 per term of a chunk's own sum, of the logits, whose mean
        # under p is below lse; and as much again.
        assert float(((r.lse.double() + r.lse_lo.double()) / lse - 1).mean().abs()) <= 2e-9 * chunk_of(hidden)


# ---- gradients of few rows ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,grads", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("workers,tokens,hidden,vocab", [(1, 1, 1, 1), (8, 2, 2354, 10), (1, 1, 64, 300), (3, 5, 65, 257), (16, 8, 136, 1000), (1, 128, 700, 50),
                                                         (2, 20, 64, 40000), (1, 64, 96, 9), (1, 129, 64, 300)])
def test_gradients_of_few_rows(pkg, dtype, grads, workers, tokens, hidden, vocab):
    """Up to 128 rows a coefficient's rounding to 16 bits decides a gradient, and does not average out: dz comes in two parts, off by
    u^2 of itself (binary16: and by what lies below 2^-25 of 2^-14 of its worker's largest coefficient) instead of u."""
    rows = workers * tokens
    x, w, b, t = head(rows, hidden, vocab, dtype, True, 25)
    a = -(torch.rand(rows, generator=gen(10), device=DEV) + 0.5) / tokens
    if rows > 3:
        a[2], t[3] = 0.0, -1
    saved = pkg.gar_linear_logprobs(x, w, t, bias=b)
    block = torch.full((workers, vocab * hidden + vocab), 7.0, dtype=DTYPES[grads], device=DEV)
    dx = pkg.gar_linear_logprobs_backward(x, w, saved, t, a, bias=b, grads=block, bias_offset=vocab * hidden)
    alone = pkg.gar_linear_logprobs_backward(x, w, saved, t, a, bias=b)
    _, _, p, d = scores_64(x, w, b, t)
    coef = torch.where(t >= 0, a.double(), 0.0)
    hot = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], (t >= 0).double()[:, None])
    dz = coef[:, None] * (hot - p)
    u = HALF[dtype]
    off = (u * u if rows <= 128 else u) * dz.abs() + coef.abs()[:, None] * p * (2 * d[:, None] + 2e-5) + TINY[dtype] * 2.0 ** -14 * coef.abs().max()
    wa, xa = w.double().abs(), x.double().abs()
    want = dz @ w.double()
    tol = off @ wa + 2 * short(vocab) * (dz.abs() @ wa) + u * want.abs() + TINY[dtype]
    close(dx, want, tol, "dx")
    close(alone, want, tol, "dx alone")
    for k in range(workers):
        at = slice(k * tokens, (k + 1) * tokens)
        want = dz[at].t() @ x[at].double()
        tol = off[at].t() @ xa[at] + 2 * short(tokens) * (dz[at].abs().t() @ xa[at]) + HALF[grads] * want.abs() + TINY[grads]
        close(block[k, :vocab * hidden].view(vocab, hidden), want, tol, "weights")
        want = dz[at].sum(0)
        close(block[k, vocab * hidden:], want, off[at].sum(0) + 2 * short(tokens) * dz[at].abs().sum(0) + HALF[grads] * want.abs() + TINY[grads], "bias")
