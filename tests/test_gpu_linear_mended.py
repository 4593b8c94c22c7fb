"""Faults of a worker's layers that were mended, one test or more for each."""
import math

import pytest
import torch

from tests.test_gpu_linear import DEV, DTYPES, check_head_gradient, close, gen, head, normal, scores_64

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
