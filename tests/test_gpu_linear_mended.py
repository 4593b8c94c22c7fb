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
