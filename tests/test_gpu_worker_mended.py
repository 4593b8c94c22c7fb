"""Faults of the worker-side operators that were mended, one test or more for each, against plain forms in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as entry
    entry.build()
    import paper_1905_04374_b200 as p
    return p


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).to(dtype)


# ---- rows that share memory ---------------------------------------------------------------------
def test_rows_that_share_memory_are_refused(pkg):
    """An expanded tensor has unit column stride and row stride 0, which the library would take for "the number of
    columns".  Every call is refused before anything is launched, for inputs and for outputs."""
    rows, cols = 4, 64
    x = normal((rows, cols), torch.bfloat16, 1)
    one = x[:1].expand(rows, cols)                           # stride (0, 1)
    near = x.view(-1).as_strided((rows, cols), (8, 1))       # rows that overlap
    t = torch.zeros(rows, dtype=torch.int64, device=DEV)
    r = pkg.gar_token_logprobs(x, t)
    ones = torch.ones(rows, device=DEV)
    f = pkg.gar_activation_forward("silu", x, x.clone())
    ck = pkg.gar_checkpoint_pack(x)
    dy = x.view(2, 2, cols)
    for bad in (one, near):
        calls = [lambda: pkg.gar_token_logprobs(bad, t),
                 lambda: pkg.gar_token_logprobs_backward(bad, r, t, ones),
                 lambda: pkg.gar_token_logprobs_backward(x, r, t, ones, dlogits=bad),
                 lambda: pkg.gar_checkpoint_pack(bad),
                 lambda: pkg.gar_checkpoint_unpack(ck, bad),
                 lambda: pkg.gar_activation_forward("silu", bad),
                 lambda: pkg.gar_activation_forward("silu", x, bad),
                 lambda: pkg.gar_activation_forward("silu", x, y=bad),
                 lambda: pkg.gar_activation_backward("silu", bad, f.x),
                 lambda: pkg.gar_activation_backward("silu", x, f.x, dx=bad),
                 lambda: pkg.gar_activation_backward("silu", x, f.x, f.up, dup=bad),
                 lambda: pkg.gar_activation_backward("silu", x, f.x._replace(q=f.x.q[:1].expand(rows, cols))),
                 lambda: pkg.gar_linear_weight_grad(bad.as_strided((2, 2, cols), (2 * bad.stride(0), bad.stride(0), 1)), ck)]
        for i, call in enumerate(calls):
            with pytest.raises(ValueError, match="share memory"):
                call()
                pytest.fail(f"call {i} was not refused")
    shared = torch.empty(1, cols * cols, device=DEV).expand(2, cols * cols)
    with pytest.raises(ValueError, match="share memory"):
        pkg.gar_linear_weight_grad(dy, ck, shared)
    # broadcast over the tokens of one worker, over workers of one token, and over both
    for shape, stride in (((1, 4, cols), (0, 0, 1)), ((4, 1, cols), (0, 0, 1)), ((2, 2, cols), (0, 0, 1))):
        bad = x.as_strided(shape, stride)
        with pytest.raises(ValueError, match="share memory"):
            pkg.gar_linear_weight_grad(bad, ck)
        with pytest.raises(ValueError, match="share memory"):
            pkg.gar_weight_grad_workspace_bytes(bad, ck)
    # what autograd passes back through a sum
    seen = []
    y = x.clone().requires_grad_() * 1
    y.register_hook(seen.append)
    y.sum(0).backward(torch.ones(cols, dtype=x.dtype, device=DEV))
    assert seen[0].stride() == (0, 1)
    with pytest.raises(ValueError, match="share memory"):
        pkg.gar_activation_backward("silu", seen[0], f.x)
    assert torch.equal(pkg.gar_activation_backward("silu", seen[0].contiguous(), f.x).dx,
                       pkg.gar_activation_backward("silu", torch.ones_like(x), f.x).dx)
    # a single row may have any stride
    pkg.gar_token_logprobs(x.as_strided((1, cols), (0, 1)), t[:1])
    pkg.gar_linear_weight_grad(x.as_strided((1, 1, cols), (0, 0, 1)), pkg.gar_checkpoint_pack(x[:1]))
