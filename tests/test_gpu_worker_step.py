"""The worker-side operators and the aggregation together, as a training step uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def step():
    import __graft_entry__ as entry
    entry.build()
    from paper_1905_04374_b200 import worker_step
    return worker_step


def restored(x, group=128):
    """x rounded to the 8-bit grid of its checkpoint (64 bits, then x's type)."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % group)).unflatten(1, (-1, group))
    top = v.abs().amax(2, keepdim=True).clamp_min(1e-300)
    return (torch.round(127 * v / top) * top / 127).flatten(1)[:, :cols].to(x.dtype).double()


def test_gradient_rows_against_the_formulas(step):
    """Every row of the block against the chain rule in 64 bits on the restored activations.  The path rounds to
    bfloat16 (2^-8 relative) at h, y, the logits, dlogits, dy and dh, and a code next to a half step may fall on
    either side of it: 3 % of a row's norm leaves those six roundings several times over."""
    n, f, tokens, inputs, hidden, classes = 5, 0, 96, 130, 72, 33
    model = step.WorkerStep(n, f, inputs, hidden, classes, DEV)
    x, t = step.batch(n, tokens, inputs, classes, 3, DEV)
    t[1, :5] = -100                                          # tokens without a target
    losses = model.gradients(x, t)
    w1, w2 = model.view("w1").bfloat16().double(), model.view("w2").bfloat16().double()
    b1, b2 = model.view("b1").double(), model.view("b2").double()
    for w in range(n):
        h = (x[w].double() @ w1.t() + b1).bfloat16()
        cdf = 0.5 * torch.special.erfc(-h.double() / math.sqrt(2))
        y = (h.double() * cdf).bfloat16()
        logp = torch.log_softmax((y.double() @ w2.t() + b2).bfloat16().double(), 1)
        live = (t[w] >= 0).double()
        picked = logp.gather(1, t[w].clamp_min(0)[:, None])[:, 0] * live
        assert abs(float(losses[w]) + float(picked.mean())) <= 2e-2
        up = torch.zeros_like(logp).scatter_(1, t[w].clamp_min(0)[:, None], (-live / tokens)[:, None])
        dlogits = up - logp.exp() * up.sum(1, keepdim=True)
        hr = restored(h)
        slope = 0.5 * torch.special.erfc(-hr / math.sqrt(2)) + hr * torch.exp(-0.5 * hr * hr) / math.sqrt(2 * math.pi)
        dh = (dlogits @ w2) * slope
        want = {"w2": dlogits.t() @ restored(y), "b2": dlogits.sum(0), "w1": dh.t() @ restored(x[w]), "b1": dh.sum(0)}
        for name, v in want.items():
            got = model.grads[w, model.offsets[name]:model.offsets[name] + v.numel()].double().view(v.shape)
            assert float((got - v).norm()) <= 0.03 * float(v.norm()), (w, name)


def test_training_survives_the_attack(step):
    """Two of eleven workers send -10 times the mean gradient: averaging diverges, multi-Bulyan learns as without them."""
    clean = step.train("average", attacked=False, steps=40)
    robust = step.train("multi_bulyan", steps=40)
    broken = step.train("average", steps=40)
    assert clean[-1] < 0.5 * clean[0] and robust[-1] < 0.5 * robust[0]
    assert not broken[-1] < broken[0]                        # NaN counts as broken
