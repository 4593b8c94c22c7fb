"""The worker-side operators on the GPU against plain implementations in 64 bits.

Tolerances, from the arithmetic (eps = 2^-24, half a unit of fp32):
  log probabilities  x - m is rounded once, its product with log2(e) once, the exponential to 2^-22: an
                     entry 20 below the maximum is off by at most 20 * 2 eps + 2^-22 < 3e-6 relative, a sum of
                     such terms added in a tree of sequential parts by less than 1e-5 relative -> 1e-5
                     absolute on log s, plus eps of each stored value's magnitude
  entropy            sum of terms |t| e^t <= ~20 of the largest, each as above -> 1e-4 absolute
  gradients          p to 1e-5 relative, times the bracket's magnitude, plus the output's rounding
  checkpoints        codes and scales exactly as the definition in fp32 gives them
  activations        1e-5 relative of the exact terms' magnitude plus the output's rounding
  weight gradients   exact products, K additions in fp32, each off by at most one unit of the
                     running sum: K 2^-23 sum |dy| |x|, plus the output's rounding"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # relative rounding error
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


# ---- log probabilities ------------------------------------------------------------------------
def logprobs_64(x, t, k):
    """(logprobs, entropy, lse, top_logprobs, top_index) on the CPU in 64 bits, rows one by one."""
    x = x.double().cpu().numpy()
    t = t.cpu().numpy()
    rows, vocab = x.shape
    out = [np.zeros(rows) for _ in range(3)] + [np.zeros((rows, k)), np.zeros((rows, k), dtype=np.int64)]
    for r in range(rows):
        v = x[r]
        bad = np.isnan(v).any() or np.isposinf(v).any()
        empty = not bad and np.isneginf(v).all()
        m = v.max() if not bad and not empty else 0.0
        e = np.exp(v - m) if not bad else v
        lse = math.nan if bad else -math.inf if empty else m + math.log(e.sum())
        lp = np.full(vocab, math.nan) if bad else np.full(vocab, -math.inf) if empty else (v - m) - math.log(e.sum())
        p = np.exp(lp)
        out[0][r] = 0.0 if t[r] < 0 else math.nan if t[r] >= vocab else lp[t[r]]
        out[1][r] = math.nan if bad else -sum((p * np.where(p > 0, lp, 0.0)).tolist()) if not empty else 0.0
        out[2][r] = lse
        order = sorted(range(vocab), key=lambda j: (np.isnan(v[j]), -v[j] if not np.isnan(v[j]) else 0.0, j))[:k]
        out[3][r], out[4][r] = lp[order], order
    return [torch.from_numpy(o) for o in out]


def check_logprobs(pkg, x, t, k, stream=None):
    r = pkg.gar_token_logprobs(x, t, top=k, stream=stream)
    torch.cuda.synchronize()
    lp, ent, lse, top, index = logprobs_64(x, t, k)
    mag = lse.abs().nan_to_num(0.0, 0.0, 0.0)
    close(r.lse.cpu(), lse, 1e-5 + 2.0 ** -23 * mag, "lse")
    close(r.logprobs.cpu(), lp, 1e-5 + 2.0 ** -22 * lp.abs().nan_to_num(0.0, 0.0, 0.0), "logprobs")
    close(r.entropy.cpu(), ent, 1e-4, "entropy")
    if k:
        assert torch.equal(r.top_index.cpu(), index)
        close(r.top_logprobs.cpu(), top, 1e-5 + 2.0 ** -22 * top.abs().nan_to_num(0.0, 0.0, 0.0), "top")
    return r


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (65, 10, 3), (33, 16, 0), (9, 17, 17), (5, 64, 32), (7, 65, 20),
                                          (3, 256, 1), (4, 257, 5), (5, 1000, 32), (3, 1024, 8), (2, 1025, 8), (4, 2049, 32),
                                          (2, 5001, 20), (1, 33001, 20), (3, 40000, 1)])
def test_logprobs(pkg, dtype, rows, vocab, k):
    x = normal((rows, vocab), dtype, 7 * vocab + rows, 3.0)
    t = torch.randint(-2, vocab, (rows,), generator=gen(vocab), device=DEV)
    check_logprobs(pkg, x, t, k)


@pytest.mark.parametrize("vocab", [50, 700, 4099, 20001])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_strides(pkg, dtype, vocab, pad, shift):
    x = strided(normal((3, vocab), dtype, vocab + pad, 2.0), pad, shift)
    check_logprobs(pkg, x, torch.tensor([0, vocab - 1, vocab // 2], device=DEV), 6)


@pytest.mark.parametrize("vocab", [12, 300, 3001, 70000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprobs_hard_rows(pkg, dtype, vocab):
    """Empty rows, rows of equal values, one live entry, the type's lowest value as a mask, infinities, NaN,
    large offsets, a target behind the mask, one past the vocabulary."""
    x = normal((14, vocab), dtype, 3 * vocab, 1.0)
    low = torch.finfo(DTYPES[dtype]).min
    x[0] = -math.inf
    x[1] = 1.5
    x[2] = -math.inf
    x[2, vocab // 3] = -2.0
    x[3, : vocab // 2] = low
    x[4] = low
    x[5, vocab - 1] = math.inf
    x[6, 0] = math.nan
    x[7] = math.nan
    x[8] += 1000.0
    x[9, : vocab - 3] = -math.inf
    x[10, 1::2] = -0.0
    x[10, 0::2] = 0.0
    x[11, vocab // 2:] = -math.inf
    x[12] = math.inf
    t = torch.randint(0, vocab, (14,), generator=gen(vocab), device=DEV)
    t[2], t[9], t[11], t[13] = vocab // 3, 0, vocab - 1, vocab
    check_logprobs(pkg, x, t, min(10, vocab))


def test_logprobs_crowded_share(pkg):
    """All the large entries in one thread's share, and more equal ones than the candidate list holds."""
    x = torch.zeros(2, 60000, device=DEV)
    x[0, ::1024] = torch.arange(59, device=DEV).float() + 1.0
    x[1, 100:2000] = 4.0
    check_logprobs(pkg, x, torch.tensor([5, 6], device=DEV), 32)


def test_logprobs_offsets_past_32_bits(pkg):
    ld = (1 << 31) + 8
    buf = torch.empty(ld * 2 + 2048, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((3, 2048), (ld, 1))
    x.copy_(normal((3, 2048), "bf16", 5, 2.0))
    t = torch.tensor([1, 2, 2047], device=DEV)
    r = check_logprobs(pkg, x, t, 4)
    dx = buf.as_strided((3, 2048), (ld, 1))
    a = torch.ones(3, device=DEV)
    want = backward_64(x, t, r, a, None, None)
    pkg.gar_token_logprobs_backward(x, r, t, a, dlogits=dx)
    torch.cuda.synchronize()
    check_grad(dx, *want, "bf16")


def backward_64(x, t, r, a, c, b):
    """Gradient and the scale of its error, in 64 bits, from the saved values the operator is given."""
    x, t = x.double().cpu(), t.cpu()
    rows, vocab = x.shape
    want, scale = torch.zeros(rows, vocab, dtype=torch.float64), torch.zeros(rows, vocab, dtype=torch.float64)
    for i in range(rows):
        lse = float(r.lse[i])
        if lse == -math.inf:
            continue
        lp = (x[i] - lse) - float(r.lse_lo[i])
        p = torch.exp(lp)
        up = torch.zeros(vocab, dtype=torch.float64)
        size = torch.zeros(vocab, dtype=torch.float64)
        total = 0.0
        if a is not None and t[i] >= 0:
            if t[i] >= vocab:
                total = math.nan
            else:
                up[t[i]] += float(a[i])
                size[t[i]] += abs(float(a[i]))
        if b is not None:
            for j in range(b.shape[1]):
                up[int(r.top_index[i, j])] += float(b[i, j])
                size[int(r.top_index[i, j])] += abs(float(b[i, j]))
        total = total + float(up.sum())
        ci = float(c[i]) if c is not None else 0.0
        h = float(r.entropy[i]) if c is not None else 0.0
        safe = torch.where(p > 0, lp, torch.zeros_like(lp))
        want[i] = up - p * (total + ci * (safe + h))
        scale[i] = size + p * (float(size.sum()) + abs(ci) * (safe.abs() + h))
    return want, scale


def check_grad(got, want, scale, dtype):
    tol = 2e-5 * scale.nan_to_num(0.0) + HALF_ULP[dtype] * want.abs().nan_to_num(0.0) + TINY[dtype]
    close(got.cpu(), want, tol, "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k,pad,shift", [(1, 1, 1, 0, 0), (40, 10, 2, 0, 0), (9, 65, 0, 1, 1), (5, 1024, 20, 0, 0),
                                                    (4, 1025, 32, 0, 0), (3, 8200, 5, 7, 3), (2, 33001, 20, 0, 0)])
@pytest.mark.parametrize("parts", ["a", "c", "b", "acb"])
def test_logprobs_backward(pkg, dtype, rows, vocab, k, pad, shift, parts):
    if parts == "b" and k == 0:
        pytest.skip("no alternatives")
    x = normal((rows, vocab), dtype, vocab, 2.0)
    if vocab > 8:
        x[0, 3:6] = -math.inf
    x = strided(x, pad, shift)
    t = torch.randint(-1, vocab, (rows,), generator=gen(rows), device=DEV)
    r = pkg.gar_token_logprobs(x, t, top=k)
    if k:
        t[0] = r.top_index[0, 0]                             # the target is one of the alternatives
    a = torch.randn(rows, generator=gen(1), device=DEV) if "a" in parts else None
    c = torch.randn(rows, generator=gen(2), device=DEV) if "c" in parts else None
    b = torch.randn(rows, k, generator=gen(3), device=DEV) if "b" in parts and k else None
    want = backward_64(x, t, r, a, c, b)
    dx = pkg.gar_token_logprobs_backward(x, r, t, a, c, b)
    check_grad(dx, *want, dtype)
    other = strided(torch.zeros_like(dx), pad + 1, shift)    # rows aligned differently from the logits'
    pkg.gar_token_logprobs_backward(x, r, t, a, c, b, dlogits=other)
    assert torch.equal(other, dx)
    pkg.gar_token_logprobs_backward(x, r, t, a, c, b, dlogits=x)
    assert torch.equal(x, dx)


def test_logprobs_backward_hard_rows(pkg):
    for vocab in (40, 3000):
        x = normal((7, vocab), "f32", vocab)
        x[0] = -math.inf
        x[1, 2] = math.nan
        x[2, 1:] = -math.inf
        x[3, 5] = math.inf
        x[6] = torch.finfo(torch.float32).min                # every entry equally likely
        t = torch.tensor([1, 1, 0, 1, vocab + 1, -100, 4], device=DEV)
        r = pkg.gar_token_logprobs(x, t, top=3)
        ones = torch.ones(7, device=DEV)
        dx = pkg.gar_token_logprobs_backward(x, r, t, ones, ones, torch.ones(7, 3, device=DEV)).cpu()
        want = torch.full((vocab,), -4.0 / vocab)
        want[:3] += 1.0                                      # the alternatives: lowest indices among equals
        want[4] += 1.0
        assert torch.all((dx[6] - want).abs() <= 2e-5)       # p and the entropy's bracket to 1e-5, |terms| <= 1
        assert torch.all(dx[0] == 0)
        assert torch.isnan(dx[[1, 3, 4]]).all()
        assert torch.isfinite(dx[[2, 5]]).all() and torch.all(dx[2, 4:] == 0)


def test_logprobs_gradient_against_differences(pkg):
    """Central differences of the operator's own forward pass along random directions.  Step h = 1e-2: the
    truncation is h^2 / 6 of third derivatives (below 1e-4 of the terms), the noise 1e-5 sqrt(rows) / h
    below 1e-2 absolute."""
    rows, vocab, k, h = 16, 3001, 4, 1e-2
    x = normal((rows, vocab), "f32", 11, 1.0)
    x[:, :k] += 6.0 + 2.0 * torch.arange(k, device=DEV)      # the alternatives keep their order within the step
    t = torch.randint(0, vocab, (rows,), generator=gen(1), device=DEV)
    t[:8] = 1
    a, c, b = (torch.randn(s, generator=gen(i), device=DEV) for i, s in enumerate([(rows,), (rows,), (rows, k)]))

    def loss(z):
        r = pkg.gar_token_logprobs(z, t, top=k)
        return float((r.logprobs.double() * a).sum() + (r.entropy.double() * c).sum() + (r.top_logprobs.double() * b).sum())
    dx = pkg.gar_token_logprobs_backward(x, pkg.gar_token_logprobs(x, t, top=k), t, a, c, b).double()
    for seed in range(4):
        v = torch.randn(rows, vocab, generator=gen(100 + seed), device=DEV)
        slope = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
        want = float((dx * v).sum())
        assert abs(slope - want) <= 2e-2 + 2e-3 * abs(want), (slope, want)


# ---- checkpoints ------------------------------------------------------------------------------
def codes_32(x, group):
    """The definition in fp32, step by step: codes, scales, restored values."""
    rows, cols = x.shape
    f = x.float().cpu().numpy()
    groups = -(-cols // group)
    q, s = np.zeros((rows, cols), dtype=np.int8), np.zeros((rows, groups), dtype=np.float32)
    with np.errstate(all="ignore"):
        for g in range(groups):
            v = f[:, g * group:(g + 1) * group]
            top = np.abs(v).max(axis=1)
            sound = np.isfinite(v).all(axis=1)
            live = sound & (top >= np.float32(2.0 ** -100))
            inv = np.where(live, (np.float32(1.0) / np.where(live, top, np.float32(1.0))) * np.float32(127.0), np.float32(0.0)).astype(np.float32)
            s[:, g] = np.where(sound, np.where(live, top / np.float32(127.0), np.float32(0.0)), np.float32(np.nan))
            prod = np.where(sound[:, None], np.where(sound[:, None], v, np.float32(0.0)) * inv[:, None], np.float32(0.0))
            q[:, g * group:(g + 1) * group] = np.rint(prod).astype(np.int8)
    scale = np.repeat(s, group, axis=1)[:, :cols]
    back = torch.from_numpy(q.astype(np.float32) * scale).to(x.dtype)
    return torch.from_numpy(q), torch.from_numpy(s), back


def same(a, b):
    a, b = a.cpu(), b.cpu()
    nan = torch.isnan(a.float())
    return torch.equal(nan, torch.isnan(b.float())) and torch.equal(a[~nan], b[~nan])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 7, 0, 0), (17, 32, 0, 0), (5, 130, 3, 1), (9, 1001, 0, 0),
                                                 (33, 256, 8, 8), (2, 4097, 7, 0)])
def test_checkpoint(pkg, dtype, group, rows, cols, pad, shift):
    x = normal((rows, cols), dtype, rows * cols, 2.0)
    x[0, cols // 2:] = 0
    x = strided(x, pad, shift)
    ck = pkg.gar_checkpoint_pack(x, group)
    q, s, back = codes_32(x, group)
    assert torch.equal(ck.q[:, :cols].cpu(), q) and same(ck.scales, s)
    got = pkg.gar_checkpoint_unpack(ck)
    assert same(got, back)
    out = strided(torch.zeros(rows, cols, dtype=x.dtype, device=DEV), pad + 1, shift)
    pkg.gar_checkpoint_unpack(ck, out)
    assert same(out, back)
    # at most half a step off, plus the rounding to the type
    step = torch.repeat_interleave(s.double(), group, dim=1)[:, :cols]
    bound = 0.5 * step * (1 + 1e-5) + HALF_ULP[dtype] * x.double().cpu().abs() * 1.01 + TINY[dtype]
    assert torch.all((got.double().cpu() - x.double().cpu()).abs() <= bound)


def test_checkpoint_special_groups(pkg):
    x = normal((6, 256), "f32", 1)
    x[0, 3] = math.nan
    x[1, 70] = math.inf
    x[2, 130] = -math.inf
    x[3] *= 1e-35                                            # below 2^-100: zeros
    x[4] *= 1e35
    x[5] = 0
    x[5, 0], x[5, 1], x[5, 2] = 127.0, 0.5, -1.5             # ties go to the even code
    ck = pkg.gar_checkpoint_pack(x, 64)
    q, s, back = codes_32(x, 64)
    assert torch.equal(ck.q.cpu(), q) and same(ck.scales, s)
    got = pkg.gar_checkpoint_unpack(ck).cpu()
    assert same(got, back)
    assert torch.isnan(got[0, :64]).all() and torch.isfinite(got[0, 64:]).all() and torch.isnan(got[1, 64:128]).all()
    assert torch.all(got[3] == 0) and q[5, 1] == 0 and q[5, 2] == -2


def test_empty_calls(pkg):
    x = torch.empty(0, 40, dtype=torch.bfloat16, device=DEV)
    assert pkg.gar_checkpoint_unpack(pkg.gar_checkpoint_pack(x)).shape == (0, 40)
    f = pkg.gar_activation_forward("silu", x, x.clone())
    assert f.y.shape == (0, 40) and pkg.gar_activation_backward("silu", x, f.x, f.up).dup.shape == (0, 40)
    r = pkg.gar_token_logprobs(x, torch.empty(0, dtype=torch.int64, device=DEV), top=2)
    assert r.top_index.shape == (0, 2)
    assert pkg.gar_token_logprobs_backward(x, r, grad_top=torch.empty(0, 2, device=DEV)).shape == (0, 40)


# ---- activations ------------------------------------------------------------------------------
def act_64(name, x):
    """act(x), act'(x) in 64 bits."""
    if name == "identity":
        return x, torch.ones_like(x)
    if name == "relu":
        return torch.where(x < 0, torch.zeros_like(x), x), (x > 0).double()
    if name == "silu":
        g = 1.0 / (1.0 + torch.exp(-x))
        return x * g, g * (1.0 + x * (1.0 - g))
    cdf = 0.5 * torch.special.erfc(-x / math.sqrt(2.0))
    return x * cdf, cdf + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["identity", "relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cols,pad,shift,group", [(1, 1, 0, 0, 32), (5, 72, 0, 0, 64), (7, 333, 1, 3, 128), (19, 512, 8, 0, 32)])
def test_activation(pkg, dtype, act, gated, rows, cols, pad, shift, group):
    # both halves of one wider buffer, as a fused projection leaves them
    wide = strided(normal((rows, 2 * cols), dtype, rows + cols, 3.0), pad, shift)
    x, up = wide[:, :cols], wide[:, cols:] if gated else None
    f = pkg.gar_activation_forward(act, x, up, group=group, save_output=True)
    xd = x.double().cpu()
    want, _ = act_64(act, xd)
    mag = xd.abs() + 1e-30
    if gated:
        want, mag = want * up.double().cpu(), mag * up.double().cpu().abs()
    close(f.y.cpu(), want, 1e-5 * mag + HALF_ULP[dtype] * want.abs() + TINY[dtype], "y")
    for ck, src in ((f.x, x), (f.up, up), (f.out, f.y)):
        if src is not None:
            q, s, _ = codes_32(src, group)
            assert torch.equal(ck.q[:, :cols].cpu(), q) and same(ck.scales, s)
    assert (f.up is None) == (not gated)

    dy = strided(normal((rows, cols), dtype, 5, 1.0), pad, shift)
    xr = pkg.gar_checkpoint_unpack(f.x).double().cpu()
    y, slope = act_64(act, xr)
    d = dy.double().cpu()
    dwide = strided(torch.zeros(rows, 2 * cols, dtype=dy.dtype, device=DEV), pad, shift)
    g = pkg.gar_activation_backward(act, dy, f.x, f.up, dx=dwide[:, :cols], dup=dwide[:, cols:] if gated else None)
    ur = pkg.gar_checkpoint_unpack(f.up).double().cpu() if gated else torch.ones_like(d)
    wdx = d * slope * ur
    close(g.dx.cpu(), wdx, 1e-5 * (d * ur).abs() * (1 + xr.abs()) + HALF_ULP[dtype] * wdx.abs() + TINY[dtype], "dx")
    if gated:
        wdup = d * y
        close(g.dup.cpu(), wdup, 1e-5 * d.abs() * (1 + xr.abs()) + HALF_ULP[dtype] * wdup.abs() + TINY[dtype], "dup")
    else:
        again = pkg.gar_activation_backward(act, dy, f.x, dx=dy)         # in place
        assert torch.equal(again.dx, g.dx)


def test_activation_in_place_and_without_checkpoints(pkg):
    x = normal((13, 200), "bf16", 3)
    want = pkg.gar_activation_forward("gelu", x).y
    f = pkg.gar_activation_forward("gelu", x, save_input=False, y=x)
    assert f.x is None and f.out is None and torch.equal(x, want)


def test_activation_extremes(pkg):
    x = torch.tensor([[0.0, -0.0, 100.0, -100.0, 3e38, -3e38, 1e-30, -1e-30]], device=DEV)
    for act in ("relu", "silu", "gelu"):
        y = pkg.gar_activation_forward(act, x, save_input=False).y.double().cpu()
        want = act_64(act, x.double().cpu())[0]
        assert torch.all((y - want).abs() <= 1e-5 * want.abs() + 1e-30), act
    bad = torch.tensor([[math.nan, 1.0, math.inf, 2.0]], device=DEV)
    y = pkg.gar_activation_forward("relu", bad, save_input=False).y.cpu()
    assert torch.isnan(y[0, 0]) and y[0, 2] == math.inf and y[0, 3] == 2.0


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_gradient_against_differences(pkg, act):
    """x is made restorable exactly, so the backward pass differentiates the forward pass at the same
    place.  Step h = 1e-2 in fp32: truncation h^2 / 6 |act'''| < 5e-5, noise 2e-6 |y| / h < 1e-3."""
    x = pkg.gar_checkpoint_unpack(pkg.gar_checkpoint_pack(normal((32, 512), "f32", 2, 1.5)))
    up = pkg.gar_checkpoint_unpack(pkg.gar_checkpoint_pack(normal((32, 512), "f32", 3, 1.0)))
    h = 1e-2
    f = pkg.gar_activation_forward(act, x, up)
    dy = torch.ones_like(x)
    g = pkg.gar_activation_backward(act, dy, f.x, f.up)

    def y(a, b):
        return pkg.gar_activation_forward(act, a, b, save_input=False).y.double()
    slope = (y(x + h, up) - y(x - h, up)) / ((x + h).double() - (x - h).double())
    assert torch.all((slope - g.dx.double()).abs() <= 3e-3 * (1 + up.double().abs()))
    slope = (y(x, up + h) - y(x, up - h)) / ((up + h).double() - (up - h).double())
    assert torch.all((slope - g.dup.double()).abs() <= 3e-3 * (1 + x.double().abs()))


# ---- weight gradients -------------------------------------------------------------------------
def weight_grad_64(dy, ck, pkg, lengths=None):
    """(dW, db, error scale of dW, of db) per worker in 64 bits from the restored activation."""
    n, t, out = dy.shape
    x = pkg.gar_checkpoint_unpack(ck).double().view(n, t, ck.cols)
    d = dy.double()
    if lengths is not None:
        live = torch.arange(t, device=DEV)[None, :, None] < lengths[:, None, None]
        d, x = torch.where(live, d, 0.0), torch.where(live, x, 0.0)
    return (torch.einsum("nto,nti->noi", d, x), d.sum(1),
            torch.einsum("nto,nti->noi", d.abs(), x.abs()), d.abs().sum(1))


def check_weight_grad(pkg, dy, ck, grads_dtype="f32", lengths=None, off=0, gap=0, tail=0):
    n, t, out = dy.shape
    weights = out * ck.cols
    d = off + weights + gap + out + tail
    grads = torch.full((n, d), 7.0, dtype=DTYPES[grads_dtype], device=DEV)
    place = dict(weight_offset=off, bias_offset=off + weights + gap, lengths=lengths)
    r = pkg.gar_linear_weight_grad(dy, ck, grads, workspace=False, **place)
    assert r is grads
    # with a workspace: the same products in the same order, the same bits, unless the tokens are cut into parts
    space = torch.full((pkg.gar_weight_grad_workspace_bytes(dy, ck, lengths, True),), 255, dtype=torch.uint8, device=DEV)
    other = pkg.gar_linear_weight_grad(dy, ck, torch.full_like(grads, 7.0), workspace=space, **place)
    cut = -(-out // 256) * (-(-ck.cols // 256) + 1) * n <= 37 and t > 7 * 64
    if not cut:
        assert torch.equal(other, grads)
    dw, db, sw, sb = weight_grad_64(dy, ck, pkg, lengths)
    unit = 2.0 ** -23 * max(t, 8)
    for block in (grads, other):
        got = block[:, off:off + weights].reshape(n, out, ck.cols)
        close(got, dw, unit * sw + HALF_ULP[grads_dtype] * dw.abs() + TINY[grads_dtype], "dW")
        got = block[:, off + weights + gap:off + weights + gap + out]
        close(got, db, unit * sb + HALF_ULP[grads_dtype] * db.abs() + TINY[grads_dtype], "db")
        # nothing else of the rows is touched
        assert torch.all(block[:, :off] == 7.0) and torch.all(block[:, off + weights:off + weights + gap] == 7.0)
        assert torch.all(block[:, d - tail:] == 7.0) if tail else True
    return grads


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,t,out,inp", [(1, 1, 1, 1), (2, 3, 5, 7), (3, 17, 10, 84), (1, 64, 128, 256), (2, 65, 129, 257),
                                         (3, 100, 500, 800), (2, 300, 136, 520), (5, 130, 264, 48), (1, 1000, 64, 1040)])
def test_weight_grad(pkg, dtype, n, t, out, inp):
    dy = normal((n, t, out), dtype, t + out)
    ck = pkg.gar_checkpoint_pack(normal((n * t, inp), dtype, inp), 32 if inp % 3 else 128)
    check_weight_grad(pkg, dy, ck)


@pytest.mark.parametrize("grads_dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("off,gap,tail", [(0, 0, 0), (1, 0, 2), (3, 5, 1), (8, 8, 8)])
@pytest.mark.parametrize("out,inp", [(72, 96), (33, 130)])
def test_weight_grad_placement(pkg, grads_dtype, off, gap, tail, out, inp):
    dy = normal((3, 40, out), "bf16", 1, 0.1)
    check_weight_grad(pkg, dy, pkg.gar_checkpoint_pack(normal((120, inp), "bf16", 2), 64), grads_dtype, None, off, gap, tail)


@pytest.mark.parametrize("out,inp", [(64, 128), (130, 200), (31, 77)])
def test_weight_grad_lengths(pkg, out, inp):
    """Workers with none, one, some and all of their tokens; what lies behind the lengths is NaN."""
    n, t = 6, 150
    dy = normal((n, t, out), "bf16", 1)
    x = normal((n * t, inp), "bf16", 2).view(n, t, inp)
    lengths = torch.tensor([0, 1, 64, 149, 150, 77], dtype=torch.int32, device=DEV)
    for w in range(n):
        dy[w, int(lengths[w]):] = math.nan
        x[w, int(lengths[w]):] = math.nan
    ck = pkg.gar_checkpoint_pack(x.view(n * t, inp), 64)
    g = check_weight_grad(pkg, dy, ck, lengths=lengths)
    assert torch.all(g[0] == 0)
    # lengths beyond the tokens and below zero are clamped
    dy, x = normal((2, 20, out), "bf16", 3), normal((40, inp), "bf16", 4)
    ck = pkg.gar_checkpoint_pack(x, 64)
    a = pkg.gar_linear_weight_grad(dy, ck, lengths=torch.tensor([1000, -3], dtype=torch.int32, device=DEV))
    b = pkg.gar_linear_weight_grad(dy, ck)
    assert torch.equal(a[0], b[0]) and torch.all(a[1] == 0)


@pytest.mark.parametrize("tokens", [40, 150, 257, 800])
def test_weight_grad_lengths_over_many_tiles(pkg, tokens):
    """Several tiles per CTA pair, workers that end inside a step, on its edge, and empty ones among them."""
    n, out, inp = 12, 1100, 2100
    dy, x = normal((n, tokens, out), "bf16", 1), normal((n * tokens, inp), "bf16", 2)
    lengths = torch.randint(0, tokens + 1, (n,), generator=gen(tokens), device=DEV, dtype=torch.int32)
    lengths[0], lengths[5], lengths[11] = tokens, 0, min(tokens, 128)
    check_weight_grad(pkg, dy, pkg.gar_checkpoint_pack(x, 128), lengths=lengths)


@pytest.mark.parametrize("dtype,grads_dtype", [("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("n,t,out,inp", [(1, 1, 264, 16), (3, 100, 520, 800), (2, 512, 1032, 264), (12, 150, 1104, 2104), (5, 513, 272, 520),
                                         (40, 65, 800, 1300)])
def test_weight_grad_panels(pkg, dtype, grads_dtype, n, t, out, inp):
    """Several output tiles per worker at up to 512 tokens (and one more): panels of one to eight steps, runs of
    tiles that begin and end inside a panel, workers and bias tiles in between; against 64 bits, and against
    the same call with lengths that leave every token in (another path, the same order of products)."""
    dy = normal((n, t, out), dtype, t + out)
    ck = pkg.gar_checkpoint_pack(normal((n * t, inp), dtype, inp), 64)
    g = check_weight_grad(pkg, dy, ck, grads_dtype)
    lengths = torch.full((n,), t, dtype=torch.int32, device=DEV)
    assert torch.equal(check_weight_grad(pkg, dy, ck, grads_dtype, lengths), g)


@pytest.mark.parametrize("n,t,out,inp", [(2, 1100, 136, 264), (1, 2500, 40, 70), (3, 1025, 300, 520), (2, 2049, 33, 250)])
@pytest.mark.parametrize("grads_dtype", ["f32", "f16"])
def test_weight_grad_long_sums(pkg, n, t, out, inp, grads_dtype):
    """Sums of more than 1024 tokens, which fp32 results join from chunks: stored and added by TMA or plainly, with
    lengths that end in the first chunk, on its edge and in the last one.  All values positive: the sums
    grow steadily, the case in which additions that truncate lose most.  The chunks' sums stay within 2e-6."""
    dy, x = normal((n, t, out), "bf16", t).abs(), normal((n * t, inp), "bf16", inp).abs()
    ck = pkg.gar_checkpoint_pack(x, 64)
    g = check_weight_grad(pkg, dy, ck, grads_dtype)
    lengths = torch.tensor([700, 1024, t][:n], dtype=torch.int32, device=DEV)
    check_weight_grad(pkg, dy, ck, grads_dtype, lengths)
    if grads_dtype == "f32":
        dw, _, _, _ = weight_grad_64(dy, ck, pkg)
        got = g[:, :out * inp].reshape(n, out, inp).double()
        assert float((got - dw).norm()) <= 2e-6 * float(dw.norm())


@pytest.mark.parametrize("grads_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,t,out,inp", [(1, 769, 24, 40), (1, 3000, 100, 77), (2, 4099, 300, 600), (5, 1500, 31, 250), (3, 12000, 64, 64)])
def test_weight_grad_cut_tokens(pkg, grads_dtype, n, t, out, inp):
    """Few output tiles, many tokens: parts of the tokens joined in order; lengths that leave parts empty."""
    dy, ck = normal((n, t, out), "bf16", t), pkg.gar_checkpoint_pack(normal((n * t, inp), "bf16", inp), 64)
    check_weight_grad(pkg, dy, ck, grads_dtype, None, 3, 1, 2)
    lengths = torch.tensor([65, t // 2, 0, t, 1][:n], dtype=torch.int32, device=DEV)
    check_weight_grad(pkg, dy, ck, grads_dtype, lengths)
    a, b = (pkg.gar_linear_weight_grad(dy, ck) for _ in range(2))
    assert torch.equal(a, b)


@pytest.mark.parametrize("n,t,out,inp", [(5, 473, 616, 15), (4, 497, 424, 403), (1, 512, 520, 64), (2, 449, 264, 100), (1, 448, 1320, 34)])
def test_weight_grad_few_tiles_of_a_panel(pkg, n, t, out, inp):
    """Few output tiles at 449 to 512 tokens: enough steps to be cut, but panels are not; with a workspace that
    is larger than asked for (of NaN bytes) and the one the call takes by itself, the same bits as without."""
    dy, ck = normal((n, t, out), "f16", t), pkg.gar_checkpoint_pack(normal((n * t, inp), "f16", inp), 64)
    grads = check_weight_grad(pkg, dy, ck, "f32", None, 7)
    want = check_weight_grad(pkg, dy, ck)
    assert torch.equal(grads[:, 7:7 + out * inp], want[:, :out * inp])
    space = torch.full((1 << 22,), 255, dtype=torch.uint8, device=DEV)
    for w in (None, space):
        got = pkg.gar_linear_weight_grad(dy, ck, torch.full_like(want, 7.0), 0, out * inp, workspace=w)
        assert torch.equal(got[:, :out * inp + out], want[:, :out * inp + out])


def test_weight_grad_workers_do_not_meet(pkg):
    """A NaN of one worker (a Byzantine one, say) stays in its own row: the others' bits do not change."""
    n, t = 4, 70                                             # 70 tokens: every worker ends inside a tile
    for out, inp in ((128, 256), (130, 200)):
        dy, x = normal((n, t, out), "bf16", 1), normal((n * t, inp), "bf16", 2)
        clean = pkg.gar_linear_weight_grad(dy, pkg.gar_checkpoint_pack(x, 64))
        dy[2] = math.nan
        x[2 * t:3 * t] = math.inf
        ck = pkg.gar_checkpoint_pack(x, 64)
        for space in (False, torch.empty(pkg.gar_weight_grad_workspace_bytes(dy, ck), dtype=torch.uint8, device=DEV)):
            got = pkg.gar_linear_weight_grad(dy, ck, workspace=space)
            assert torch.equal(got[[0, 1, 3]], clean[[0, 1, 3]]) and torch.isnan(got[2]).all()


def test_weight_grad_strided_dy_and_no_tokens(pkg):
    wide = normal((2 * 50, 300), "f16", 1)
    for c0, out in ((0, 128), (3, 99), (8, 264)):
        dy = wide.view(2, 50, 300)[:, :, c0:c0 + out]
        check_weight_grad(pkg, dy, pkg.gar_checkpoint_pack(normal((100, 90), "f16", 2), 32))
    dy = torch.empty(2, 0, 24, dtype=torch.bfloat16, device=DEV)
    ck = pkg.gar_checkpoint_pack(torch.empty(0, 40, dtype=torch.bfloat16, device=DEV), 32)
    g = torch.full((2, 24 * 40), 3.0, device=DEV)
    assert torch.all(pkg.gar_linear_weight_grad(dy, ck, g) == 0)


def test_weight_grad_is_the_derivative(pkg):
    """The layer is linear in W: the difference quotient along V is <dy, x' V^T> exactly."""
    n, t, out, inp = 2, 90, 48, 112
    dy = normal((n, t, out), "bf16", 1)
    ck = pkg.gar_checkpoint_pack(normal((n * t, inp), "bf16", 2), 64)
    g = pkg.gar_linear_weight_grad(dy, ck).double().view(n, out, inp)
    x = pkg.gar_checkpoint_unpack(ck).double().view(n, t, inp)
    for seed in range(3):
        v = torch.randn(out, inp, generator=gen(seed), device=DEV).double()
        want = torch.einsum("nto,nto->n", dy.double(), torch.einsum("nti,oi->nto", x, v))
        got = torch.einsum("noi,oi->n", g, v)
        bound = torch.einsum("nto,nto->n", dy.double().abs(), torch.einsum("nti,oi->nto", x.abs(), v.abs())) * t * 2.0 ** -23
        assert torch.all((got - want).abs() <= bound)


def test_repeated_calls_give_the_same_bits_on_any_stream(pkg):
    x = normal((300, 4000), "bf16", 1, 2.0)
    t = torch.randint(0, 4000, (300,), generator=gen(2), device=DEV)
    dy = normal((3, 100, 264), "bf16", 3)

    def all_of(stream=None):
        r = pkg.gar_token_logprobs(x, t, top=7, stream=stream)
        d = pkg.gar_token_logprobs_backward(x, r, t, r.entropy, r.entropy, r.top_logprobs, stream=stream)
        f = pkg.gar_activation_forward("gelu", x, x.clone() if stream is None else up, stream=stream)
        b = pkg.gar_activation_backward("gelu", x, f.x, f.up, stream=stream)
        w = pkg.gar_linear_weight_grad(dy, f.x, stream=stream)
        return [*r, d, f.y, f.x.q, f.x.scales, b.dx, b.dup, w]
    up = x.clone()
    first = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = all_of(side)
    torch.cuda.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_python_refusals(pkg):
    x = normal((4, 64), "bf16", 1)
    with pytest.raises(TypeError):
        pkg.gar_token_logprobs(x.cpu())
    with pytest.raises(TypeError):
        pkg.gar_token_logprobs(x, torch.zeros(4, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        pkg.gar_token_logprobs(x.t())
    with pytest.raises(pkg.GarError):
        pkg.gar_token_logprobs(x, top=33)
    with pytest.raises(ValueError):
        pkg.gar_checkpoint_pack(x, 48)
    with pytest.raises(KeyError):
        pkg.gar_activation_forward("tanh", x)
    ck = pkg.gar_checkpoint_pack(x)
    with pytest.raises(ValueError):
        pkg.gar_linear_weight_grad(x.view(2, 1, 128), ck)
    with pytest.raises(pkg.GarError):
        pkg.gar_linear_weight_grad(x.float().view(1, 4, 64), pkg.gar_checkpoint_pack(x.float()))
    with pytest.raises(ValueError):
        pkg.gar_linear_weight_grad(x.view(1, 4, 64), ck, torch.empty(1, 4096, device=DEV), weight_offset=1)
