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


# ---- sums over many tokens ------------------------------------------------------------------------
def products_64(pkg, dy, ck, lengths=None):
    """dW, db and the sum of the terms' magnitudes per worker in 64 bits from the restored activation."""
    n, t, out = dy.shape
    x, d = pkg.gar_checkpoint_unpack(ck).double().view(n, t, ck.cols), dy.double()
    if lengths is not None:
        live = torch.arange(t, device=DEV)[None, :, None] < lengths[:, None, None]
        d, x = torch.where(live, d, 0.0), torch.where(live, x, 0.0)
    return torch.einsum("nto,nti->noi", d, x), d.sum(1), torch.einsum("nto,nti->noi", d.abs(), x.abs()), d.abs().sum(1)


def weight_grads(pkg, dy, ck, dtype, lengths, off, space):
    """(dW, db) from a block whose rows are 1 longer than the layer and start it at `off`."""
    n, _, out = dy.shape
    weights = out * ck.cols
    g = torch.full((n, off + weights + out + 1), 7.0, dtype=dtype, device=DEV)
    pkg.gar_linear_weight_grad(dy, ck, g, off, off + weights, lengths, workspace=space)
    assert torch.all(g[:, :off] == 7.0) and torch.all(g[:, -1] == 7.0)
    return g[:, off:off + weights].reshape(n, out, ck.cols), g[:, off + weights:-1]


def half_unit(x, dtype):
    """Half the distance of the type's numbers around x (normal numbers)."""
    bits = {torch.float32: 24, torch.bfloat16: 8, torch.float16: 11}[dtype]
    return torch.exp2(torch.floor(torch.log2(x.abs())) - bits)


@pytest.mark.parametrize("out,inp,off", [(300, 520, 3), (264, 264, 8)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens", [769, 2049, 16384])
def test_weight_grad_16_bit_results_of_many_tokens(pkg, out, inp, off, dtype, tokens):
    """Positive operands, so that sums grow steadily, the case in which additions that truncate lose most.  An accumulator
    takes 2048 tokens in 128 instructions, each of which may lose a unit of the accumulator (half the final one on
    average) and one of the products' common exponent: 128 2^-23 at most; the joins add 8 2^-24.  That on top
    of the result's own rounding, half a unit.  One accumulator of 16384 tokens loses 3e-5 and more."""
    dy = normal((1, tokens, out), torch.bfloat16, tokens).abs()
    ck = pkg.gar_checkpoint_pack(normal((tokens, inp), torch.bfloat16, out).abs(), 64)
    dw, db, _, _ = products_64(pkg, dy, ck)
    for space in (False, True):
        for got, want in zip(weight_grads(pkg, dy, ck, getattr(torch, dtype), None, off, space), (dw, db)):
            assert torch.all((got.double() - want).abs() <= half_unit(want, got.dtype) + (128 * 2.0 ** -23 + 8 * 2.0 ** -24) * want)


def test_weight_grad_16_bit_results_are_not_biased(pkg):
    """Positive operands, 16384 tokens, binary16 results.  A result's rounding is off by at most 2^-11 of it either way,
    2.9e-4 rms, so the mean over 66560 of them by 1.1e-6, five times that at most 5.6e-6; the sums of 2048 tokens
    are short by 5.7e-6.  A single truncating accumulator is short by 3e-5 and more."""
    t, out, inp = 16384, 64, 1040
    dy = normal((1, t, out), torch.bfloat16, 1).abs()
    ck = pkg.gar_checkpoint_pack(normal((t, inp), torch.bfloat16, 2).abs(), 64)
    want = products_64(pkg, dy, ck)[0]
    for space in (False, True):
        got = weight_grads(pkg, dy, ck, torch.float16, None, 0, space)[0].double()
        assert abs(float(((got - want) / want).mean())) <= 1.2e-5


@pytest.mark.parametrize("out,inp,off", [(40, 72, 0), (33, 70, 3), (520, 264, 0)])
@pytest.mark.parametrize("dtype,tokens,ends", [("float32", 768, None), ("float32", 1536, None), ("float32", 2304, (767, 768, 769, 1536)),
                                               ("float32", 1537, (1535, 1536, 1537, 0)), ("bfloat16", 2048, None), ("bfloat16", 4096, None),
                                               ("float16", 4097, (2047, 2048, 2049, 4096)), ("bfloat16", 6145, (6144, 4095, 6145, 0))])
def test_weight_grad_at_the_edges_of_chunks(pkg, out, inp, off, dtype, tokens, ends):
    """Tokens that end on, before and behind a multiple of what an accumulator sums (768 tokens, 2048 for 16-bit
    results), stored by TMA and plainly, with a bias, several tiles to a pair.  Additions are off by a unit of the running
    sum at most: one for every token of a chunk, and one for every chunk."""
    n = 4 if ends else 2
    dy = normal((n, tokens, out), torch.bfloat16, tokens)
    ck = pkg.gar_checkpoint_pack(normal((n * tokens, inp), torch.bfloat16, inp), 32)
    lengths = torch.tensor(ends, dtype=torch.int32, device=DEV) if ends else None
    dw, db, sw, sb = products_64(pkg, dy, ck, lengths)
    unit = ((768 if dtype == "float32" else 2048) + 4) * 2.0 ** -23
    half = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    for space in (False, True):
        w, b = weight_grads(pkg, dy, ck, getattr(torch, dtype), lengths, off, space)
        assert torch.all((w.double() - dw).abs() <= unit * sw + half * dw.abs() + 2.0 ** -25)
        assert torch.all((b.double() - db).abs() <= unit * sb + half * db.abs() + 2.0 ** -25)
        if dtype == "float32":
            assert float((w.double() - dw).norm()) <= 2e-6 * float(dw.norm())


@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_weight_grad_chunks_over_many_tiles(pkg, dtype):
    """Several tiles of one, two and more chunks for every pair of CTAs, empty workers among them: the halves of tensor
    memory change hands between tiles and chunks."""
    n, t, out, inp = 12, 2304, 1100, 1600
    dy = normal((n, t, out), torch.bfloat16, 1)
    ck = pkg.gar_checkpoint_pack(normal((n * t, inp), torch.bfloat16, 2), 128)
    lengths = torch.tensor([t, 0, 700, 768, 769, 2048, 2049, 1, 1536, 0, 1537, t], dtype=torch.int32, device=DEV)
    dw, db, sw, sb = products_64(pkg, dy, ck, lengths)
    unit = ((768 if dtype == "float32" else 2048) + 4) * 2.0 ** -23
    half = {"float32": 2.0 ** -24, "float16": 2.0 ** -11}[dtype]
    for space in (False, True):
        w, b = weight_grads(pkg, dy, ck, getattr(torch, dtype), lengths, 0, space)
        assert torch.all((w.double() - dw).abs() <= unit * sw + half * dw.abs() + 2.0 ** -25)
        assert torch.all((b.double() - db).abs() <= unit * sb + half * db.abs() + 2.0 ** -25)


# ---- GELU of negative values -----------------------------------------------------------------------
TYPES = {"float32": (2.0 ** -24, 1e-37), "bfloat16": (2.0 ** -8, 1e-37), "float16": (2.0 ** -11, 2.0 ** -25)}


def gelu_64(x):
    """GELU and its derivative in 64 bits."""
    cdf = 0.5 * torch.special.erfc(-x / math.sqrt(2.0))
    return x * cdf, cdf + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_gelu_of_negative_values(pkg, dtype):
    """x in [-6, -2], where GELU falls to 6e-9 of x: relative to the result.  The argument x / sqrt 2 is off by 1.5 units of
    2^-24, which erfc amplifies by x^2 <= 36, erfc itself by 4 units, the exponential of -x^2 / 2 by about as much as
    the argument: below 5e-6, and the derivative's two terms are of one size and sign or 4 times apart.  On top of that the
    output's rounding."""
    half, tiny = TYPES[dtype]
    x = torch.linspace(-6.0, -2.0, 8192, device=DEV).view(64, 128).to(getattr(torch, dtype))
    want, _ = gelu_64(x.double())
    f = pkg.gar_activation_forward("gelu", x, group=32)
    assert torch.all((f.y.double() - want).abs() <= (5e-6 + half) * want.abs() + tiny)
    xr = pkg.gar_checkpoint_unpack(f.x)
    assert torch.all(xr < -1.9)
    _, slope = gelu_64(xr.double())
    g = pkg.gar_activation_backward("gelu", torch.ones_like(x), f.x)
    assert torch.all((g.dx.double() - slope).abs() <= (1e-5 + half) * slope.abs() + tiny)
    # gated: the gradient at `up` is dy act(x)
    f = pkg.gar_activation_forward("gelu", x, torch.ones_like(x), group=32)
    g = pkg.gar_activation_backward("gelu", torch.ones_like(x), f.x, f.up)
    want, _ = gelu_64(xr.double())
    assert torch.all((g.dup.double() - want).abs() <= (5e-6 + half) * want.abs() + tiny)


# ---- the gradient of rows that are masked throughout -------------------------------------------------
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [5, 64, 65, 300, 3000, 20000])
def test_empty_rows_have_gradient_zero_whatever_comes_in(pkg, dtype, vocab):
    """A row of -inf has log probabilities of -inf, so what comes back from a loss over them is often infinite or
    NaN.  Its gradient is 0 at every vocabulary, with targets and indices outside of it too; other rows that name
    such a target are NaN."""
    top, rows = 3, 8
    x = normal((rows, vocab), getattr(torch, dtype), vocab)
    x[:6] = -math.inf
    t = torch.tensor([0, 1, 2, 3, vocab, -1, vocab, 1], device=DEV)
    r = pkg.gar_token_logprobs(x, t, top=top)
    r.top_index[4, 1] = vocab + 7
    a, c, b = (torch.ones(s, device=DEV) for s in ((rows,), (rows,), (rows, top)))
    a[0], a[1], c[2], c[3], b[3, 1], b[5, 0] = math.inf, math.nan, -math.inf, math.nan, math.nan, math.inf
    for out in (None, torch.full_like(x, 7.0), x.clone()):
        src = out if out is not None and torch.isinf(out[0, 0]) else x
        dx = pkg.gar_token_logprobs_backward(src, r, t, a, c, b, dlogits=out)
        assert torch.all(dx[:6] == 0) and torch.isnan(dx[6]).all() and torch.isfinite(dx[7]).all()


# ---- groups that hold the type's largest value --------------------------------------------------------
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_finite_value_is_restored_finite(pkg, dtype, sign):
    """Masks of the type's lowest value (or its highest) in an activation: a finite group is restored finite, each value
    within half a step and two roundings (2^-23 of the largest)."""
    x = normal((4, 256), getattr(torch, dtype), 1)
    big = torch.finfo(x.dtype).max
    x[0, 3] = sign * big
    x[1] = sign * big
    x[2, 64:] = torch.nextafter(torch.tensor(big), torch.tensor(0.0)) if dtype == "float32" else big / 2
    ck = pkg.gar_checkpoint_pack(x, 64)
    got = pkg.gar_checkpoint_unpack(ck).double()
    assert torch.isfinite(got).all()
    top = x.double().unflatten(1, (-1, 64)).abs().amax(2).repeat_interleave(64, 1)
    half = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    assert torch.all((got - x.double()).abs() <= top * (0.5 / 127 * (1 + 1e-5) + 2.0 ** -23 + half))
    f = pkg.gar_activation_forward("silu", x, group=64)
    assert torch.isfinite(pkg.gar_activation_backward("silu", torch.ones_like(x), f.x).dx).all()


# ---- autograd -----------------------------------------------------------------------------------------
def test_tensors_that_a_call_writes_count_as_modified(pkg):
    """Autograd has to see that a tensor it saved was overwritten; results themselves carry no gradient function."""
    x = normal((4, 64), torch.bfloat16, 1)
    t = torch.zeros(4, dtype=torch.int64, device=DEV)
    ones = torch.ones(4, device=DEV)
    r = pkg.gar_token_logprobs(x, t)
    f = pkg.gar_activation_forward("silu", x, x.clone())

    def versions(*outs):
        return [o._version for o in outs]
    y, dx, dup, g = (torch.empty_like(x) for _ in range(4))
    block = torch.empty(1, 64 * 64, device=DEV)
    before = versions(x, y, dx, dup, g, block)
    pkg.gar_activation_forward("silu", x, y=y)
    pkg.gar_activation_backward("silu", x, f.x, f.up, dx=dx, dup=dup)
    pkg.gar_token_logprobs_backward(x, r, t, ones, dlogits=g)
    pkg.gar_linear_weight_grad(x.view(1, 4, 64), f.x, block)
    after = versions(x, y, dx, dup, g, block)
    assert after[0] == before[0] and all(a > b for a, b in zip(after[1:], before[1:]))
    pkg.gar_checkpoint_unpack(f.x, y)
    assert y._version > after[1]

    w = x.float().requires_grad_()
    h = w * 1
    loss = (h * h).sum()                                     # saves h
    out = pkg.gar_activation_forward("relu", h, save_input=False, y=h)
    assert out.y is h or out.y.data_ptr() == h.data_ptr()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    assert pkg.gar_activation_forward("relu", w, save_input=False).y.grad_fn is None
    with torch.inference_mode():
        z = torch.ones(2, 64, device=DEV)
        pkg.gar_activation_forward("relu", z, save_input=False, y=z)
    pkg.gar_activation_forward("relu", z, save_input=False, y=z)      # an inference tensor has no version


# ---- rings of slots -----------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens", [60, 128, 250, 320, 513, 700])
@pytest.mark.parametrize("lead", [0, 1])
def test_weight_grad_bias_tiles_between_tiles_with_codes(pkg, tokens, lead):
    """Several tiles for every pair of CTAs, a bias tile (whose steps have no codes) after every eight, one to eleven
    steps a tile: the slots of codes change between the groups of restore warps.  dy by TMA, and (rows that start
    anywhere) by the restore warps."""
    n, out, inp = 37, 200, 2000
    dy = normal((n, tokens, out + lead), torch.bfloat16, tokens)[:, :, lead:]
    ck = pkg.gar_checkpoint_pack(normal((n * tokens, inp), torch.bfloat16, inp), 32)
    lengths = torch.randint(0, tokens + 1, (n,), generator=gen(tokens), device=DEV, dtype=torch.int32)
    for lens in (None, lengths):
        dw, db, sw, sb = products_64(pkg, dy, ck, lens)
        w, b = weight_grads(pkg, dy, ck, torch.float32, lens, 0, False)
        unit = max(tokens, 8) * 2.0 ** -23
        assert torch.all((w.double() - dw).abs() <= unit * sw + 2.0 ** -24 * dw.abs())
        assert torch.all((b.double() - db).abs() <= unit * sb + 2.0 ** -24 * db.abs())


# ---- graphs and threads -------------------------------------------------------------------------------
def all_calls(pkg, x, t, dy, stream=None):
    """Every operator once, on shapes that take several paths (a small and a long vocabulary, panels, restored x, cut
    tokens); the results."""
    out = []
    for z in (x[:, :50], x):
        r = pkg.gar_token_logprobs(z, t, top=5, stream=stream)
        out += [*r, pkg.gar_token_logprobs_backward(z, r, t, r.entropy, r.entropy, r.top_logprobs, stream=stream)]
    f = pkg.gar_activation_forward("gelu", x, x, save_output=True, stream=stream)
    b = pkg.gar_activation_backward("gelu", x, f.x, f.up, stream=stream)
    rows, cols = x.shape
    out += [q[:, :cols] for q in (f.x.q, f.up.q, f.out.q)]   # the padding of the codes is not written
    out += [f.y, f.x.scales, f.out.scales, b.dx, b.dup, pkg.gar_checkpoint_unpack(f.out, stream=stream)]
    for workers in (1, 2, 8):                                # 2048 and 1024 tokens cut or restored, 256: panels
        ck = pkg.gar_checkpoint_pack(x, 64, stream=stream)
        d = dy.view(workers, rows // workers, -1)
        out += [pkg.gar_linear_weight_grad(d, ck, stream=stream),
                pkg.gar_linear_weight_grad(d[:, :, :40].contiguous(), ck, grads_dtype=torch.bfloat16, stream=stream)]
    return out


def test_calls_in_a_graph(pkg):
    """A captured sequence of all calls, replayed on other inputs, gives the bits of the plain calls."""
    x, dy = normal((2048, 2056), torch.bfloat16, 1), normal((2048, 2048), torch.bfloat16, 2)
    t = torch.randint(-1, 50, (2048,), generator=gen(3), device=DEV)
    all_calls(pkg, x, t, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_calls(pkg, x, t, dy)
    for seed in (10, 20):
        x.copy_(normal(x.shape, x.dtype, seed))
        dy.copy_(normal(dy.shape, dy.dtype, seed + 1))
        t.copy_(torch.randint(-1, 50, (2048,), generator=gen(seed + 2), device=DEV))
        graph.replay()
        want = all_calls(pkg, x, t, dy)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(held, want)):
            assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b), i


def test_calls_from_two_threads(pkg):
    """Two threads, each with inputs and a stream of its own, give the bits of one."""
    import threading
    data = [(normal((2048, 2056), torch.bfloat16, s), torch.randint(-1, 50, (2048,), generator=gen(s), device=DEV),
             normal((2048, 2048), torch.bfloat16, s + 1)) for s in (1, 5)]
    want = [all_calls(pkg, *d) for d in data]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                for _ in range(5):
                    got[i].append(all_calls(pkg, *data[i]))
            side.synchronize()
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors
    for i in range(2):
        for run in got[i]:
            for a, b in zip(run, want[i]):
                assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)
