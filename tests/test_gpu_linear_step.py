"""A worker's layers together with the worker-side operators and the aggregation, as a training step uses them, and their calls
captured, from several threads and on several streams."""
import math
import threading

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


@pytest.fixture(scope="module")
def step(pkg):
    from paper_1905_04374_b200 import worker_step
    return worker_step


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).bfloat16()


def in_8_bits(x, group=128):
    """x on the grid of its checkpoint (64 bits, then bfloat16)."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % group)).unflatten(1, (-1, group))
    top = v.abs().amax(2, keepdim=True).clamp_min(1e-300)
    return (torch.round(127 * v / top) * top / 127).flatten(1)[:, :cols].bfloat16().double()


@pytest.mark.parametrize("dropout", [0.0, 0.25])
def test_gradient_rows_against_the_formulas(pkg, step, dropout):
    """Every row of the block against the chain rule in 64 bits on the restored activations.  The path rounds to
    bfloat16 (2^-8 relative) at y, twice with dropout, dz, dy and dgate / dup, and a code next to a half step may fall on
    either side of it: 3 % of a row's norm leaves those roundings several times over."""
    n, tokens, inputs, hidden, classes = 5, 96, 130, 72, 33
    model = step.GatedStep(n, 0, inputs, hidden, classes, DEV, dropout=dropout)
    with torch.no_grad():
        for name in ("bg", "bu", "b2"):
            model.view(name).normal_(0.0, 0.3, generator=gen(1))
    model.steps += 4
    mask = pkg.gar_dropout(torch.ones(n * tokens, hidden, device=DEV), dropout, model.seed, 4).double()
    x, t = step.batch(n, tokens, inputs, classes, 3, DEV)
    t[1, :5] = -100                                          # tokens without a target
    losses = model.gradients(x, t)
    assert int(model.steps) == 5
    w = {name: model.view(name).bfloat16().double() for name in model.shapes}
    for k in range(n):
        xs, m = x[k].double(), mask[k * tokens:(k + 1) * tokens]
        g, u = xs @ w["wg"].t() + w["bg"], xs @ w["wu"].t() + w["bu"]
        y = g * torch.sigmoid(g) * u * m
        logp = torch.log_softmax(y @ w["w2"].t() + w["b2"], 1)
        live = (t[k] >= 0).double()
        picked = logp.gather(1, t[k].clamp_min(0)[:, None])[:, 0] * live
        assert abs(float(losses[k]) + float(picked.mean())) <= 2e-2
        up = torch.zeros_like(logp).scatter_(1, t[k].clamp_min(0)[:, None], (-live / tokens)[:, None])
        dz = up - logp.exp() * up.sum(1, keepdim=True)
        dy = dz @ w["w2"] * m
        g, u, xr = in_8_bits(g), in_8_bits(u), in_8_bits(x[k])
        s = torch.sigmoid(g)
        dg, du = dy * u * (s + g * s * (1 - s)), dy * g * s
        want = {"w2": dz.t() @ y, "b2": dz.sum(0), "wg": dg.t() @ xr, "bg": dg.sum(0), "wu": du.t() @ xr, "bu": du.sum(0)}
        for name, v in want.items():
            got = model.grads[k, model.offsets[name]:model.offsets[name] + v.numel()].double().view(v.shape)
            assert float((got - v).norm()) <= 0.03 * float(v.norm()), (k, name)


def test_the_gated_model_runs(step):
    """A few steps with the aggregation, two of eleven workers Byzantine: the losses are numbers, and a selection was made."""
    history = step.train("multi_bulyan", steps=4, tokens=40, model="gated", dropout=0.1)
    assert len(history) == 4 and all(math.isfinite(v) for v in history)


# ---- graphs, threads, streams -------------------------------------------------------------------
def all_calls(pkg, x, t, w, wg, wu, counter, stream=None):
    """Every operator, on shapes that take several paths (few rows, copies, several pieces, parts of sums, rows that start
    anywhere); the results."""
    kw = dict(stream=stream)
    out = []
    rows = x.shape[0]
    for xs, ws in ((x, w), (x[:5], w), (x[:, :-3], w[:, :-3]), (x[:64], w[:300])):
        r = pkg.gar_linear_logprobs(xs, ws, t[:xs.shape[0]] % ws.shape[0], **kw)
        grads = torch.empty(1, ws.numel(), device=x.device)
        a = torch.full((xs.shape[0],), -1.0 / rows, device=x.device)
        dx = pkg.gar_linear_logprobs_backward(xs, ws, r, t[:xs.shape[0]] % ws.shape[0], a, grads=grads, **kw)
        out += [*r, grads, dx]
    for xs in (x, x[:5]):
        f = pkg.gar_gated_linear_forward("silu", xs, wg, wu, save_output=True, **kw)
        b = pkg.gar_gated_linear_backward("silu", f.y, f.x, f.up, wg, wu, **kw)
        out += [f.y, f.x.scales, f.up.scales, f.out.scales, *b, pkg.gar_gated_linear_forward("gelu", xs, wg, wu, save_input=False, **kw).y]
    out += [pkg.gar_dropout(x, 0.3, 5, 7, counter=counter, **kw), pkg.gar_dropout(x[:, 1:], 0.3, 5, 7, residual=x[:, :-1], **kw)]
    return out


def inputs(seed, rows=700):
    return (normal((rows, 136), seed), torch.randint(-1, 40000, (rows,), generator=gen(seed), device=DEV), normal((40000, 136), seed + 1, 0.2),
            normal((250, 136), seed + 2, 0.1), normal((250, 136), seed + 3, 0.1), torch.zeros(1, dtype=torch.int64, device=DEV))


def same(a, b):
    return all(torch.equal(p.nan_to_num(), q.nan_to_num()) for p, q in zip(a, b))


def test_calls_in_a_graph(pkg):
    """A captured sequence of all calls, replayed on other inputs, gives the bits of the plain calls; a mask that is advanced on
    the device is another one at every replay."""
    data = inputs(1)
    all_calls(pkg, *data)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_calls(pkg, *data)
        data[-1].add_(1)
    masks = []
    for k, seed in enumerate((10, 20, 20)):
        for d, v in zip(data[:-1], inputs(seed)):
            d.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert int(data[-1]) == k + 1
        want = all_calls(pkg, *data[:-1], torch.full((1,), k, dtype=torch.int64, device=DEV))
        torch.cuda.synchronize()
        assert same(held, want)
        masks.append(held[-2].clone())
    assert not torch.equal(masks[1], masks[2])               # the same inputs


def test_calls_from_two_threads(pkg):
    """Two threads, each with inputs and a stream of its own, give the bits of one."""
    data = [inputs(1), inputs(30)]
    want = [all_calls(pkg, *d) for d in data]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                for _ in range(4):
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
    assert all(same(run, want[i]) for i in range(2) for run in got[i])


def test_calls_on_a_named_stream(pkg):
    """stream= another than the current one: results and workspaces belong to it."""
    data = inputs(3)
    want = all_calls(pkg, *data)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):                        # (the inputs' own kernels are over: synchronised)
            got = all_calls(pkg, *data, stream=side)
    side.synchronize()
    assert same(got, want)
    side2 = torch.cuda.Stream()
    r = pkg.gar_linear_logprobs(data[0], data[2], data[1], stream=side2)
    d = pkg.gar_dropout(data[0], 0.3, 5, 7, counter=data[-1], stream=side2)
    side2.synchronize()
    assert torch.equal(r.lse, want[1]) and torch.equal(d, want[-2])


def test_repeated_calls_have_the_same_bits(pkg):
    data = inputs(4)
    want = all_calls(pkg, *data)
    junk = [torch.full((1 << 20,), float("nan"), device=DEV) for _ in range(8)]
    del junk                                                 # memory that the workspaces may get holds NaN
    for _ in range(3):
        assert same(all_calls(pkg, *data), want)


def test_one_workspace_for_call_after_call(pkg):
    """A workspace of the caller's, larger than needed and full of NaN, used by one call after the other."""
    x, t, w, wg, wu, _ = inputs(5)
    t = t.clamp_min(0)
    space = torch.full((64 << 20,), float("nan"), device=DEV).view(torch.uint8)
    r = pkg.gar_linear_logprobs(x, w, t)
    a = torch.rand(x.shape[0], generator=gen(1), device=DEV)
    g0, g1 = (torch.empty(2, w.numel(), device=DEV) for _ in range(2))
    dx = pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=g0)
    assert 0 < pkg.gar_linear_logprobs_workspace_bytes(x, w) <= space.numel()
    assert 0 < pkg.gar_linear_logprobs_backward_workspace_bytes(x, w, g0) <= space.numel()
    exact = torch.empty(pkg.gar_linear_logprobs_backward_workspace_bytes(x, w, g0), dtype=torch.uint8, device=DEV)
    assert torch.equal(pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=g1, workspace=exact), dx) and torch.equal(g0, g1)
    wide = wg[:, 1:]                                         # rows that do not start on 16 bytes are copied
    assert pkg.gar_gated_linear_workspace_bytes(x, wg, wu) == 0 and pkg.gar_gated_linear_workspace_bytes(x[:, 1:], wide, wu[:, 1:]) > 0
    f = pkg.gar_gated_linear_forward("silu", x, wg, wu)
    need = pkg.gar_gated_linear_backward_workspace_bytes(wg, wu, torch.empty_like(f.y), torch.empty_like(f.y))
    own = torch.empty(need, dtype=torch.uint8, device=DEV)
    b0 = pkg.gar_gated_linear_backward("silu", f.y, f.x, f.up, wg, wu)
    b1 = pkg.gar_gated_linear_backward("silu", f.y, f.x, f.up, wg, wu, dgate=torch.empty_like(f.y), dup=torch.empty_like(f.y), workspace=own)
    assert need > 0 and same(b0, b1)
    for _ in range(2):
        assert same(pkg.gar_linear_logprobs(x, w, t, workspace=space), r)
        assert torch.equal(pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=g1, workspace=space), dx) and torch.equal(g0, g1)


def test_refusals(pkg):
    x, t, w, wg, wu, counter = inputs(6)
    r = pkg.gar_linear_logprobs(x, w, t)
    a = torch.ones(x.shape[0], device=DEV)
    f = pkg.gar_gated_linear_forward("silu", x, wg, wu)
    dy = torch.zeros_like(f.y)
    one = x[:1].expand(x.shape)
    space = torch.empty(1 << 10, dtype=torch.uint8, device=DEV)
    block = torch.empty(3, w.numel() + 10, device=DEV)        # 700 rows are no three equal runs
    bad = [(pkg.GarError, lambda: pkg.gar_linear_logprobs(x.float(), w.float(), t)),
           (TypeError, lambda: pkg.gar_linear_logprobs(x, w.half(), t)),
           (ValueError, lambda: pkg.gar_linear_logprobs(x, w[:, :-8], t)),
           (ValueError, lambda: pkg.gar_linear_logprobs(one, w, t)),
           (ValueError, lambda: pkg.gar_linear_logprobs(x.t(), w, t)),
           (TypeError, lambda: pkg.gar_linear_logprobs(x, w, t.int())),
           (TypeError, lambda: pkg.gar_linear_logprobs(x, w, t[:-1])),
           (TypeError, lambda: pkg.gar_linear_logprobs(x, w, t, bias=torch.zeros(40000, device=DEV))),
           (TypeError, lambda: pkg.gar_linear_logprobs(x.cpu(), w, t)),
           (pkg.GarError, lambda: pkg.gar_linear_logprobs(x, w, t, workspace=space)),
           (ValueError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=block)),
           (ValueError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=block[:1], weight_offset=11)),
           (ValueError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=block[:1], bias_offset=w.numel())),
           (ValueError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, bias_offset=0)),
           (pkg.GarError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, dx=False)),
           (pkg.GarError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a, dx=x)),
           (TypeError, lambda: pkg.gar_linear_logprobs_backward(x, w, r, t, a.double())),
           (KeyError, lambda: pkg.gar_gated_linear_forward("tanh", x, wg, wu)),
           (ValueError, lambda: pkg.gar_gated_linear_forward("silu", x, wg, wu[:-1])),
           (ValueError, lambda: pkg.gar_gated_linear_forward("silu", x, wg, wu, group=16)),
           (pkg.GarError, lambda: pkg.gar_gated_linear_forward("silu", x.float(), wg.float(), wu.float())),
           (TypeError, lambda: pkg.gar_gated_linear_backward("silu", dy.half(), f.x, f.up, wg, wu)),
           (ValueError, lambda: pkg.gar_gated_linear_backward("silu", dy, f.x, f.up._replace(group=64), wg, wu)),
           (ValueError, lambda: pkg.gar_gated_linear_backward("silu", dy[:, :-1], f.x, f.up, wg, wu)),
           (pkg.GarError, lambda: pkg.gar_gated_linear_backward("silu", dy, f.x, f.up, wg, wu, dup=dy)),
           (pkg.GarError, lambda: pkg.gar_dropout(x, 1.5, 0)),
           (pkg.GarError, lambda: pkg.gar_dropout(x, -0.1, 0)),
           (OverflowError, lambda: pkg.gar_dropout(x, 0.1, 2 ** 64)),
           (ValueError, lambda: pkg.gar_dropout(one, 0.1, 0)),
           (ValueError, lambda: pkg.gar_dropout(x, 0.1, 0, residual=x[:-1])),
           (TypeError, lambda: pkg.gar_dropout(x, 0.1, 0, counter=counter.int())),
           (pkg.GarError, lambda: pkg.gar_dropout(x[:, 8:], 0.1, 0, y=x[:, :-8]))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")


def test_offsets_near_the_end_of_64_bits_are_refused(pkg):
    x, t, w, wg, wu, counter = inputs(6)
    r = pkg.gar_linear_logprobs(x, w, t)
    a = torch.ones(x.shape[0], device=DEV)
    block = torch.empty(1, w.numel() + w.shape[0], device=DEV)
    saved = pkg.gar_checkpoint_pack(x)
    dy = torch.zeros(1, x.shape[0], 64, dtype=x.dtype, device=DEV)
    far = 2 ** 63 - 1
    for call in (lambda **at: pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=block, **at),
                 lambda **at: pkg.gar_linear_weight_grad(dy, saved, block, **at)):
        for at in (dict(weight_offset=far), dict(weight_offset=far - w.numel()), dict(weight_offset=0, bias_offset=far)):
            with pytest.raises(ValueError):
                call(**at)


def test_written_tensors_count_as_modified(pkg):
    x, t, w, wg, wu, _ = inputs(7)
    f = pkg.gar_gated_linear_forward("silu", x, wg, wu)
    for name, call in (("y", lambda v: pkg.gar_dropout(x, 0.1, 0, y=v)), ("dx", lambda v: pkg.gar_gated_linear_backward("silu", f.y, f.x, f.up, wg, wu, dx=v))):
        v = torch.empty_like(x)
        before = v._version
        call(v)
        assert v._version > before, name


def test_empty_batches(pkg):
    _, _, w, wg, wu, _ = inputs(8)
    x, t, a = normal((0, 136), 1), torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, device=DEV)
    r = pkg.gar_linear_logprobs(x, w, t)
    grads = torch.full((3, w.numel()), 7.0, device=DEV)
    assert pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=grads).shape == (0, 136) and bool((grads == 0).all())
    f = pkg.gar_gated_linear_forward("silu", x, wg, wu)
    assert f.y.shape == (0, 250) and pkg.gar_gated_linear_backward("silu", f.y, f.x, f.up, wg, wu).dx.shape == (0, 136)


def test_offsets_past_32_bits(pkg):
    """A block and a dropout of more than 2^31 elements: what lies past them is the same as in a small call."""
    if torch.cuda.get_device_properties(0).total_memory < 40 << 30:
        pytest.skip("needs 40 GB")
    vocab, hidden, workers, tokens = 70000, 4096, 8, 4
    w = normal((vocab, hidden), 1, 0.02)
    x = normal((workers * tokens, hidden), 2)
    t = torch.randint(0, vocab, (workers * tokens,), generator=gen(3), device=DEV)
    a = -torch.rand(workers * tokens, generator=gen(4), device=DEV)
    r = pkg.gar_linear_logprobs(x, w, t)
    grads = torch.empty(workers, vocab * hidden, dtype=torch.bfloat16, device=DEV)       # 2.3 * 2^30 elements
    dx = pkg.gar_linear_logprobs_backward(x, w, r, t, a, grads=grads)
    last = slice((workers - 1) * tokens, None)
    one = torch.empty(1, vocab * hidden, dtype=torch.bfloat16, device=DEV)
    dx1 = pkg.gar_linear_logprobs_backward(x[last], w, r._replace(lse=r.lse[last].clone(), lse_lo=r.lse_lo[last].clone()), t[last].clone(), a[last].clone(), grads=one)
    assert torch.equal(grads[-1], one[0])
    # 2^-8 twice (dx itself, and a sum cut into other parts) of the terms' size
    assert float((dx[last].double() - dx1.double()).norm()) <= 2.0 ** -7 * float(dx1.double().norm())
    del grads, one, w
    rows, cols = 1 << 16, (1 << 15) + 8
    z = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    y = pkg.gar_dropout(z, 0.5, 9, y=z)
    per = cols // 8
    # the last row's last eight columns, from the generator's definition
    words = philox((rows - 1) * per + per - 1, 0, 9)
    want = [2.0 if ((words[j // 2] >> 16 * (j % 2)) & 0xFFFF) >= 32768 else 0.0 for j in range(8)]
    assert y[-1, -8:].tolist() == want


def philox(block, offset, seed):
    c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c
