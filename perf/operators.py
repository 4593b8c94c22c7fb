"""Cases of the operators around a worker's gradient: token log probabilities and their gradient, 8-bit activation
checkpoints, the activation's backward pass from them, and the per-worker weight gradients they yield.

`run` computes a case in elementary torch operations in fp32 (own = False) or through the package's entry points
(own = True); `exact` computes it from the definitions in fp64."""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # next-token scores of a handful of sequences, with alternatives shown to a user: latency counts
        dict(name="logprobs_4x32768", op="logprobs", rows=4, vocab=32768, dtype="bf16", top=8, padded=0),
        # the paper's classification tasks (10 classes), the workers' evaluation batches in one call
        dict(name="logprobs_60000x10", op="logprobs", rows=60000, vocab=10, dtype="f32", top=1, padded=0),
        # a language-model batch with a large vocabulary whose last columns are padding (masked)
        dict(name="logprobs_4096x131072", op="logprobs", rows=4096, vocab=131072, dtype="bf16", top=20, padded=72),
        # training: loss and entropy bonus over one micro-batch of every worker, some targets ignored
        dict(name="logprobs_grad_2048x32000", op="logprobs_grad", rows=2048, vocab=32000, dtype="bf16", top=0, padded=0),
        # distillation on the top alternatives, odd vocabulary, fp32 logits
        dict(name="logprobs_grad_300x50001", op="logprobs_grad", rows=300, vocab=50001, dtype="f32", top=5, padded=0),
        # a hidden activation saved after the forward pass and restored for the backward pass
        dict(name="checkpoint_8192x4096", op="checkpoint", rows=8192, cols=4096, dtype="bf16", group=128),
        # odd widths and a fine group, fp32
        dict(name="checkpoint_333x1001", op="checkpoint", rows=333, cols=1001, dtype="f32", group=32),
        # a gated feed-forward block: forward with both inputs kept in 8 bits, backward from them
        dict(name="activation_8192x8192", op="activation", rows=8192, cols=8192, dtype="bf16", act="silu", gated=True,
             group=128, save_output=False),
        # a small plain feed-forward block whose output is kept too (the next layer's input)
        dict(name="activation_500x2050", op="activation", rows=500, cols=2050, dtype="f16", act="gelu", gated=False,
             group=64, save_output=True),
        # a small convolutional network's dense layer (500 x 800) for seven workers, with bias
        dict(name="weight_grad_7x100_500x800", op="weight_grad", workers=7, tokens=100, out=500, inp=800, dtype="bf16",
             grads="f32", bias=True, ragged=True, group=32),
        # eleven workers, short batches: the rows of the gradient block dominate
        dict(name="weight_grad_11x512_4096x4096", op="weight_grad", workers=11, tokens=512, out=4096, inp=4096, dtype="bf16",
             grads="f32", bias=False, ragged=False, group=128),
        # long batches: the products dominate
        dict(name="weight_grad_4x8192_4096x4096", op="weight_grad", workers=4, tokens=8192, out=4096, inp=4096, dtype="bf16",
             grads="bf16", bias=False, ragged=False, group=128),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_grad", "checkpoint", "activation", "weight_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("logprobs", "logprobs_grad"):
        vocab = _log(rng, 10, 131072)
        rows = _log(rng, 1, min(65536, (1 << 28) // vocab))
        if rng.random() < 0.5 and vocab > 64:
            vocab -= vocab % 64
        return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, top=rng.randint(0, min(20, vocab)),
                    padded=rng.randint(0, vocab // 8) if rng.random() < 0.3 else 0)
    if op in ("checkpoint", "activation"):
        cols = _log(rng, 16, 16384)
        rows = _log(rng, 1, (1 << 26) // cols)
        if rng.random() < 0.6 and cols > 64:
            cols -= cols % 64
        case = dict(op=op, rows=rows, cols=cols, dtype=dtype, group=rng.choice([32, 64, 128]))
        if op == "activation":
            case.update(act=rng.choice(["relu", "silu", "gelu"]), gated=rng.random() < 0.5, save_output=rng.random() < 0.3)
        return case
    workers, tokens = rng.randint(1, 16), _log(rng, 1, 4096)
    out, inp = _log(rng, 10, 8192), _log(rng, 10, 8192)
    if rng.random() < 0.6:
        out, inp = -(-out // 16) * 16, -(-inp // 16) * 16
    while workers * out * inp > 11 * 4096 * 4096 or workers * tokens * out * inp > 4 * 8192 * 4096 * 4096:
        out, inp, workers = max(10, out // 2), max(10, inp // 2), max(1, workers // 2)
    return dict(op=op, workers=workers, tokens=tokens, out=out, inp=inp, dtype=rng.choice(["bf16", "f16"]),
                grads=rng.choice(["f32", "f32", "bf16"]), bias=rng.random() < 0.5, ragged=rng.random() < 0.4,
                group=rng.choice([32, 64, 128]))


# ---- inputs -------------------------------------------------------------------------------------
def _normal(shape, scale, dtype, gen):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    return x.normal_(0.0, scale, generator=gen)


def _codes(x, group):
    """The checkpoint of x as its definition gives it: int8 codes [rows, columns rounded up to 16] and fp32 scales."""
    rows, cols = x.shape
    groups = -(-cols // group)
    f = torch.zeros(rows, groups * group, dtype=torch.float32, device=x.device)
    f[:, :cols] = x
    f = f.view(rows, groups, group)
    amax = f.abs().amax(2)
    q = torch.round(f * (127.0 / amax.clamp_min(2.0 ** -100))[:, :, None]).to(torch.int8)
    ld = -(-cols // 16) * 16
    codes = torch.zeros(rows, ld, dtype=torch.int8, device=x.device)
    codes[:, :cols] = q.view(rows, -1)[:, :cols]
    return codes, amax / torch.full_like(amax, 127.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case=case)
    if op in ("logprobs", "logprobs_grad"):
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = x = _normal((rows, vocab), 2.5, dtype, gen)
        live = vocab - case["padded"]
        if live < vocab:
            x[:, live:] = -math.inf
        s["targets"] = t = torch.randint(0, live, (rows,), generator=gen, device="cuda")
        # a model in training: most targets score well above chance
        at = torch.arange(rows, device="cuda")
        x[at, t] += (8.0 * torch.rand(rows, generator=gen, device="cuda")).to(dtype)
        if op == "logprobs_grad":
            t[torch.rand(rows, generator=gen, device="cuda") < 0.1] = -100
            s["grad_logprobs"] = -torch.rand(rows, generator=gen, device="cuda") / rows
            s["grad_entropy"] = torch.full((rows,), 0.01 / rows, device="cuda")
            if case["top"]:
                s["grad_top"] = _normal((rows, case["top"]), 1.0 / rows, torch.float32, gen)
            s["saved"] = _logprobs(x, t, case["top"])
    elif op == "checkpoint":
        s["x"] = _normal((case["rows"], case["cols"]), 1.0, dtype, gen)
    elif op == "activation":
        shape = (case["rows"], case["cols"])
        s["x"] = _normal(shape, 1.5, dtype, gen)
        s["up"] = _normal(shape, 1.0, dtype, gen) if case["gated"] else None
        s["dy"] = _normal(shape, 0.02, dtype, gen)
    else:
        n, t, o, i = case["workers"], case["tokens"], case["out"], case["inp"]
        s["dy"] = _normal((n, t, o), 0.02, dtype, gen)
        s["q"], s["scales"] = _codes(_normal((n * t, i), 1.0, dtype, gen), case["group"])
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, t + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["grads"] = torch.empty(n, o * i + (o if case["bias"] else 0), dtype=DTYPES[case["grads"]], device="cuda")
    return s


# ---- plain forms, fp32 --------------------------------------------------------------------------
def _logprobs(x, t, k):
    x = x.float()
    rows, vocab = x.shape
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(1)
    u = (e * d.clamp_min(-1e4)).sum(1)
    lse = m[:, 0] + torch.log(z)
    entropy = torch.log(z) - u / z
    at = torch.arange(rows, device=x.device)
    logprobs = torch.where(t >= 0, d[at, t.clamp_min(0)] - torch.log(z), torch.zeros_like(z))
    r = dict(logprobs=logprobs, entropy=entropy, lse=lse)
    if k:
        # one whole number for each entry, larger for the larger value, for equal values at the lower index
        b = (x + 0.0).view(torch.int32)
        key = (b ^ ((b >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (vocab - 1 - torch.arange(vocab, device=x.device))
        index = vocab - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
        r["top_logprobs"] = torch.gather(d, 1, index) - torch.log(z)[:, None]
        r["top_index"] = index
    return r


def _logprobs_grad(s):
    x, t, sv = s["logits"].float(), s["targets"], s["saved"]
    lp = x - sv["lse"][:, None]
    p = torch.exp(lp)
    a = torch.where(t >= 0, s["grad_logprobs"], torch.zeros_like(sv["lse"]))
    total = a + s["grad_top"].sum(1) if "grad_top" in s else a
    dx = -p * (total[:, None] + s["grad_entropy"][:, None] * (lp.clamp_min(-1e4) + sv["entropy"][:, None]))
    at = torch.arange(x.shape[0], device=x.device)
    dx[at, t.clamp_min(0)] += a
    if "grad_top" in s:
        dx.scatter_add_(1, sv["top_index"], s["grad_top"])
    return dx.to(s["logits"].dtype)


def _restore(q, scales, cols, group, dtype):
    return (q[:, :cols].float() * scales.repeat_interleave(group, 1)[:, :cols]).to(dtype)


def _act(name, x):
    if name == "relu":
        return x.clamp_min(0.0)
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _act_grad(name, x):
    if name == "relu":
        return (x > 0).to(x.dtype)
    if name == "silu":
        g = 1.0 / (1.0 + torch.exp(-x))
        return g * (1.0 + x * (1.0 - g))
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


def _activation(s):
    c, x, up = s["case"], s["x"], s["up"]
    y = _act(c["act"], x.float())
    if up is not None:
        y = y * up.float()
    r = dict(y=y.to(x.dtype))
    xr = _restore(*_codes(x, c["group"]), c["cols"], c["group"], x.dtype).float()
    dy = s["dy"].float()
    if up is None:
        r["dx"] = (dy * _act_grad(c["act"], xr)).to(x.dtype)
    else:
        ur = _restore(*_codes(up, c["group"]), c["cols"], c["group"], x.dtype).float()
        r["dx"] = (dy * ur * _act_grad(c["act"], xr)).to(x.dtype)
        r["dup"] = (dy * _act(c["act"], xr)).to(x.dtype)
    if c["save_output"]:
        r["y_restored"] = _restore(*_codes(r["y"], c["group"]), c["cols"], c["group"], x.dtype)
    return r


def _weight_grad(s):
    c = s["case"]
    n, t, o, i = c["workers"], c["tokens"], c["out"], c["inp"]
    x = _restore(s["q"], s["scales"], i, c["group"], s["dy"].dtype).float().view(n, t, i)
    dy = s["dy"].float()
    if s["lengths"] is not None:
        dy = torch.where(torch.arange(t, device=dy.device)[None, :, None] < s["lengths"][:, None, None], dy, 0.0)
    g = s["grads"]
    g[:, :o * i] = torch.matmul(dy.transpose(1, 2), x).reshape(n, o * i)
    if c["bias"]:
        g[:, o * i:] = dy.sum(1)
    return dict(grads=g)


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "logprobs":
            return _logprobs(s["logits"], s["targets"], c["top"])
        if op == "logprobs_grad":
            return dict(dlogits=_logprobs_grad(s))
        if op == "checkpoint":
            return dict(restored=_restore(*_codes(s["x"], c["group"]), c["cols"], c["group"], s["x"].dtype))
        return _activation(s) if op == "activation" else _weight_grad(s)

    import paper_1905_04374_b200 as gar
    if op == "logprobs":
        r = gar.gar_token_logprobs(s["logits"], s["targets"], top=c["top"])
        out = dict(logprobs=r.logprobs, entropy=r.entropy, lse=r.lse)
        if c["top"]:
            out.update(top_logprobs=r.top_logprobs, top_index=r.top_index)
        return out
    if op == "logprobs_grad":
        sv = s["saved"]
        saved = gar.TokenLogprobs(sv["logprobs"], sv["entropy"], sv["lse"], sv.get("top_logprobs"), sv.get("top_index"))
        return dict(dlogits=gar.gar_token_logprobs_backward(s["logits"], saved, s["targets"], s["grad_logprobs"],
                                                            s["grad_entropy"], s.get("grad_top")))
    if op == "checkpoint":
        return dict(restored=gar.gar_checkpoint_unpack(gar.gar_checkpoint_pack(s["x"], c["group"])))
    if op == "activation":
        f = gar.gar_activation_forward(c["act"], s["x"], s["up"], group=c["group"], save_output=c["save_output"])
        r = dict(y=f.y)
        b = gar.gar_activation_backward(c["act"], s["dy"], f.x, f.up)
        r["dx"] = b.dx
        if c["gated"]:
            r["dup"] = b.dup
        if c["save_output"]:
            r["y_restored"] = gar.gar_checkpoint_unpack(f.out)
        return r
    ck = gar.Checkpoint(s["q"], s["scales"], c["inp"], c["group"], s["dy"].dtype)
    gar.gar_linear_weight_grad(s["dy"], ck, s["grads"], bias_offset=c["out"] * c["inp"] if c["bias"] else None,
                               lengths=s["lengths"])
    return dict(grads=s["grads"])


def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op in ("logprobs", "logprobs_grad"):
        n, r, k = case["rows"] * case["vocab"], case["rows"], case["top"]
        if op == "logprobs":
            return dict(bytes=n * e + r * (8 + 12) + 12 * r * k, flops=5 * n)
        return dict(bytes=2 * n * e + r * (8 + 16) + 12 * r * k, flops=6 * n)
    if op in ("checkpoint", "activation"):
        n = case["rows"] * case["cols"]
        held = case["rows"] * (case["cols"] + 4 * -(-case["cols"] // case["group"]))
        if op == "checkpoint":
            return dict(bytes=2 * n * e + 2 * held, flops=4 * n)
        inputs = 2 if case["gated"] else 1
        b = (2 * inputs + 2) * n * e + 2 * inputs * held          # x, up, dy read; y, dx, dup written; checkpoints both
        if case["save_output"]:
            b += 2 * held + n * e
        return dict(bytes=b, flops=24 * n * inputs)
    n, t, o, i = case["workers"], case["tokens"], case["out"], case["inp"]
    held = n * t * (i + 4 * -(-i // case["group"]))
    rows = n * (o * i + (o if case["bias"] else 0)) * SIZE[case["grads"]]
    return dict(bytes=n * t * o * e + held + rows, flops=2 * n * t * o * i)


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _exact_restore(x, group):
    """round(127 x / max|group|) max|group| / 127, rounded to x's type, as fp64."""
    rows, cols = x.shape
    pad = torch.nn.functional.pad(x.double(), (0, -cols % group)).unflatten(1, (-1, group))
    top = pad.abs().max(dim=2, keepdim=True).values
    r = torch.where(top > 0, torch.round(127.0 * pad / top) * top / 127.0, 0.0)
    return r.flatten(1)[:, :cols].to(x.dtype).double()


def _exact_act(name, x):
    """act(x) and its derivative."""
    if name == "relu":
        return torch.relu(x), torch.where(x > 0, 1.0, 0.0)
    if name == "silu":
        g = torch.sigmoid(x)
        return x * g, g + x * g * torch.sigmoid(-x)
    cdf = 0.5 * torch.erfc(-x / math.sqrt(2.0))
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("logprobs", "logprobs_grad"):
        parts = []
        step = max(1, (1 << 26) // case["vocab"])
        for r0 in range(0, case["rows"], step):
            x = s["logits"][r0:r0 + step].double()
            t = s["targets"][r0:r0 + step]
            logp = torch.log_softmax(x, 1)
            p = logp.exp()
            entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
            has = (t >= 0).double()
            if op == "logprobs":
                part = dict(logprobs=has * logp.gather(1, t.clamp_min(0)[:, None])[:, 0], entropy=entropy,
                            lse=torch.logsumexp(x, 1))
                if case["top"]:
                    part["top_logprobs"] = logp.topk(case["top"], dim=1).values
            else:
                up = torch.zeros_like(x)                      # the gradient at log_softmax
                up.scatter_add_(1, t.clamp_min(0)[:, None], (has * s["grad_logprobs"][r0:r0 + step].double())[:, None])
                if case["top"]:
                    up.scatter_add_(1, s["saved"]["top_index"][r0:r0 + step], s["grad_top"][r0:r0 + step].double())
                dx = up - p * up.sum(1, keepdim=True)
                c = s["grad_entropy"][r0:r0 + step].double()[:, None]
                part = dict(dlogits=dx - c * torch.where(p > 0, p * (logp + entropy[:, None]), 0.0))
            parts.append(part)
        out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
        if op == "logprobs" and case["top"]:
            out["top_index"] = None
        return out
    if op == "checkpoint":
        return dict(restored=_exact_restore(s["x"], case["group"]))
    if op == "activation":
        dy = s["dy"].double()
        y = _exact_act(case["act"], s["x"].double())[0]
        back, slope = _exact_act(case["act"], _exact_restore(s["x"], case["group"]))
        if case["gated"]:
            y = y * s["up"].double()
            out = dict(y=y, dx=dy * slope * _exact_restore(s["up"], case["group"]), dup=dy * back)
        else:
            out = dict(y=y, dx=dy * slope)
        if case["save_output"]:
            out["y_restored"] = _exact_restore(y.to(s["x"].dtype), case["group"])
        return out
    n, o, i = case["workers"], case["out"], case["inp"]
    rows = []
    for w in range(n):
        t = case["tokens"] if s["lengths"] is None else int(s["lengths"][w])
        at = slice(w * case["tokens"], w * case["tokens"] + t)
        scale = s["scales"][at].double().repeat_interleave(case["group"], 1)[:, :i]
        x = (s["q"][at, :i].double() * scale).to(s["dy"].dtype).double()
        dy = s["dy"][w, :t].double()
        row = [(dy.T @ x).reshape(-1)]
        if case["bias"]:
            row.append(dy.sum(0))
        rows.append(torch.cat(row))
    return dict(grads=torch.stack(rows))
