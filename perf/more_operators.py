"""Cases of a worker's layers: log probabilities of tokens straight from the hidden states (the logits are not kept) with
their gradients, the gated feed-forward block with its gradients, and dropout whose mask is never stored.

`run` computes a case in elementary torch operations in fp32 (own = False) or through the package's entry points
(own = True); `exact` computes it from the definitions in fp64."""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the scores of a handful of next tokens: latency counts, the head's weights are read once
        dict(name="scores_4x32000", op="scores", rows=4, hidden=1024, vocab=32000, dtype="bf16", bias=False, padded=0),
        # evaluation of a batch under a model
        dict(name="scores_8192x32000", op="scores", rows=8192, hidden=2048, vocab=32000, dtype="bf16", bias=False, padded=0),
        # odd sizes, a bias that masks the vocabulary's padding
        dict(name="scores_1000x50001", op="scores", rows=1000, hidden=1000, vocab=50001, dtype="f16", bias=True, padded=81),
        # loss and gradients of the head for eleven workers with short batches
        dict(name="head_11x128_32000x1024", op="head", workers=11, tokens=128, hidden=1024, vocab=32000, dtype="bf16", bias=False),
        # two workers with long batches and a large vocabulary: the products dominate
        dict(name="head_2x2048_131072x4096", op="head", workers=2, tokens=2048, hidden=4096, vocab=131072, dtype="bf16", bias=False),
        # a small classifier's head with bias for eleven workers
        dict(name="head_11x128_100x512", op="head", workers=11, tokens=128, hidden=512, vocab=100, dtype="bf16", bias=True),
        # a large gated block in evaluation: nothing is kept
        dict(name="gated_8192_4096x8192", op="gated", rows=8192, hidden=4096, inner=8192, dtype="bf16", act="silu", bias=False),
        # a small one with odd widths and biases
        dict(name="gated_500_800x2050", op="gated", rows=500, hidden=800, inner=2050, dtype="f16", act="gelu", bias=True),
        # a training step of the block for four workers: forward with everything kept in 8 bits, backward, weight gradients
        dict(name="gated_step_4x2048_4096x8192", op="gated_step", workers=4, tokens=2048, hidden=4096, inner=8192, dtype="bf16",
             act="silu", bias=False, group=128),
        # the same for seven workers with small batches of a small model
        dict(name="gated_step_7x100_500x800", op="gated_step", workers=7, tokens=100, hidden=500, inner=800, dtype="bf16",
             act="gelu", bias=True, group=32),
        # dropout in front of a residual connection, forward and backward
        dict(name="dropout_8192x8192", op="dropout", rows=8192, cols=8192, dtype="bf16", p=0.1, residual=True),
        # odd width, fp32
        dict(name="dropout_333x1001", op="dropout", rows=333, cols=1001, dtype="f32", p=0.5, residual=False),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["scores", "head", "gated", "gated_step", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "dropout":
        cols = _log(rng, 16, 16384)
        rows = _log(rng, 1, (1 << 26) // cols)
        if rng.random() < 0.6 and cols > 64:
            cols -= cols % 64
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["bf16", "f16", "f32"]), p=rng.choice([0.05, 0.1, 0.25, 0.5]),
                    residual=rng.random() < 0.5)
    hidden = _log(rng, 32, 4096)
    wide = _log(rng, 10, 131072 if op in ("scores", "head") else 8192)
    if rng.random() < 0.6:
        hidden, wide = -(-hidden // 64) * 64, -(-wide // 16) * 16
    if op in ("scores", "gated"):
        rows = _log(rng, 1, 8192)
        while rows * hidden * wide > 1 << 39:
            rows = max(1, rows // 2)
        case = dict(op=op, rows=rows, hidden=hidden, dtype=dtype, bias=rng.random() < 0.4)
        if op == "scores":
            return dict(case, vocab=wide, padded=rng.randint(0, wide // 8) if case["bias"] else 0)
        return dict(case, inner=wide, act=rng.choice(["relu", "silu", "gelu"]))
    workers, tokens = rng.randint(1, 16), _log(rng, 1, 2048)
    while workers * hidden * wide > 1 << 29 or workers * tokens * hidden * wide > 1 << 40:
        workers, hidden, wide = max(1, workers // 2), max(32, hidden // 2), max(10, wide // 2)
    case = dict(op=op, workers=workers, tokens=tokens, hidden=hidden, dtype=dtype, bias=rng.random() < 0.4)
    if op == "head":
        return dict(case, vocab=wide)
    return dict(case, inner=wide, act=rng.choice(["relu", "silu", "gelu"]), group=rng.choice([32, 64, 128]))


# ---- inputs -------------------------------------------------------------------------------------
def _normal(shape, scale, dtype, gen):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    return x.normal_(0.0, scale, generator=gen)


def _uniform(shape, gen):
    return torch.rand(shape, generator=gen, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case=case)
    if op == "dropout":
        shape = (case["rows"], case["cols"])
        s["x"], s["dy"] = _normal(shape, 1.0, dtype, gen), _normal(shape, 0.02, dtype, gen)
        s["residual"] = _normal(shape, 1.0, dtype, gen) if case["residual"] else None
        s["key"], s["offset"] = (int(seed) * 0x9E3779B97F4A7C15 + 12345) & 0x7FFFFFFFFFFFFFFF, int(seed) % 1000
        return s
    h = case["hidden"]
    rows = case["rows"] if "rows" in case else case["workers"] * case["tokens"]
    if op in ("scores", "head"):
        vocab, live = case["vocab"], case["vocab"] - case.get("padded", 0)
        # logits of a standard deviation of 2.5, the target's raised as by a model in training
        s["weight"] = w = _normal((vocab, h), 2.5 / math.sqrt(h), dtype, gen)
        s["targets"] = t = torch.randint(0, live, (rows,), generator=gen, device="cuda")
        x = torch.empty(rows, h, device="cuda").normal_(generator=gen)
        at = w[t].float()
        x += (8.0 * _uniform((rows, 1), gen)) * at / at.square().sum(1, keepdim=True).clamp_min(1.0)
        s["x"] = x.to(dtype)
        s["bias"] = None
        if case["bias"]:
            s["bias"] = _normal((vocab,), 0.5, dtype, gen)
            s["bias"][live:] = -math.inf
        t[_uniform((rows,), gen) < 0.1] = -100                # tokens without a target
        if op == "head":
            # the mean loss of each worker's tokens, with the loss scale that training in binary16 takes
            scale = (4096.0 if case["dtype"] == "f16" else 1.0) / case["tokens"]
            s["grad_logprobs"] = -scale * (0.5 + _uniform((rows,), gen))
            s["grads"] = torch.empty(case["workers"], vocab * h + (vocab if case["bias"] else 0), dtype=dtype, device="cuda")
        return s
    f = case["inner"]
    s["x"] = _normal((rows, h), 1.0, dtype, gen)
    s["w_gate"], s["w_up"] = _normal((f, h), 1.5 / math.sqrt(h), dtype, gen), _normal((f, h), 1.0 / math.sqrt(h), dtype, gen)
    s["b_gate"], s["b_up"] = (_normal((f,), 0.2, dtype, gen), _normal((f,), 0.2, dtype, gen)) if case["bias"] else (None, None)
    if op == "gated_step":
        s["dy"] = _normal((rows, f), 0.02, dtype, gen)
        s["grads"] = torch.empty(case["workers"], 2 * f * h + (2 * f if case["bias"] else 0), dtype=dtype, device="cuda")
    return s


# ---- plain forms, fp32 --------------------------------------------------------------------------
def _logits(s):
    z = s["x"].float() @ s["weight"].float().t()
    return z if s["bias"] is None else z + s["bias"].float()


def _scores(s, z):
    t = s["targets"]
    m = z.amax(1, keepdim=True)
    d = z - m
    total = torch.log(torch.exp(d).sum(1))
    picked = torch.gather(d, 1, t.clamp_min(0)[:, None])[:, 0] - total
    return torch.where(t >= 0, picked, torch.zeros_like(picked)), m[:, 0] + total


def _head(s):
    c = s["case"]
    n, tokens, vocab, h = c["workers"], c["tokens"], c["vocab"], c["hidden"]
    t = s["targets"]
    z = _logits(s)
    logprobs, lse = _scores(s, z)
    a = torch.where(t >= 0, s["grad_logprobs"], torch.zeros_like(lse))
    dz = torch.exp(z - lse[:, None]) * -a[:, None]
    dz.scatter_add_(1, t.clamp_min(0)[:, None], a[:, None])
    dx = (dz @ s["weight"].float()).to(s["x"].dtype)
    dz = dz.view(n, tokens, vocab)
    g = s["grads"]
    g[:, :vocab * h] = torch.matmul(dz.transpose(1, 2), s["x"].float().view(n, tokens, h)).reshape(n, vocab * h)
    if c["bias"]:
        g[:, vocab * h:] = dz.sum(1)
    return dict(logprobs=logprobs, dx=dx, grads=g)


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


def _in_8_bits(x, group, dtype):
    """x as its checkpoint restores it: whole steps of a 127th of the largest magnitude of `group` columns, in dtype."""
    rows, cols = x.shape
    groups = -(-cols // group)
    v = torch.zeros(rows, groups * group, dtype=torch.float32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, groups, group)
    amax = v.abs().amax(2, keepdim=True)
    q = torch.round(v * (127.0 / amax.clamp_min(2.0 ** -100)))
    return (q * (amax / 127.0)).view(rows, -1)[:, :cols].to(dtype)


def _projections(s):
    x = s["x"].float()
    g, u = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    return (g, u) if s["b_gate"] is None else (g + s["b_gate"].float(), u + s["b_up"].float())


def _gated_step(s):
    c, dtype = s["case"], s["x"].dtype
    n, tokens, h, f, group = c["workers"], c["tokens"], c["hidden"], c["inner"], c["group"]
    g, u = _projections(s)
    y = (_act(c["act"], g) * u).to(dtype)
    g, u, x = _in_8_bits(g, group, dtype).float(), _in_8_bits(u, group, dtype).float(), _in_8_bits(s["x"].float(), 128, dtype).float()
    dy = s["dy"].float()
    dgate, dup = dy * u * _act_grad(c["act"], g), dy * _act(c["act"], g)
    dx = (dgate @ s["w_gate"].float() + dup @ s["w_up"].float()).to(dtype)
    x, dgate, dup = x.view(n, tokens, h), dgate.view(n, tokens, f), dup.view(n, tokens, f)
    out = s["grads"]
    out[:, :f * h] = torch.matmul(dgate.transpose(1, 2), x).reshape(n, f * h)
    out[:, f * h:2 * f * h] = torch.matmul(dup.transpose(1, 2), x).reshape(n, f * h)
    if c["bias"]:
        out[:, 2 * f * h:2 * f * h + f] = dgate.sum(1)
        out[:, 2 * f * h + f:] = dup.sum(1)
    return dict(y=y, dx=dx, grads=out)


def _draws(rows, cols, key, offset, device):
    """16 bits for every element: Philox 4x32-10 under the 64-bit key, counter (number of the eight columns, offset);
    column j of eight takes half j % 2 of word j // 2."""
    low = 0xFFFFFFFF
    blocks = -(-cols // 8)
    at = torch.arange(rows * blocks, device=device)
    c0, c1 = at & low, at >> 32
    c2, c3 = torch.full_like(at, offset & low), torch.full_like(at, (offset >> 32) & low)
    k0, k1 = key & low, (key >> 32) & low
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).view(rows, blocks * 8)[:, :cols]


def _dropout(s):
    c, dtype = s["case"], s["x"].dtype
    limit = round(c["p"] * 65536)
    keep = _draws(c["rows"], c["cols"], s["key"], s["offset"], s["x"].device) >= limit
    scale = 65536.0 / (65536 - limit)
    y = torch.where(keep, s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(dtype), dx=torch.where(keep, s["dy"].float() * scale, 0.0).to(dtype))


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "scores":
            logprobs, lse = _scores(s, _logits(s))
            return dict(logprobs=logprobs, lse=lse)
        if op == "head":
            return _head(s)
        if op == "gated":
            g, u = _projections(s)
            return dict(y=(_act(c["act"], g) * u).to(s["x"].dtype))
        return _gated_step(s) if op == "gated_step" else _dropout(s)

    import paper_1905_04374_b200 as gar
    if op == "scores":
        r = gar.gar_linear_logprobs(s["x"], s["weight"], s["targets"], bias=s["bias"])
        return dict(logprobs=r.logprobs, lse=r.lse)
    if op == "head":
        r = gar.gar_linear_logprobs(s["x"], s["weight"], s["targets"], bias=s["bias"])
        dx = gar.gar_linear_logprobs_backward(s["x"], s["weight"], r, s["targets"], s["grad_logprobs"], bias=s["bias"], grads=s["grads"],
                                              bias_offset=c["vocab"] * c["hidden"] if c["bias"] else None)
        return dict(logprobs=r.logprobs, dx=dx, grads=s["grads"])
    if op == "gated":
        return dict(y=gar.gar_gated_linear_forward(c["act"], s["x"], s["w_gate"], s["w_up"], s["b_gate"], s["b_up"], save_input=False).y)
    if op == "gated_step":
        n, tokens, h, f = c["workers"], c["tokens"], c["hidden"], c["inner"]
        x = gar.gar_checkpoint_pack(s["x"])
        r = gar.gar_gated_linear_forward(c["act"], s["x"], s["w_gate"], s["w_up"], s["b_gate"], s["b_up"], group=c["group"])
        b = gar.gar_gated_linear_backward(c["act"], s["dy"], r.x, r.up, s["w_gate"], s["w_up"])
        gar.gar_linear_weight_grad(b.dgate.view(n, tokens, f), x, s["grads"], 0, 2 * f * h if c["bias"] else None)
        gar.gar_linear_weight_grad(b.dup.view(n, tokens, f), x, s["grads"], f * h, 2 * f * h + f if c["bias"] else None)
        return dict(y=r.y, dx=b.dx, grads=s["grads"])
    return dict(y=gar.gar_dropout(s["x"], c["p"], s["key"], s["offset"], residual=s["residual"]),
                dx=gar.gar_dropout(s["dy"], c["p"], s["key"], s["offset"]))


def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op == "dropout":
        n = case["rows"] * case["cols"]
        return dict(bytes=(5 if case["residual"] else 4) * n * e, flops=4 * n)
    h = case["hidden"]
    rows = case["rows"] if "rows" in case else case["workers"] * case["tokens"]
    wide = case["vocab"] if "vocab" in case else case["inner"]
    if op == "scores":
        return dict(bytes=(rows * h + wide * (h + case["bias"])) * e + 16 * rows, flops=2 * rows * h * wide)
    if op == "head":
        # the logits, the gradient at the hidden states and the one at the weights
        block = case["workers"] * wide * (h + case["bias"])
        return dict(bytes=(2 * rows * h + wide * (h + case["bias"]) + block) * e + 16 * rows, flops=6 * rows * h * wide)
    weights = 2 * wide * (h + case["bias"])
    if op == "gated":
        return dict(bytes=(rows * (h + wide) + weights) * e, flops=4 * rows * h * wide)
    held = 2 * rows * (wide + 4 * -(-wide // case["group"])) + rows * (h + 4 * -(-h // 128))
    return dict(bytes=(rows * (2 * h + 2 * wide) + weights + case["workers"] * weights) * e + 2 * held, flops=12 * rows * h * wide)


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _exact_head(case, s):
    w, vocab, h = s["weight"].double(), case["vocab"], case["hidden"]
    parts, dxs, rows_out = [], [], []
    workers = case["workers"] if case["op"] == "head" else 1
    tokens = s["x"].shape[0] // workers
    step = max(1, (1 << 27) // vocab)
    for k in range(workers):
        dw = torch.zeros(vocab, h, dtype=torch.float64, device=w.device) if case["op"] == "head" else None
        db = torch.zeros(vocab, dtype=torch.float64, device=w.device)
        for r0 in range(k * tokens, (k + 1) * tokens, step):
            at = slice(r0, min(r0 + step, (k + 1) * tokens))
            x, t = s["x"][at].double(), s["targets"][at]
            z = torch.nn.functional.linear(x, w, None if s["bias"] is None else s["bias"].double())
            lse = torch.logsumexp(z, 1)
            has = t >= 0
            picked = z.gather(1, t.clamp_min(0)[:, None])[:, 0] - lse
            parts.append((torch.where(has, picked, 0.0), lse))
            if case["op"] == "head":
                a = torch.where(has, s["grad_logprobs"][at].double(), 0.0)
                hot = torch.zeros_like(z).scatter_(1, t.clamp_min(0)[:, None], 1.0)
                dz = a[:, None] * (hot - torch.softmax(z, 1))
                dxs.append(dz @ w)
                dw.addmm_(dz.t(), x)
                db += dz.sum(0)
        if case["op"] == "head":
            rows_out.append(torch.cat([dw.view(-1), db]) if case["bias"] else dw.view(-1))
    logprobs, lse = (torch.cat(p) for p in zip(*parts))
    if case["op"] == "scores":
        return dict(logprobs=logprobs, lse=lse)
    return dict(logprobs=logprobs, dx=torch.cat(dxs), grads=torch.stack(rows_out))


def _exact_act(name, x):
    """act(x) and its derivative."""
    if name == "relu":
        return torch.relu(x), torch.where(x > 0, 1.0, 0.0)
    if name == "silu":
        g = torch.sigmoid(x)
        return x * g, g + x * g * torch.sigmoid(-x)
    cdf = 0.5 * torch.erfc(-x / math.sqrt(2.0))
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def _exact_8_bits(x, group, dtype):
    cols = x.shape[1]
    pad = torch.nn.functional.pad(x, (0, -cols % group)).unflatten(1, (-1, group))
    top = pad.abs().max(dim=2, keepdim=True).values
    r = torch.where(top > 0, torch.round(127.0 * pad / top) * top / 127.0, 0.0)
    return r.flatten(1)[:, :cols].to(dtype).double()


def _exact_draws(rows, cols, key, offset):
    """The generator on the host, in numpy's unsigned 64-bit numbers."""
    u = np.uint64
    number = np.arange(rows * -(-cols // 8), dtype=u)
    word = u(0xFFFFFFFF)
    ctr = [number & word, number >> u(32), np.full_like(number, offset & 0xFFFFFFFF), np.full_like(number, offset >> 32)]
    keys = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        a, b = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = [(b >> u(32)) ^ ctr[1] ^ u(keys[0]), b & word, (a >> u(32)) ^ ctr[3] ^ u(keys[1]), a & word]
        keys = [(keys[0] + 0x9E3779B9) % 2 ** 32, (keys[1] + 0xBB67AE85) % 2 ** 32]
    halves = np.stack([h for w in ctr for h in (w & u(0xFFFF), w >> u(16))], axis=1)
    return halves.reshape(rows, -1)[:, :cols].astype(np.int32)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("scores", "head"):
        return _exact_head(case, s)
    if op == "dropout":
        limit = round(case["p"] * 65536)
        keep = torch.from_numpy(_exact_draws(case["rows"], case["cols"], s["key"], s["offset"]) >= limit).to(s["x"].device)
        weight = keep.double() / (1.0 - limit / 65536.0)
        y = weight * s["x"].double()
        return dict(y=y if s["residual"] is None else y + s["residual"].double(), dx=weight * s["dy"].double())
    linear = torch.nn.functional.linear
    x = s["x"].double()
    b_gate, b_up = (None, None) if s["b_gate"] is None else (s["b_gate"].double(), s["b_up"].double())
    w_gate, w_up = s["w_gate"].double(), s["w_up"].double()
    g, u = linear(x, w_gate, b_gate), linear(x, w_up, b_up)
    y = _exact_act(case["act"], g)[0] * u
    if op == "gated":
        return dict(y=y)
    dtype, n = s["x"].dtype, case["workers"]
    g, u, x = _exact_8_bits(g, case["group"], dtype), _exact_8_bits(u, case["group"], dtype), _exact_8_bits(x, 128, dtype)
    value, slope = _exact_act(case["act"], g)
    dy = s["dy"].double()
    dgate, dup = dy * u * slope, dy * value
    rows = []
    for xs, dgs, dus in zip(x.chunk(n), dgate.chunk(n), dup.chunk(n)):
        row = [(dgs.t() @ xs).reshape(-1), (dus.t() @ xs).reshape(-1)]
        if case["bias"]:
            row += [dgs.sum(0), dus.sum(0)]
        rows.append(torch.cat(row))
    return dict(y=y, dx=dgate @ w_gate + dup @ w_up, grads=torch.stack(rows))
