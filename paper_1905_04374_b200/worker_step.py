"""A whole training step for n workers on one GPU, some of them Byzantine: the workers' gradients are
computed by the worker-side operators straight into the rows of the n x d block, which is then
aggregated with the SGD step fused into the store.

The model is a classifier of tokens with one hidden layer,
    h = x W1^T + b1,   y = gelu(h),   logits = y W2^T + b2,   loss = mean of -log p(target)
over every worker's own batch.  Between forward and backward pass nothing of the batch is kept but
8-bit checkpoints of x, h and y (and the logits, which become their own gradient in place).

    python -m paper_1905_04374_b200.worker_step [--rule multi_bulyan] [--steps 60]
"""
from __future__ import annotations

import argparse

import torch

from . import worker as W
from .binding import gar_aggregate_ex, new_selection, read_selection


class WorkerStep:
    """Parameters (fp32, one vector of d), their momentum and the n x d gradient block."""

    def __init__(self, n: int, f: int, inputs: int, hidden: int, classes: int, device="cuda", seed: int = 0):
        self.n, self.f = n, f
        self.shapes = {"w1": (hidden, inputs), "b1": (hidden,), "w2": (classes, hidden), "b2": (classes,)}
        self.offsets, d = {}, 0
        for name, shape in self.shapes.items():
            self.offsets[name] = d
            d += torch.Size(shape).numel()
        self.d = d
        gen = torch.Generator(device=device).manual_seed(seed)
        self.params = torch.zeros(d, device=device)
        for name, fan in (("w1", inputs), ("w2", hidden)):
            self.view(name).normal_(0.0, fan ** -0.5, generator=gen)
        self.momentum = torch.zeros(d, device=device)
        self.grads = torch.empty(n, d, device=device)
        self.selection = new_selection(device)

    def view(self, name: str) -> torch.Tensor:
        """One parameter as a matrix or vector."""
        shape = self.shapes[name]
        return self.params[self.offsets[name]:self.offsets[name] + torch.Size(shape).numel()].view(shape)

    def gradients(self, x: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Every worker's gradient into its row of the block; returns the workers' losses [n].
        x: bfloat16 [n, tokens, inputs]; targets: int64 [n, tokens] (negative: no target)."""
        n, tokens, _ = x.shape
        w1, w2 = self.view("w1").to(x.dtype), self.view("w2").to(x.dtype)
        x = x.flatten(0, 1)
        targets = targets.reshape(-1)
        # forward: what the backward pass needs is kept in 8 bits
        x_saved = W.gar_checkpoint_pack(x)
        h = torch.addmm(self.view("b1").to(x.dtype), x, w1.t())
        act = W.gar_activation_forward("gelu", h, save_output=True, y=h)
        logits = torch.addmm(self.view("b2").to(x.dtype), act.y, w2.t())
        scores = W.gar_token_logprobs(logits, targets)
        losses = -scores.logprobs.view(n, tokens).mean(1)
        # backward: the logits become their gradient, the weight gradients go into the block's rows
        up = torch.full((n * tokens,), -1.0 / tokens, device=x.device)
        dlogits = W.gar_token_logprobs_backward(logits, scores, targets, up, dlogits=logits)
        W.gar_linear_weight_grad(dlogits.view(n, tokens, -1), act.out, self.grads, self.offsets["w2"], self.offsets["b2"])
        dy = dlogits @ w2
        dh = W.gar_activation_backward("gelu", dy, act.x, dx=dy).dx
        W.gar_linear_weight_grad(dh.view(n, tokens, -1), x_saved, self.grads, self.offsets["w1"], self.offsets["b1"])
        return losses

    def attack(self, scale: float = -10.0) -> None:
        """The last f workers send the negated, scaled mean of the others' gradients."""
        if self.f:
            self.grads[self.n - self.f:] = scale * self.grads[:self.n - self.f].mean(0)

    def update(self, rule="multi_bulyan", lr: float = 0.1, momentum: float = 0.9) -> None:
        """Aggregates the block and applies the SGD step to the parameters (Eq. 2 and Section 5.1)."""
        gar_aggregate_ex(rule, self.grads, self.f if rule != "average" else 0, selection_out=self.selection, sgd_params=self.params,
                         sgd_momentum_buf=self.momentum, sgd_lr=lr, sgd_momentum=momentum, store_out=False)


def batch(n: int, tokens: int, inputs: int, classes: int, step: int, device="cuda"):
    """A seeded synthetic task: every class is a direction, a token is its class's direction plus noise."""
    centres = torch.randn(classes, inputs, generator=torch.Generator(device=device).manual_seed(7), device=device)
    gen = torch.Generator(device=device).manual_seed(1000 + step)
    targets = torch.randint(0, classes, (n, tokens), generator=gen, device=device)
    x = centres[targets] + 2.0 * torch.randn(n, tokens, inputs, generator=gen, device=device)
    return x.bfloat16(), targets


def train(rule="multi_bulyan", n: int = 11, f: int = 2, steps: int = 60, tokens: int = 128, inputs: int = 256, hidden: int = 512,
          classes: int = 100, attacked: bool = True, device="cuda"):
    """The honest workers' mean loss before every step."""
    model = WorkerStep(n, f, inputs, hidden, classes, device)
    history = []
    for step in range(steps):
        losses = model.gradients(*batch(n, tokens, inputs, classes, step, device))
        history.append(losses[:n - f].mean())
        if attacked:
            model.attack()
        model.update(rule)
    status = read_selection(model.selection).status
    if status != 0:
        raise RuntimeError(f"the last selection reports status {status}")
    return [float(v) for v in history]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rule", default="multi_bulyan", choices=["average", "median", "krum", "multi_krum", "bulyan", "multi_bulyan"])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=11)
    ap.add_argument("--byzantine", type=int, default=2)
    ap.add_argument("--no-attack", action="store_true")
    args = ap.parse_args()
    history = train(args.rule, args.workers, args.byzantine, args.steps, attacked=not args.no_attack)
    for step in sorted({0, len(history) // 4, len(history) // 2, 3 * len(history) // 4, len(history) - 1}):
        print(f"step {step:4d}  loss of the honest workers {history[step]:.4f}")


if __name__ == "__main__":
    main()
