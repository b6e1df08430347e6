"""Trains one transformer feed-forward block on synthetic data with this
library's layer operators, its Muon step and its AdamW step, then serves single tokens.

    python examples/train_block.py --block mlp
    python examples/train_block.py --block moe --experts 8 --top 2 --steps 50

The block is pre-norm: ``x + down(act(up(norm(x))))``, either one MLP (bias and
GELU fused into the first product, bias and the residual into the second) or a
bank of experts (the router's choices sorted by expert, tokens dispatched to their
experts, gate and up projections, SiLU gating, the experts' outputs weighted and
combined with the residual).  It learns to imitate a block of the same kind with
other weights.  ``Muon`` steps the 2-D weights, whose gradients the backward passes
leave in the layout the step reads; ``AdamW`` the norm's and the biases' vectors.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_27153_amd import AdamW, Muon, layers  # noqa: E402


class Mlp(torch.nn.Module):
    def __init__(self, width, hidden, dtype, device):
        super().__init__()
        par = lambda *s, std: torch.nn.Parameter((torch.randn(*s, device=device) * std).to(dtype))
        self.norm_w = torch.nn.Parameter(torch.ones(width, device=device))
        self.norm_b = torch.nn.Parameter(torch.zeros(width, device=device))
        self.up, self.up_b = par(width, hidden, std=width ** -0.5), par(hidden, std=0.0)
        self.down, self.down_b = par(hidden, width, std=hidden ** -0.5), par(width, std=0.0)

    def forward(self, x):
        h = layers.layer_norm(x, self.norm_w, self.norm_b)
        h = layers.linear(h, self.up, self.up_b, activation="gelu_tanh")
        return layers.linear(h, self.down, self.down_b, residual=x)


class Experts(torch.nn.Module):
    """A bank of experts; each expert's weights are matrices of their own, so
    that Muon steps them one by one."""

    def __init__(self, width, hidden, experts, top, dtype, device):
        super().__init__()
        par = lambda *s, std: torch.nn.Parameter((torch.randn(*s, device=device) * std).to(dtype))
        bank = lambda a, b: torch.nn.ParameterList([par(a, b, std=a ** -0.5) for _ in range(experts)])
        self.top = top
        self.norm_w = torch.nn.Parameter(torch.ones(width, device=device))
        self.norm_b = torch.nn.Parameter(torch.zeros(width, device=device))
        self.router = par(width, experts, std=width ** -0.5)
        self.gate, self.up, self.down = bank(width, hidden), bank(width, hidden), bank(hidden, width)

    def forward(self, x):
        h = layers.layer_norm(x, self.norm_w, self.norm_b)
        score = torch.softmax(layers.linear(h, self.router).float(), dim=-1)
        weight, expert = torch.topk(score, self.top, dim=-1)
        # entirely on the GPU: the host never sees which expert has how many rows
        routing = layers.sort_by_expert(expert, len(self.gate))
        rows = layers.dispatch(h, routing)
        g = layers.grouped_linear(rows, list(self.gate), routing.offsets)
        u = layers.grouped_linear(rows, list(self.up), routing.offsets)
        a = (torch.nn.functional.silu(g.float()) * u.float()).to(x.dtype)
        y = layers.grouped_linear(a, list(self.down), routing.offsets)
        return layers.combine(y, weight, routing, residual=x)


def make(args, device):
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[args.dtype]
    if args.block == "mlp":
        return Mlp(args.width, args.hidden, dtype, device)
    return Experts(args.width, args.hidden, args.experts, args.top, dtype, device)


def train(args, log=print):
    """Returns the losses of the steps, and the trained block."""
    device = torch.device("cuda")
    torch.manual_seed(args.seed)
    teacher, block = make(args, device), make(args, device)
    if args.block == "moe":     # the same routing, so that the experts can match one by one
        block.router.data.copy_(teacher.router.data)
    matrices = [p for n, p in block.named_parameters() if p.ndim == 2 and n != "router"]
    vectors = [p for p in block.parameters() if p.ndim == 1]
    opt = Muon(matrices, lr=args.lr, momentum=0.95, weight_decay=0.0)
    adamw = AdamW(vectors, lr=0.1 * args.lr, weight_decay=0.0)
    losses = []
    for step in range(args.steps):
        x = torch.randn(args.tokens, args.width, device=device).to(block.norm_w.dtype if args.dtype == "f32"
                                                                   else torch.bfloat16)
        with torch.no_grad():
            want = teacher(x).float()
        # the residual is the same on both sides
        loss = ((block(x).float() - want) ** 2).mean()
        opt.zero_grad()
        adamw.zero_grad()
        loss.backward()
        scale = 0.5 * (1 + math.cos(math.pi * step / args.steps))
        for o, lr in ((opt, args.lr), (adamw, 0.1 * args.lr)):
            for g in o.param_groups:
                g["lr"] = lr * scale
            o.step()
        losses.append(loss.detach())
        if step % max(1, args.steps // 10) == 0 or step == args.steps - 1:
            log(f"step {step:4d}  loss {float(losses[-1]):.5f}")
    return [float(v) for v in losses], block


def serve(block, args, tokens=4):
    """Single tokens through the trained block: the same operators' few-row form."""
    x = torch.randn(tokens, args.width, device="cuda").to(torch.bfloat16 if args.dtype == "bf16" else torch.float32)
    with torch.no_grad():
        one = torch.cat([block(x[i:i + 1]) for i in range(tokens)])
        return one, block(x)


def parser():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--block", choices=("mlp", "moe"), default="mlp")
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--top", type=int, default=2)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--lr", type=float, default=0.05)
    p.add_argument("--seed", type=int, default=0)
    return p


if __name__ == "__main__":
    a = parser().parse_args()
    losses, trained = train(a)
    one, together = serve(trained, a)
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f}; single tokens against a batch: largest difference "
          f"{float((one.float() - together.float()).abs().max()):.4f}")
