"""Trains a small token model from one end to the other with this library's operators:
embedding, MoE blocks, and the loss over a vocabulary whose table both ends share.

    python examples/train_model.py
    python examples/train_model.py --vocab 32000 --width 1024 --layers 2 --steps 50 --state-bits 8

The next token is a fixed function of the one before it, on synthetic sequences.
``Muon`` steps the experts' matrices, ``AdamW`` the table, the routers and the
norms, with states in 32 bits or in 8.  Nothing of a step but its printed loss
comes to the host.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_27153_amd import AdamW, Muon, layers  # noqa: E402
from train_block import Experts  # noqa: E402


class TokenModel(torch.nn.Module):
    def __init__(self, vocab, width, hidden, experts, top, depth, dtype, device):
        super().__init__()
        self.scale = width ** 0.5
        self.table = torch.nn.Parameter((torch.randn(vocab, width, device=device) * width ** -0.5).to(dtype))
        self.blocks = torch.nn.ModuleList([Experts(width, hidden, experts, top, dtype, device) for _ in range(depth)])
        self.norm_w = torch.nn.Parameter(torch.ones(width, device=device))

    def forward(self, ids):
        h = layers.embedding(ids.flatten(), self.table, scale=self.scale)
        for block in self.blocks:
            h = block(h)
        return layers.layer_norm(h, self.norm_w)

    def loss(self, ids, targets):
        return layers.linear_cross_entropy(self(ids), self.table.t(), targets.flatten())

    def optimizers(self, lr, state_bits):
        matrices = [p for b in self.blocks for bank in (b.gate, b.up, b.down) for p in bank]
        stepped = {id(p) for p in matrices}
        rest = [p for p in self.parameters() if id(p) not in stepped]
        return Muon(matrices, lr=lr, momentum=0.95, weight_decay=0.0), \
            AdamW(rest, lr=0.1 * lr, betas=(0.9, 0.95), weight_decay=0.0, state_bits=state_bits)


def batch(args, device):
    """Sequences and their next tokens; the last of each sequence has none."""
    ids = torch.randint(args.vocab, (args.sequences, args.length), device=device)
    targets = (ids * 7 + 3) % args.vocab
    targets[:, -1] = -100
    return ids, targets


def train(args, log=print):
    """Returns the steps' losses and the model."""
    device = torch.device("cuda")
    torch.manual_seed(args.seed)
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[args.dtype]
    model = TokenModel(args.vocab, args.width, args.hidden, args.experts, args.top, args.layers, dtype, device)
    optimizers = model.optimizers(args.lr, args.state_bits)
    losses = []
    for step in range(args.steps):
        loss = model.loss(*batch(args, device))
        for o in optimizers:
            o.zero_grad()
        loss.backward()
        for o in optimizers:
            o.step()
        losses.append(loss.detach())
        if step % max(1, args.steps // 10) == 0 or step == args.steps - 1:
            log(f"step {step:4d}  loss {float(losses[-1]):.5f}")
    return [float(v) for v in losses], model


def parser():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--vocab", type=int, default=1000)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--top", type=int, default=2)
    p.add_argument("--layers", type=int, default=1)
    p.add_argument("--sequences", type=int, default=16)
    p.add_argument("--length", type=int, default=128)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--lr", type=float, default=0.03)
    p.add_argument("--state-bits", type=int, choices=(32, 8), default=32)
    p.add_argument("--seed", type=int, default=0)
    return p


if __name__ == "__main__":
    train(parser().parse_args())
