"""The example that trains a token model from one end to the other: it runs, and its
gradients are those of the formulas."""
import importlib.util
import os

import pytest
import torch

import layers_ref as L

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_model", os.path.join(ROOT, "examples", "train_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype,bits", [("bf16", 32), ("bf16", 8), ("f32", 8)])
def test_example_runs(dtype, bits):
    m = _example()
    args = m.parser().parse_args(["--dtype", dtype, "--state-bits", str(bits), "--steps", "6", "--layers", "2"])
    lines = []
    losses, model = m.train(args, log=lines.append)
    assert len(losses) == 6 and all(v == v and abs(v) < 1e4 for v in losses) and lines
    assert all(torch.isfinite(p).all() for p in model.parameters())


def _plain_loss(model, params, ids, targets):
    """The model's loss by plain operations on 64-bit parameters."""
    f = torch.nn.functional
    table = params["table"]
    h = model.scale * table[ids.flatten()]
    for i, block in enumerate(model.blocks):
        q = lambda name: params[f"blocks.{i}.{name}"]
        n = f.layer_norm(h, h.shape[-1:], q("norm_w"), q("norm_b"))
        weight, chosen = torch.topk(torch.softmax(n @ q("router"), -1), block.top, dim=-1)
        out = h
        for e in range(len(block.gate)):
            y = (f.silu(n @ q(f"gate.{e}")) * (n @ q(f"up.{e}"))) @ q(f"down.{e}")
            out = out + y * (weight * (chosen == e)).sum(-1, keepdim=True)
        h = out
    h = f.layer_norm(h, h.shape[-1:], params["norm_w"])
    return f.cross_entropy(h @ table.t(), targets.flatten(), ignore_index=-100)


def test_example_has_the_gradients_of_the_formulas():
    m = _example()
    args = m.parser().parse_args(["--dtype", "f32", "--vocab", "120", "--width", "48", "--hidden", "40", "--layers", "2",
                                  "--sequences", "3", "--length", "21"])
    torch.manual_seed(5)
    model = m.TokenModel(args.vocab, args.width, args.hidden, args.experts, args.top, args.layers, torch.float32,
                         torch.device("cuda"))
    ids, targets = m.batch(args, torch.device("cuda"))
    names, own = zip(*model.named_parameters())
    loss = model.loss(ids, targets)
    got = torch.autograd.grad(loss, own)
    params = {n: p.detach().double().requires_grad_() for n, p in zip(names, own)}
    exact = _plain_loss(model, params, ids, targets)
    want = torch.autograd.grad(exact, list(params.values()))
    assert abs(float(loss) - float(exact)) < 100 * L.U * abs(float(exact))
    # a dozen operators deep, fp32 sums of up to 120 terms each: some thousand roundings of 2^-24 at most
    for n, a, b in zip(names, got, want):
        assert float((a.double() - b).norm()) <= 4000 * L.U * float(b.norm()), n
