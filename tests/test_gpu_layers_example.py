"""The example that trains a block with the layer operators and the Muon step."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("block,dtype", [("mlp", "bf16"), ("mlp", "f32"), ("moe", "bf16")])
def test_block_learns_and_serves_single_tokens(block, dtype):
    m = _example()
    # an expert sees a quarter of the tokens (2 of 8): more of them, for as many rows per weight
    tokens = {"mlp": "512", "moe": "4096"}[block]
    args = m.parser().parse_args(["--block", block, "--dtype", dtype, "--steps", "40", "--tokens", tokens])
    losses, trained = m.train(args, log=lambda *_: None)
    assert all(v == v for v in losses)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5]), (losses[:5], losses[-5:])
    one, together = m.serve(trained, args)
    # a token alone and in a batch run on different kernels: equal up to rounding
    tol = 2 ** -6 if dtype == "bf16" else 1e-4
    assert torch.allclose(one.float(), together.float(), rtol=tol, atol=tol)
