"""GPU cases for the kernels that the other layer tests' sizes do not reach: the
fp32 128 x 128 tiles, sums cut into ranges on every tile and grouping
(test_layers_dispatch.py holds these lists and the others' against the kernels
that are reachable at all), and the layer norm's shapes of 1537 to 2048 and of
8193 to 12288 columns.  The same checks as the other tests, in 64 bits on the GPU."""
import pytest
import torch

import layers_ref as R
import test_gpu_layers as small
import test_gpu_layers_large as large

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _reference_on_the_gpu(monkeypatch):
    monkeypatch.setattr(R, "f64", lambda t: None if t is None else t.detach().double())
    yield
    torch.cuda.empty_cache()


# rows, inner, outer, dtype, activation, transposed
LINEAR = [(20, 2048, 1024, BF, "gelu", False), (31, 1024, 2721, F32, "none", False), (30, 2721, 1024, F32, "silu", True),
          (27, 1030, 2050, BF, "relu", True), (3557, 768, 2048, F32, "none", False), (3557, 2048, 768, F32, "silu", True), (64768, 2, 2, F32, "relu", False),
          (1, 13926, 201, F32, "none", True), (24110, 1987, 66, F32, "relu", True), (68, 14336, 4304, F32, "relu", True),
          (505, 14336, 3456, BF, "none", False), (2778, 14336, 1024, BF, "silu", False),
          (9168, 70, 4455, BF, "gelu_tanh", False), (225, 3456, 5632, BF, "relu", True),
          (69, 14336, 5632, BF, "silu", False), (10026, 6858, 76, BF, "silu", True),
          (20148, 9034, 134, BF, "none", False), (21518, 133, 5706, BF, "none", False)]
# experts, rows, inner, outer, dtype, transposed
GROUPED = [(64, 27513, 536, 256, F32, False), (16, 9001, 256, 520, F32, True), (2, 62093, 28, 1, F32, True),
           (3, 3891, 81, 11775, F32, False), (1, 9504, 86, 12785, F32, True), (1, 2, 1271, 2, BF, True),
           (1, 4, 1065, 24, BF, True), (2, 690, 1, 6712, BF, True), (39, 8197, 79, 3512, BF, True),
           (6, 9979, 3810, 75, BF, True), (4, 210, 5632, 4304, BF, True), (13, 288, 2286, 6882, BF, True),
           (4, 2190, 2048, 14336, BF, True), (6, 6354, 14336, 768, BF, True)]


def _name(c):
    return "-".join(str(v).replace("torch.", "") for v in c)


@pytest.mark.parametrize("case", LINEAR, ids=_name)
def test_linear(case):
    large.test_linear_large(case)


@pytest.mark.parametrize("case", GROUPED, ids=_name)
def test_grouped(case):
    large.test_grouped_large(*case)


# 64 threads with four chunks forward, 256 with one and 512 with three backward
@pytest.mark.parametrize("dtype", [F32, BF], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("shape", [(5, 1800), (4000, 2048), (3, 1537), (2, 8193), (1500, 9001), (4, 12288)], ids=str)
def test_layer_norm(shape, dtype):
    small.test_layer_norm_both_passes(shape, dtype)
