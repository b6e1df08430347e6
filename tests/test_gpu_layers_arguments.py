"""The layer functions' arguments on the GPU: what is refused, and what is kept
where nothing will be differentiated."""
import pytest
import torch

from paper_2606_27153_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_no_preactivation_is_written_where_no_gradient_will_be_taken(mode):
    x = torch.randn(512, 256, device=DEV).bfloat16()
    w = torch.nn.Parameter(torch.randn(256, 4096, device=DEV).bfloat16())
    y = layers.linear(x, w, activation="silu")
    size = y.numel() * y.element_size()
    with mode():
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = layers.linear(x, w, activation="silu")
        assert torch.cuda.max_memory_allocated() - before < 1.5 * size
    assert not got.requires_grad and torch.equal(got, y)
