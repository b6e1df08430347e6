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


def test_strided_output_gradients_give_the_same_gradients():
    """Halves of a concatenation's gradient, at aligned and unaligned rows, against contiguous ones."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        for rows, inner, outer, wide, act in ((300, 128, 64, 192, "none"), (300, 128, 64, 192, "gelu"),
                                              (70, 65, 33, 40, "none"), (5, 40, 24, 27, "silu")):
            x = torch.randn(rows, inner, generator=g, device=DEV).to(dtype)
            w = torch.randn(inner, outer, generator=g, device=DEV).to(dtype)
            dy = torch.randn(rows, wide, generator=g, device=DEV).to(dtype)
            grads = []
            for d in (dy[:, :outer], dy[:, :outer].clone()):
                xx, ww = x.clone().requires_grad_(), w.clone().requires_grad_()
                layers.linear(xx, ww, activation=act).backward(d)
                grads.append((xx.grad, ww.grad))
            for a, b in zip(*grads):
                assert torch.equal(a, b)


def test_arguments_that_are_no_tensors_are_type_errors():
    x, w, r = torch.randn(4, 8, device=DEV), torch.randn(8, 6, device=DEV), torch.randn(4, device=DEV)
    dy = torch.randn(4, 6, device=DEV)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    for bad in (3, [1.0], "w"):
        for f in (lambda: layers.linear(x, bad), lambda: layers.linear(x, w, bad),
                  lambda: layers.linear(x, w, residual=bad), lambda: layers.linear_forward(x, bad),
                  lambda: layers.linear_forward(x, w, bias=bad), lambda: layers.linear_forward(x, w, residual=bad),
                  lambda: layers.linear_backward(bad, x, w),
                  lambda: layers.linear_backward(dy, x, w, preactivation=bad, activation="silu"),
                  lambda: layers.grouped_linear_forward(x, [w, bad], off),
                  lambda: layers.grouped_linear_forward(x, [bad, w], off),
                  lambda: layers.grouped_linear_forward(x, [w, w], bad),
                  lambda: layers.grouped_linear(x, [bad], off), lambda: layers.grouped_linear(x, bad, off),
                  lambda: layers.grouped_linear(x, [w, w], bad), lambda: layers.layer_norm(x, bad),
                  lambda: layers.grouped_linear_backward(bad, x, [w, w], off),
                  lambda: layers.layer_norm_forward(x, bad), lambda: layers.layer_norm_forward(x, None, bad),
                  lambda: layers.layer_norm_backward(bad, x, None, r, r),
                  lambda: layers.layer_norm_backward(x, x, None, bad, r),
                  lambda: layers.layer_norm_backward(x, x, None, r, bad)):
            with pytest.raises(TypeError):
                f()
    with pytest.raises(TypeError):
        layers.layer_norm_backward(x, x, None, None, r)
    with pytest.raises(TypeError):
        layers.layer_norm_forward(x, eps=None)
