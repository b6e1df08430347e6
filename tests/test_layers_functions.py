"""The differentiable layer functions without a GPU: what they check themselves
and what they ask of the passes, which are replaced by plain torch ones."""
import pytest
import torch

from paper_2606_27153_amd import layers


@pytest.fixture
def passes(monkeypatch):
    """Plain passes that note how they were called."""
    seen = []

    def linear_forward(x, weight, *, bias=None, residual=None, activation="none", keep_preactivation=False):
        seen.append(("linear_forward", keep_preactivation))
        z = x @ weight if bias is None else x @ weight + bias
        y = torch.relu(z) if activation == "relu" else z
        y = y if residual is None else y + residual
        return (y, z) if keep_preactivation else y

    def linear_backward(dy, x, weight, *, preactivation=None, activation="none", bias_grad=False, input_grad=True,
                        weight_grad=True):
        seen.append(("linear_backward", dy.stride(), dy.data_ptr()))
        dz = dy * (preactivation > 0) if activation == "relu" else dy
        return (dz @ weight.t() if input_grad else None, x.t() @ dz if weight_grad else None,
                dz.sum(0) if bias_grad else None)

    def layer_norm_forward(x, weight=None, bias=None, *, eps=1e-5, keep_stats=False):
        seen.append(("layer_norm_forward", keep_stats))
        mean = x.mean(1)
        rstd = torch.rsqrt(x.var(1, unbiased=False) + eps)
        y = (x - mean[:, None]) * rstd[:, None]
        return (y, mean, rstd) if keep_stats else y

    for f in (linear_forward, linear_backward, layer_norm_forward):
        monkeypatch.setattr(layers, f.__name__, f)
    return seen


def test_linear_refuses_a_residual_of_other_leading_dimensions(passes):
    """As many rows are not enough: with its dimensions swapped, the residual's rows are others."""
    x, w = torch.randn(2, 9, 20), torch.randn(20, 12)
    for shape in ((9, 2, 12), (18, 12), (1, 2, 9, 12), (3, 6, 12), (12,)):
        with pytest.raises(ValueError, match="residual"):
            layers.linear(x, w, residual=torch.randn(shape))
    with pytest.raises(ValueError, match="residual"):
        layers.linear(x.view(18, 20), w, residual=torch.randn(2, 9, 12))
    r = torch.randn(2, 9, 12)
    assert torch.allclose(layers.linear(x, w, residual=r), x @ w + r, atol=1e-5)
    assert layers.linear(x[0, 0], w, residual=r[0, 0]).shape == (12,)
    assert layers.linear(x[:0], w, residual=r[:0]).shape == (0, 9, 12)


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_nothing_is_kept_where_nothing_will_be_differentiated(passes, mode):
    x, w, b = torch.randn(5, 8), torch.nn.Parameter(torch.randn(8, 6)), torch.nn.Parameter(torch.zeros(6))
    n = torch.nn.Parameter(torch.ones(8))
    with mode():
        layers.linear(x, w, b, activation="relu")
        layers.layer_norm(x, n)
    assert passes == [("linear_forward", False), ("layer_norm_forward", False)]
    passes.clear()
    layers.linear(x, w.detach(), residual=torch.zeros(5, 6, requires_grad=True), activation="relu")
    layers.layer_norm(x, n.detach())
    assert passes == [("linear_forward", False), ("layer_norm_forward", False)]
    passes.clear()
    layers.linear(x, w.detach(), b, activation="relu").sum().backward()
    layers.layer_norm(x, n)
    assert [p[:2] for p in passes if "forward" in p[0]] == [("linear_forward", True), ("layer_norm_forward", True)]
    assert b.grad is not None


def test_a_strided_output_gradient_is_taken_as_it_lies(passes):
    """Half of a concatenation's gradient: rows of 6 in rows of 16."""
    x, w = torch.randn(5, 8), torch.randn(8, 6, requires_grad=True)
    other = torch.randn(5, 10)
    g = torch.randn(5, 16)
    torch.cat([layers.linear(x, w), other], dim=1).backward(g)
    assert passes[-1][0] == "linear_backward" and passes[-1][1] == (16, 1)
    assert torch.allclose(w.grad, x.t() @ g[:, :6], atol=1e-5)
    w.grad = None
    layers.linear(x, w).backward(torch.randn(6, 5).t())      # rows that are not contiguous are copied
    assert passes[-1][1] == (6, 1)
    w.grad = None
    layers.linear(x, w).sum().backward()                      # so is an expanded one
    assert passes[-1][1] == (6, 1)
    w.grad = None
    torch.cat([layers.linear(x, w), other[:, :9]], dim=1).backward(torch.randn(5, 15))
    assert passes[-1][1] == (6, 1)                            # and one off 16-byte rows: once, for both products


def test_arguments_that_are_no_tensors_are_type_errors():
    x, w = torch.randn(4, 8), torch.randn(8, 6)
    off = torch.zeros(2, dtype=torch.int32)
    for bad in (None, 3, [[1.0] * 8] * 4, "x"):
        for f in (lambda: layers.linear(bad, w), lambda: layers.layer_norm(bad), lambda: layers.grouped_linear(bad, [w], off),
                  lambda: layers.linear_forward(bad, w), lambda: layers.linear_backward(x, bad, w),
                  lambda: layers.layer_norm_forward(bad), lambda: layers.grouped_linear_forward(bad, [w], off),
                  lambda: layers.linear_forward(x=bad, weight=w),
                  lambda: layers.layer_norm_backward(x, bad, None, x, x)):
            with pytest.raises(TypeError):
                f()
    with pytest.raises(TypeError):
        layers.linear(x, w, residual=[1.0])


def test_inputs_without_features_are_value_errors():
    w = torch.randn(8, 6)
    for bad in (torch.tensor(1.0), torch.zeros(2, 3, 0), torch.zeros(0)):
        with pytest.raises(ValueError):
            layers.linear(bad, w)
        with pytest.raises(ValueError):
            layers.layer_norm(bad)
    with pytest.raises(ValueError):
        layers.linear(torch.zeros(2, 8), torch.tensor(1.0), residual=torch.zeros(2, 1, 6))


def test_strides_of_single_rows_and_columns_do_not_tell_experts_apart():
    x = torch.randn(3, 1)
    ws = [torch.randn(1, 8), torch.randn(1, 16)[:, :8], torch.randn(4, 8)[::4]]
    assert len({w.stride() for w in ws}) > 1
    ptrs, _, transposed, outer, n = layers._experts(ws, x, 1)
    assert ptrs == [w.data_ptr() for w in ws] and (transposed, outer, n) == (0, 8, 3)
    x = torch.randn(3, 8)
    ws = [torch.randn(8, 1), torch.randn(1, 8).t(), torch.randn(1, 16)[:, :8].t()]
    assert len({w.stride() for w in ws}) > 1
    ptrs, ld, transposed, outer, n = layers._experts(ws, x, 8)
    assert ptrs == [w.data_ptr() for w in ws] and (ld, transposed, outer, n) == (1, 0, 1, 3)
    with pytest.raises(ValueError):
        layers._experts([torch.randn(8, 1), torch.randn(8, 2)[:, :1]], x, 8)    # columns of other strides
    with pytest.raises(ValueError):
        layers._experts([torch.randn(8, 6), torch.randn(6, 8).t()], x, 8)
