"""The layer operators at sizes that fill the chip: every tile kernel, several
tiles per block, split sums, many experts, copies of unaligned operands.  The
reference is the same as in the small tests, computed in 64 bits on the GPU."""
import pytest
import torch

import layers_ref as R
from paper_2606_27153_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _reference_on_the_gpu(monkeypatch):
    monkeypatch.setattr(R, "f64", lambda t: None if t is None else t.detach().double())
    yield
    torch.cuda.empty_cache()


def rand(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


# rows, inner, outer, dtype, activation, transposed: several rounds of 256 x 256
# tiles; 128 x 256 and 128 x 128 ones; a long sum cut into ranges; few columns;
# a weight kept the other way round; odd sizes, whose operands are copied
CASES = [(5832, 1152, 4304, BF, "gelu_tanh", False), (5000, 2048, 5632, BF, "none", True),
         (5832, 4304, 1152, BF, "silu", False), (300, 14336, 1024, BF, "gelu", False),
         (130, 4096, 520, BF, "relu", True), (20000, 256, 72, BF, "none", False), (2500, 1001, 3333, BF, "gelu", False),
         (70, 5000, 4300, BF, "none", True), (2048, 1024, 1152, F32, "silu", False),
         (3001, 515, 1030, F32, "gelu_tanh", True), (400, 4096, 260, F32, "none", False)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v).replace("torch.", "") for v in c))
def test_linear_large(case):
    rows, inner, outer, dtype, act, transposed = case
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + inner)
    x = rand(g, rows, inner, dtype=dtype)
    w = rand(g, outer, inner, dtype=dtype, scale=inner ** -0.5).t() if transposed else \
        rand(g, inner, outer, dtype=dtype, scale=inner ** -0.5)
    b, r, dy = rand(g, outer, dtype=dtype), rand(g, rows, outer, dtype=dtype), rand(g, rows, outer, dtype=dtype)
    y, z = layers.linear_forward(x, w, bias=b, residual=r, activation=act, keep_preactivation=True)
    zr, ez, yr, ey = R.linear_forward(x, w, b, r, act, dtype)
    R.check(y, yr, ey, "y")
    if z is not None:
        R.check(z, zr, ez, "z")
    del zr, ez, yr, ey
    got = layers.linear_backward(dy, x, w, preactivation=z, activation=act, bias_grad=True)
    want = R.linear_backward(dy, x, w, z, act, dtype)
    for name, t in zip(("dx", "dw", "db"), got):
        R.check(t, *want[name], name)
    again = layers.linear_backward(dy, x, w, preactivation=z, activation=act, bias_grad=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("experts,rows,inner,outer,dtype,transposed", [
    (64, 24576, 512, 1408, BF, False), (64, 24576, 1408, 264, BF, True), (8, 9000, 1024, 520, BF, False),
    (64, 1000, 2048, 264, BF, False), (256, 20000, 136, 200, BF, False), (16, 6000, 257, 333, BF, True),
    (16, 3000, 256, 516, F32, False), (7, 2000, 201, 65, F32, True)])
def test_grouped_large(experts, rows, inner, outer, dtype, transposed):
    g = torch.Generator(device=DEV)
    g.manual_seed(experts + rows)
    # uneven shares, a few experts without rows
    share = torch.exp(torch.randn(experts, generator=g, device=DEV))
    share[torch.randperm(experts, generator=g, device=DEV)[:experts // 4]] = 0
    ends = torch.round(torch.cumsum(share, 0) / share.sum() * rows).to(torch.int32)
    off = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), ends])
    off[-1] = rows
    x, dy = rand(g, rows, inner, dtype=dtype), rand(g, rows, outer, dtype=dtype)
    w = rand(g, experts, outer, inner, dtype=dtype, scale=0.1).transpose(1, 2) if transposed else \
        rand(g, experts, inner, outer, dtype=dtype, scale=0.1)
    y = layers.grouped_linear_forward(x, w, off)
    dx, dw = layers.grouped_linear_backward(dy, x, w, off)
    host = off.tolist()
    for e in range(experts):
        a, b = host[e], host[e + 1]
        if a == b:
            assert (dw[e] == 0).all()
            continue
        _, _, yr, ey = R.linear_forward(x[a:b], w[e], None, None, "none", dtype)
        R.check(y[a:b], yr, ey, f"y of expert {e}")
        want = R.linear_backward(dy[a:b], x[a:b], w[e], None, "none", dtype)
        R.check(dx[a:b], *want["dx"], f"dx of expert {e}")
        R.check(dw[e], *want["dw"], f"dw of expert {e}")
    dx2, dw2 = layers.grouped_linear_backward(dy, x, w, off)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_equal_experts_and_all_rows_on_one():
    """Ranks of equal sizes are told apart, and one expert may hold every row."""
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    for experts, n in ((256, 16), (65, 40)):
        x, dy = rand(g, experts * n, 72, dtype=BF), rand(g, experts * n, 136, dtype=BF)
        w = rand(g, experts, 72, 136, dtype=BF)
        for off in (torch.arange(experts + 1, device=DEV) * n, torch.cat([torch.zeros(experts // 2 + 1, device=DEV),
                                                                         torch.full((experts - experts // 2,),
                                                                                    experts * n, device=DEV)])):
            off = off.to(torch.int32)
            dx, dw = layers.grouped_linear_backward(dy, x, w, off)
            host = off.tolist()
            for e in range(experts):
                a, b = host[e], host[e + 1]
                want = R.linear_backward(dy[a:b], x[a:b], w[e], None, "none", BF)
                R.check(dw[e], *want["dw"], f"dw of expert {e}")
                R.check(dx[a:b], *want["dx"], f"dx of expert {e}")


@pytest.mark.parametrize("rows,cols,dtype", [(20000, 1152, BF), (6000, 4096, BF), (9000, 1001, F32), (3000, 6000, F32)])
def test_layer_norm_large(rows, cols, dtype):
    """Many rows per block: against the operator on every row alone, and its column sums in 64 bits."""
    g = torch.Generator(device=DEV)
    g.manual_seed(cols)
    x, dy = rand(g, rows, cols, dtype=dtype), rand(g, rows, cols, dtype=dtype)
    w = (1 + rand(g, cols, scale=0.2)).to(dtype)
    y, mean, rstd = layers.layer_norm_forward(x, w, keep_stats=True)
    dx, dw, db = layers.layer_norm_backward(dy, x, w, mean, rstd)
    for a in (0, rows // 3, rows - 7):
        part = slice(a, a + 7)
        y2, m2, r2 = layers.layer_norm_forward(x[part], w, keep_stats=True)
        assert torch.equal(y[part], y2) and torch.equal(mean[part], m2) and torch.equal(rstd[part], r2)
        assert torch.equal(dx[part], layers.layer_norm_backward(dy[part], x[part], w, m2, r2)[0])
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    q = R.ROUND[dtype]
    for got, terms in ((dw, dy.double() * h), (db, dy.double())):
        want, e = terms.sum(0), (rows + 16) * R.U * terms.abs().sum(0)
        R.check(got, want, e + q * (want.abs() + e), "column sums")


@pytest.mark.parametrize("experts,rows,inner,outer,dtype,transposed", [
    (4, 3, 5632, 4096, F32, False), (8, 345, 14336, 264, BF, False), (8, 345, 4096, 264, F32, True),
    (16, 2, 2257, 727, BF, False), (64, 48, 2048, 1408, BF, True), (2, 30, 8192, 72, BF, False)])
def test_grouped_few_rows_long_sums(experts, rows, inner, outer, dtype, transposed):
    """Sums cut into ranges, whose partial results of all experts' rows are added in one go."""
    test_grouped_large(experts, rows, inner, outer, dtype, transposed)
