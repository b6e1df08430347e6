"""The layer operators on the GPU against a plain implementation in 64 bits
(tests/layers_ref.py, which derives the bounds)."""
import ctypes
import importlib.util
import os

import pytest
import torch

import layers_ref as R
from paper_2606_27153_amd import _layers_lib as LL
from paper_2606_27153_amd._lib import MuonError
from paper_2606_27153_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16]
ids = lambda v: str(v).replace("torch.", "")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


# rows x inner x outer: one element, odd ones, exact tiles, one past and one
# short of a tile, long sums with few outputs, the workloads' odd widths
SHAPES = [(1, 1, 1), (3, 7, 13), (1, 64, 256), (1, 1030, 5), (2, 4096, 136), (5, 65, 200), (16, 200, 65), (17, 128, 128),
          (33, 2048, 264), (48, 513, 257), (63, 1152, 96), (64, 64, 64), (65, 256, 768), (129, 257, 513), (127, 136, 1000),
          (300, 1000, 129), (256, 320, 256), (513, 96, 520), (777, 1152, 4304), (1030, 264, 2056), (5000, 40, 24)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_linear_both_passes(shape, dtype):
    rows, inner, outer = shape
    g = gen(rows * 7 + inner)
    act = R.ACTS[(rows + inner + outer) % 5]
    for transposed in (False, True):
        x = rand(g, rows, inner, dtype=dtype)
        w = rand(g, outer, inner, dtype=dtype, scale=inner ** -0.5).t() if transposed else \
            rand(g, inner, outer, dtype=dtype, scale=inner ** -0.5)
        b = rand(g, outer, dtype=dtype) if not transposed or act != "none" else None
        r = rand(g, rows, outer, dtype=dtype) if transposed else None
        y, z = layers.linear_forward(x, w, bias=b, residual=r, activation=act, keep_preactivation=True)
        zr, ez, yr, ey = R.linear_forward(x, w, b, r, act, dtype)
        R.check(y, yr, ey, "y")
        if act != "none":
            R.check(z, zr, ez, "z")
        y1 = layers.linear_forward(x, w, bias=b, residual=r, activation=act)
        assert torch.equal(y, y1)
        dy = rand(g, rows, outer, dtype=dtype)
        dx, dw, db = layers.linear_backward(dy, x, w, preactivation=z, activation=act, bias_grad=True)
        assert dw.stride() == w.stride() or min(w.shape) == 1
        want = R.linear_backward(dy, x, w, z, act, dtype)
        for name, got in (("dx", dx), ("dw", dw), ("db", db)):
            R.check(got, *want[name], f"{name} transposed={transposed}")


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("act", R.ACTS)
def test_linear_epilogue_combinations(act, dtype):
    g = gen(5)
    for rows, inner, outer in ((70, 72, 136), (9, 520, 130)):
        x, w = rand(g, rows, inner, dtype=dtype), rand(g, inner, outer, dtype=dtype, scale=0.3)
        for bias in (False, True):
            for res in (False, True):
                b = rand(g, outer, dtype=dtype) if bias else None
                r = rand(g, rows, outer, dtype=dtype) if res else None
                y, z = layers.linear_forward(x, w, bias=b, residual=r, activation=act, keep_preactivation=True)
                zr, ez, yr, ey = R.linear_forward(x, w, b, r, act, dtype)
                R.check(y, yr, ey, f"y {bias} {res}")
                assert (z is None) == (act == "none")
                if z is not None:
                    R.check(z, zr, ez, "z")
        dy = rand(g, rows, outer, dtype=dtype)
        zin = rand(g, rows, outer, dtype=dtype, scale=3) if act != "none" else None
        want = R.linear_backward(dy, x, w, zin, act, dtype)
        for need in ((True, False, False), (False, True, False), (False, False, True), (True, True, True)):
            got = layers.linear_backward(dy, x, w, preactivation=zin, activation=act, input_grad=need[0],
                                         weight_grad=need[1], bias_grad=need[2])
            for name, t, n in zip(("dx", "dw", "db"), got, need):
                assert (t is not None) == n
                if n:
                    R.check(t, *want[name], name)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows", [1, 20, 200, 600])
def test_linear_strided_and_unaligned_rows(rows, dtype):
    """Slices of wider tensors, at every alignment; outputs of other sizes next to them stay as they are."""
    g = gen(rows)
    for inner, outer, off, pad in ((256, 264, 8, 16), (64, 128, 1, 3), (130, 72, 4, 6), (1024, 520, 3, 8)):
        x = rand(g, rows, inner + pad, dtype=dtype)[:, off:off + inner] if off + inner <= inner + pad else None
        for transposed in (False, True):
            a, b2 = (outer, inner) if transposed else (inner, outer)
            w = rand(g, a + 1, b2 + pad, dtype=dtype, scale=0.1)[1:, off % pad:off % pad + b2]
            w = w.t() if transposed else w
            r = rand(g, rows, outer + pad, dtype=dtype)[:, 1:1 + outer]
            y, z = layers.linear_forward(x, w, residual=r, activation="silu", keep_preactivation=True)
            zr, ez, yr, ey = R.linear_forward(x, w, None, r, "silu", dtype)
            R.check(y, yr, ey, "y")
            dy = rand(g, rows, outer + pad, dtype=dtype)[:, off % pad:off % pad + outer]
            got = layers.linear_backward(dy, x, w, preactivation=z, activation="silu", bias_grad=True)
            want = R.linear_backward(dy, x, w, z, "silu", dtype)
            for name, t in zip(("dx", "dw", "db"), got):
                R.check(t, *want[name], name)


def _call_forward(x, w, y, rows, inner, outer, ldx, ldw, ldy, dtype=1):
    lib = LL.load()
    n = ctypes.c_size_t()
    LL.check(lib.muon_linear_workspace_bytes(rows, inner, outer, dtype, 0, 0, ctypes.byref(n)))
    ws = torch.empty(max(n.value, 256), dtype=torch.uint8, device=DEV)
    LL.check(lib.muon_linear_forward(x, ldx, w, ldw, 0, None, None, 0, y, ldy, None, 0, rows, inner, outer, dtype, 0,
                                     ws.data_ptr(), n.value, torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,inner,outer", [(3, 64, 100), (100, 72, 130), (300, 264, 300)])
def test_linear_writes_its_output_only(rows, inner, outer):
    """The gap between the output's rows, and what lies before and after it, keep their values."""
    g = gen(1)
    x, w = rand(g, rows, inner, dtype=torch.bfloat16), rand(g, inner, outer, dtype=torch.bfloat16)
    for ld, off in ((outer + 12, 8), (outer + 5, 3)):
        buf = torch.full((rows * ld + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
        y = buf[off:off + rows * ld].view(rows, ld)
        _call_forward(x.data_ptr(), w.data_ptr(), y.data_ptr(), rows, inner, outer, inner, outer, ld)
        _, _, yr, ey = R.linear_forward(x, w, None, None, "none", torch.bfloat16)
        R.check(y[:, :outer], yr, ey, "y")
        assert (buf[:off] == 7).all() and (buf[off + rows * ld:] == 7).all() and (y[:, outer:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_linear_residual_in_place(dtype):
    g = gen(3)
    lib = LL.load()
    for rows, inner, outer in ((1, 512, 256), (40, 2048, 72), (300, 96, 264)):
        x, w, r = (rand(g, rows, inner, dtype=dtype), rand(g, inner, outer, dtype=dtype, scale=0.1),
                   rand(g, rows, outer, dtype=dtype))
        want = layers.linear_forward(x, w, residual=r)
        y = r.clone()
        code = 0 if dtype == torch.float32 else 1
        n = ctypes.c_size_t()
        LL.check(lib.muon_linear_workspace_bytes(rows, inner, outer, code, 0, 0, ctypes.byref(n)))
        ws = torch.empty(max(n.value, 256), dtype=torch.uint8, device=DEV)
        LL.check(lib.muon_linear_forward(x.data_ptr(), inner, w.data_ptr(), outer, 0, None, y.data_ptr(), outer,
                                         y.data_ptr(), outer, None, 0, rows, inner, outer, code, 0, ws.data_ptr(),
                                         n.value, torch.cuda.current_stream().cuda_stream))
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_linear_no_rows(dtype):
    x = torch.empty(0, 96, dtype=dtype, device=DEV)
    w = rand(gen(0), 96, 40, dtype=dtype)
    y, z = layers.linear_forward(x, w, activation="gelu", keep_preactivation=True)
    assert y.shape == (0, 40) and z.shape == (0, 40)
    dx, dw, db = layers.linear_backward(y, x, w, preactivation=z, activation="gelu", bias_grad=True)
    assert dx.shape == (0, 96) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,inner,outer", [(6, 96, 40), (70, 100, 90), (300, 264, 520), (260, 65, 300)])
def test_linear_non_finite_values_stay_in_their_rows_and_columns(rows, inner, outer, dtype):
    g = gen(9)
    x, w, dy = (rand(g, rows, inner, dtype=dtype), rand(g, inner, outer, dtype=dtype, scale=0.1),
                rand(g, rows, outer, dtype=dtype))
    clean = layers.linear_forward(x, w)
    cdx, cdw, _ = layers.linear_backward(dy, x, w)
    x2, w2, dy2 = x.clone(), w.clone(), dy.clone()
    x2[rows - 1, inner - 1] = float("nan")
    w2[0, outer - 1] = float("inf")
    y = layers.linear_forward(x2, w2)
    assert torch.equal(y[:-1, :-1], clean[:-1, :-1])
    assert y[-1].isnan().all() and not y[:, -1].isfinite().any()
    dy2[0, 0] = float("-inf")
    dx, dw, _ = layers.linear_backward(dy2, x2, w)
    assert torch.equal(dx[1:], cdx[1:]) and not dx[0].isfinite().any()
    assert torch.equal(dw[:-1, 1:], cdw[:-1, 1:])
    assert not dw[:, 0].isfinite().any() and dw[-1].isnan().all()


@pytest.mark.parametrize("act", R.ACTS[1:])
def test_activations_far_out(act):
    """Values where squares and exponentials overflow: the activation and its slope take their limits."""
    z = torch.tensor([[-3e38, -1e20, -200.0, -88.0, -0.0, 0.0, 88.0, 200.0, 1e20, 3e38]], device=DEV)
    one = torch.ones(1, 1, device=DEV)
    y = layers.linear_forward(one, z, activation=act).cpu().double()
    want = torch.clamp(z, min=0).cpu().double()
    assert ((y - want).abs() <= 1e-30 + 1e-6 * want).all(), y
    dx, dw, db = layers.linear_backward(torch.ones_like(z), one, z, preactivation=z, activation=act, bias_grad=True)
    slope = torch.tensor([[0, 0, 0, 0, 0.5, 0.5, 1, 1, 1, 1.]])
    if act == "relu":
        slope[0, 4:6] = 0
    assert ((dw.cpu() - slope).abs() <= 1e-6).all(), dw
    assert torch.equal(db.cpu(), dw.cpu()[0])


def test_linear_is_deterministic_and_follows_the_stream():
    g = gen(11)
    x, w = rand(g, 200, 4096, dtype=torch.bfloat16), rand(g, 4096, 520, dtype=torch.bfloat16)
    dy = rand(g, 200, 520, dtype=torch.bfloat16)
    first = (layers.linear_forward(x, w), *layers.linear_backward(dy, x, w, bias_grad=True))
    for _ in range(3):
        again = (layers.linear_forward(x, w), *layers.linear_backward(dy, x, w, bias_grad=True))
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-3
        xs = x + (big[:1, :1] * 0).to(x.dtype)   # ready only once the side stream got there
        y = layers.linear_forward(xs, w)
    side.synchronize()
    assert torch.equal(y, first[0])


def test_operators_captured_in_a_graph_match_eager():
    g = gen(12)
    bf = torch.bfloat16
    x, w1, b1 = rand(g, 96, 256, dtype=bf), rand(g, 256, 512, dtype=bf, scale=0.06), rand(g, 512, dtype=bf)
    nw, nb = rand(g, 256), rand(g, 256)
    ws = rand(g, 5, 512, 72, dtype=bf, scale=0.05)
    off = torch.tensor([0, 10, 10, 50, 90, 96], dtype=torch.int32, device=DEV)
    dy = rand(g, 96, 72, dtype=bf)

    def step():
        h, mean, rstd = layers.layer_norm_forward(x, nw, nb, keep_stats=True)
        a, z = layers.linear_forward(h, w1, bias=b1, activation="gelu", keep_preactivation=True)
        y = layers.grouped_linear_forward(a, ws, off)
        da, dws = layers.grouped_linear_backward(dy, a, ws, off)
        dh, dw1, db1 = layers.linear_backward(da, h, w1, preactivation=z, activation="gelu", bias_grad=True)
        return (y, dws, dw1, db1, *layers.layer_norm_backward(dh, x, nw, mean, rstd))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(rand(g, 96, 256, dtype=bf))
        off.copy_(torch.tensor([0, 3 * i, 40, 40 + i, 96 - 7 * i, 96 - i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, step()):
            assert torch.equal(got, want)
        torch.cuda.synchronize()


# ------------------------------------------------------------------ grouped

GROUPED = [  # counts per expert, inner, outer
    ([1], 1, 1), ([0, 0, 3], 7, 13), ([5, 0, 17, 1], 65, 200), ([64, 64], 64, 64), ([0] * 7, 32, 16),
    ([130, 0, 1, 255, 300, 64], 264, 520), ([1] * 48, 256, 136), ([3, 700, 2], 96, 1000), ([40, 90, 513], 513, 257),
    ([int(i % 7 == 0) * i for i in range(200)], 72, 40), ([260, 520, 130, 0, 255], 1152, 264)]


def _offsets(counts, lead=0):
    ends = [lead]
    for c in counts:
        ends.append(ends[-1] + c)
    return ends, torch.tensor(ends, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("case", GROUPED, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[2]}")
def test_grouped_both_passes(case, dtype):
    counts, inner, outer = case
    g = gen(sum(counts) + inner)
    lead, tail = sum(counts) % 3 * 5, sum(counts) % 4 * 9      # rows nobody owns
    ends, off = _offsets(counts, lead)
    rows = ends[-1] + tail
    x, dy = rand(g, rows, inner, dtype=dtype), rand(g, rows, outer, dtype=dtype)
    for transposed in (False, True):
        w = rand(g, len(counts), outer, inner, dtype=dtype, scale=0.1).transpose(1, 2) if transposed else \
            rand(g, len(counts), inner, outer, dtype=dtype, scale=0.1)
        y = layers.grouped_linear_forward(x, w, off)
        dx, dw = layers.grouped_linear_backward(dy, x, w, off)
        assert dw.shape == w.shape
        for t in (y, dx):
            assert (t[:lead] == 0).all() and (t[ends[-1]:] == 0).all()
        for e, n in enumerate(counts):
            a, b = ends[e], ends[e + 1]
            if n == 0:
                assert (dw[e] == 0).all()
                continue
            _, _, yr, ey = R.linear_forward(x[a:b], w[e], None, None, "none", dtype)
            R.check(y[a:b], yr, ey, f"y of expert {e}")
            want = R.linear_backward(dy[a:b], x[a:b], w[e], None, "none", dtype)
            R.check(dx[a:b], *want["dx"], f"dx of expert {e}")
            R.check(dw[e], *want["dw"], f"dw of expert {e}")


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_grouped_weights_as_separate_matrices(dtype):
    g = gen(21)
    counts = [20, 0, 33, 100, 7]
    ends, off = _offsets(counts)
    x, dy = rand(g, ends[-1], 72, dtype=dtype), rand(g, ends[-1], 40, dtype=dtype)
    bank = rand(g, 5, 72, 40, dtype=dtype)
    ws = [bank[i].clone() for i in (0, 1, 2, 3, 4)]
    y = layers.grouped_linear_forward(x, ws, off)
    assert torch.equal(y, layers.grouped_linear_forward(x, bank, off))
    dx, dw = layers.grouped_linear_backward(dy, x, bank, off)
    dx2, dws = layers.grouped_linear_backward(dy, x, ws, off, weight_grad=[True, False, True, True, False])
    assert torch.equal(dx, dx2)
    for i, t in enumerate(dws):
        assert (t is None) == (i in (1, 4))
        if t is not None:
            assert torch.equal(t, dw[i]) and t.is_contiguous()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_grouped_strided_and_unaligned(dtype):
    g = gen(22)
    counts = [20, 0, 33, 200, 7]
    ends, off = _offsets(counts)
    for inner, outer, o, pad in ((64, 72, 8, 16), (100, 130, 1, 3), (264, 33, 2, 4)):
        x = rand(g, ends[-1], inner + pad, dtype=dtype)[:, o:o + inner]
        dy = rand(g, ends[-1], outer + pad, dtype=dtype)[:, o:o + outer]
        w = rand(g, 5, inner, outer + pad, dtype=dtype)[:, :, o:o + outer]
        y = layers.grouped_linear_forward(x, w, off)
        dx, dw = layers.grouped_linear_backward(dy, x, w, off)
        for e, n in enumerate(counts):
            a, b = ends[e], ends[e + 1]
            if n:
                _, _, yr, ey = R.linear_forward(x[a:b], w[e], None, None, "none", dtype)
                R.check(y[a:b], yr, ey, "y")
                want = R.linear_backward(dy[a:b], x[a:b], w[e], None, "none", dtype)
                R.check(dx[a:b], *want["dx"], "dx")
                R.check(dw[e], *want["dw"], "dw")


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("offs", [[50, 10, 30, 100], [-5, 20, 10 ** 9, 60], [0, 64, 64, -(2 ** 31)], [200, 300, 5, 6]],
                         ids=ids)
def test_grouped_offsets_out_of_order_are_clamped(offs, dtype):
    """What such offsets mean is fixed: each counts as the largest so far, within the rows."""
    g = gen(23)
    rows, inner, outer = 128, 40, 72
    x, dy, w = (rand(g, rows, inner, dtype=dtype), rand(g, rows, outer, dtype=dtype),
                rand(g, 3, inner, outer, dtype=dtype))
    top, ends = 0, []
    for v in offs:
        top = max(top, min(max(v, 0), rows))
        ends.append(top)
    bad = torch.tensor(offs, dtype=torch.int32, device=DEV)
    good = torch.tensor(ends, dtype=torch.int32, device=DEV)
    assert torch.equal(layers.grouped_linear_forward(x, w, bad), layers.grouped_linear_forward(x, w, good))
    for a, b in zip(layers.grouped_linear_backward(dy, x, w, bad), layers.grouped_linear_backward(dy, x, w, good)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_grouped_non_finite_rows_stay_with_their_expert(dtype):
    g = gen(24)
    counts = [37, 60, 11, 150]
    ends, off = _offsets(counts)
    x, dy, w = (rand(g, ends[-1], 72, dtype=dtype), rand(g, ends[-1], 136, dtype=dtype),
                rand(g, 4, 72, 136, dtype=dtype))
    y = layers.grouped_linear_forward(x, w, off)
    dx, dw = layers.grouped_linear_backward(dy, x, w, off)
    x2, dy2 = x.clone(), dy.clone()
    x2[37:97] = float("nan")
    dy2[37:97] = float("inf")
    y2 = layers.grouped_linear_forward(x2, w, off)
    dx2, dw2 = layers.grouped_linear_backward(dy2, x2, w, off)
    keep = torch.ones(ends[-1], dtype=torch.bool, device=DEV)
    keep[37:97] = False
    assert torch.equal(y2[keep], y[keep]) and torch.equal(dx2[keep], dx[keep])
    assert all(torch.equal(dw2[e], dw[e]) for e in (0, 2, 3)) and dw2[1].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_grouped_no_rows(dtype):
    x, w = torch.empty(0, 24, dtype=dtype, device=DEV), rand(gen(0), 3, 24, 16, dtype=dtype)
    off = torch.zeros(4, dtype=torch.int32, device=DEV)
    y = layers.grouped_linear_forward(x, w, off)
    dx, dw = layers.grouped_linear_backward(y, x, w, off)
    assert y.shape == (0, 16) and dx.shape == (0, 24) and (dw == 0).all()


# --------------------------------------------------------------- layer norm

NORMS = [(1, 1), (3, 2), (1, 17), (2, 64), (5, 130), (300, 96), (7, 513), (64, 768), (777, 1152), (33, 1408), (4, 2050),
         (20, 4096), (9, 4304), (3, 8191), (5, 14336), (2, 40001), (2000, 8), (4100, 264)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", NORMS, ids=ids)
def test_layer_norm_both_passes(shape, dtype):
    """The bound of the statistics: a mean of n terms is within (n + 2) u mean|x|,
    the variance's sum within (n + 4) u of itself plus the squared error of the
    mean; h, y and dx follow.  The pairwise sums of the kernels are far better
    than n u, so n is taken as at most 64 terms in a row."""
    rows, cols = shape
    g = gen(rows + cols)
    eps = 1e-5
    q = R.ROUND[dtype]
    for wdt, bias in ((dtype, True), (torch.float32, False), (None, False)):
        x = (torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(torch.randn(rows, 1, generator=g, device=DEV))
             + torch.randn(rows, 1, generator=g, device=DEV)).to(dtype)
        w = None if wdt is None else (1 + 0.3 * torch.randn(cols, generator=g, device=DEV)).to(wdt)
        b = torch.randn(cols, generator=g, device=DEV).to(wdt) if bias else None
        y, mean, rstd = layers.layer_norm_forward(x, w, b, eps=eps, keep_stats=True)
        yr, mr, rr, h = R.norm(x, w, b, eps)
        n = 64 * R.U
        em = n * R.f64(x).abs().mean(1)
        R.check(mean, mr, em + 1e-30, "mean")
        er = rr * (n + em * rr) + 1e-30              # relative: half the variance's error, and the mean's
        R.check(rstd, rr, er, "rstd")
        wa = 1.0 if w is None else R.f64(w).abs()
        eh = (em * rr)[:, None] + h.abs() * (er / rr)[:, None] + 4 * R.U * (h.abs() + (mr.abs() * rr)[:, None])
        ey = eh * wa + 4 * R.U * (yr.abs() + (h * wa).abs())
        R.check(y, yr, ey + q * (yr.abs() + ey), "y")
        assert torch.equal(y, layers.layer_norm_forward(x, w, b, eps=eps))
        dy = rand(g, rows, cols, dtype=dtype)
        dx, dw, db = layers.layer_norm_backward(dy, x, w, mean, rstd, bias_grad=True)
        md, rd = R.f64(mean), R.f64(rstd)
        _, _, _, h = R.norm(x, w, b, eps, md, rd)
        d = R.f64(dy)
        gw = d if w is None else d * R.f64(w)
        s1, s2 = gw.mean(1, keepdim=True), (gw * h).mean(1, keepdim=True)
        want = rd[:, None] * (gw - s1 - h * s2)
        eh = 4 * R.U * (h.abs() + (md.abs() * rd)[:, None])
        e1 = n * gw.abs().mean(1, keepdim=True)
        e2 = n * (gw * h).abs().mean(1, keepdim=True) + (gw.abs() * eh).mean(1, keepdim=True)
        e = rd[:, None] * (e1 + h.abs() * e2 + eh * s2.abs() + 4 * R.U * (gw.abs() + s1.abs() + (h * s2).abs()))
        R.check(dx, want, e + q * (want.abs() + e) + 1e-30, "dx")
        wq = R.ROUND[dw.dtype]
        v, e = (d * h).sum(0), (d.abs() * eh).sum(0) + (rows + 8) * R.U * (d * h).abs().sum(0)
        R.check(dw, v, e + wq * (v.abs() + e) + 1e-30, "dw")
        v, e = d.sum(0), (rows + 8) * R.U * d.abs().sum(0)
        R.check(db, v, e + wq * (v.abs() + e) + 1e-30, "db")
        some = layers.layer_norm_backward(dy, x, w, mean, rstd, input_grad=False, bias_grad=False)
        assert some[0] is None and some[2] is None and torch.equal(some[1], dw)
        some = layers.layer_norm_backward(dy, x, w, mean, rstd, weight_grad=False, bias_grad=False)
        assert some[1] is None and some[2] is None and torch.equal(some[0], dx)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("cols,off,pad", [(256, 8, 16), (1152, 1, 3), (130, 2, 4), (4096, 5, 7), (4097, 0, 3)])
def test_layer_norm_strided_and_unaligned_rows(cols, off, pad, dtype):
    g = gen(cols)
    x = rand(g, 37, cols + pad, dtype=dtype)[:, off:off + cols] if off + cols <= cols + pad else None
    dy = rand(g, 37, cols + pad, dtype=dtype)[:, pad - 1:pad - 1 + cols]
    big = rand(g, cols + 3, dtype=dtype)
    w, b = big[1:1 + cols], big[3:3 + cols]
    xc, dyc, wc, bc = x.contiguous(), dy.contiguous(), w.clone(), b.clone()
    got = layers.layer_norm_forward(x, w, b, keep_stats=True)
    for a, c in zip(got, layers.layer_norm_forward(xc, wc, bc, keep_stats=True)):
        assert torch.equal(a, c)
    _, mean, rstd = got
    for a, c in zip(layers.layer_norm_backward(dy, x, w, mean, rstd),
                    layers.layer_norm_backward(dyc, xc, wc, mean, rstd)):
        assert torch.equal(a, c)


def test_layer_norm_rows_far_from_zero_and_constant_rows():
    x = torch.full((2, 1024), 1000.0, device=DEV)
    x[0] += torch.linspace(-1, 1, 1024, device=DEV)
    y, mean, rstd = layers.layer_norm_forward(x, keep_stats=True)
    yr, mr, rr, _ = R.norm(x, None, None, 1e-5)
    # the mean is good to a few u of 1000, h to that over the deviation (0.58)
    assert (R.f64(mean) - mr).abs().max() <= 8 * R.U * 1000
    assert (R.f64(y) - yr)[0].abs().max() <= 16 * R.U * 1000 / 0.58
    assert ((R.f64(rstd) - rr).abs() <= 1e-5 * rr).all()
    assert (y[1] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_layer_norm_non_finite_rows_stay_alone(dtype):
    g = gen(31)
    x, dy, w = rand(g, 50, 264, dtype=dtype), rand(g, 50, 264, dtype=dtype), rand(g, 264, dtype=dtype)
    y, mean, rstd = layers.layer_norm_forward(x, w, keep_stats=True)
    dx, _, _ = layers.layer_norm_backward(dy, x, w, mean, rstd)
    x2 = x.clone()
    x2[7, 3], x2[20, 263] = float("nan"), float("inf")
    y2, m2, r2 = layers.layer_norm_forward(x2, w, keep_stats=True)
    dx2, _, _ = layers.layer_norm_backward(dy, x2, w, m2, r2)
    keep = torch.ones(50, dtype=torch.bool, device=DEV)
    keep[[7, 20]] = False
    assert torch.equal(y[keep], y2[keep]) and torch.equal(dx[keep], dx2[keep])
    assert y2[7].isnan().all() and y2[20].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_layer_norm_no_rows(dtype):
    x, w = torch.empty(0, 24, dtype=dtype, device=DEV), torch.ones(24, dtype=dtype, device=DEV)
    y, mean, rstd = layers.layer_norm_forward(x, w, keep_stats=True)
    dx, dw, db = layers.layer_norm_backward(y, x, w, mean, rstd)
    assert y.shape == (0, 24) and dx.shape == (0, 24) and (dw == 0).all() and (db == 0).all()


# ------------------------------------------------------ offsets past 32 bits

@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_rows_that_lie_past_32_bit_offsets(dtype):
    """Row strides that put later rows past 2^31 elements (and 2^32 bytes)."""
    g = gen(41)
    rows, ld = 5, (1 << 29) + 8
    buf = torch.empty(4 * ld + 4096, dtype=dtype, device=DEV)

    def far(cols, at=0):
        v = buf[at:].as_strided((rows, cols), (ld, 1))
        v.copy_(rand(g, rows, cols, dtype=dtype, scale=0.3))
        return v

    x, dy, w = far(264), far(136, 512), rand(g, 264, 136, dtype=dtype)
    wf = far(136, 1024)    # a weight of 5 far rows
    off = torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV)
    bank = rand(g, 2, 264, 136, dtype=dtype)
    xc, dyc, wfc = x.contiguous(), dy.contiguous(), wf.contiguous()
    x5 = rand(g, 7, 5, dtype=dtype)
    pairs = [(layers.linear_forward(x, w, residual=dy), layers.linear_forward(xc, w, residual=dyc)),
             (layers.linear_forward(x5, wf), layers.linear_forward(x5, wfc)),
             (layers.grouped_linear_forward(x, bank, off), layers.grouped_linear_forward(xc, bank, off))]
    pairs += zip(layers.linear_backward(dy, x, w, preactivation=dy, activation="silu", bias_grad=True),
                 layers.linear_backward(dyc, xc, w, preactivation=dyc, activation="silu", bias_grad=True))
    pairs += zip(layers.grouped_linear_backward(dy, x, bank, off), layers.grouped_linear_backward(dyc, xc, bank, off))
    fwd, fwdc = layers.layer_norm_forward(x, keep_stats=True), layers.layer_norm_forward(xc, keep_stats=True)
    pairs += zip(fwd, fwdc)
    pairs += zip(layers.layer_norm_backward(x, x, None, fwd[1], fwd[2]),
                 layers.layer_norm_backward(xc, xc, None, fwd[1], fwd[2]))
    for a, b in pairs:
        assert torch.allclose(a.float(), b.float(), rtol=2 ** -7 if dtype == torch.bfloat16 else 1e-5, atol=1e-5)
    del buf
    torch.cuda.empty_cache()


# ----------------------------------------------------------------- autograd

def _directional(f, inputs, grads, g):
    """<grad, v> against a central difference of the loss along v, per input."""
    for i, (t, gr) in enumerate(zip(inputs, grads)):
        v = torch.randn(t.shape, generator=g, device=DEV)
        h = 1e-2
        with torch.no_grad():
            up = f(*[u + h * v if j == i else u for j, u in enumerate(inputs)])
            dn = f(*[u - h * v if j == i else u for j, u in enumerate(inputs)])
        diff = float((up - dn) / (2 * h))
        an = float((gr.double() * v.double()).sum())
        scale = float((gr.double() ** 2).sum().sqrt() * (v.double() ** 2).sum().sqrt())
        # a central difference is off by h^2 times the third derivative, and the
        # fp32 loss by its own rounding over 2h
        assert abs(diff - an) <= 2e-3 * scale + 1e-3, (i, diff, an, scale)


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_autograd_of_linear_against_differences(act):
    g = gen(51)
    x, w, b, r = rand(g, 2, 9, 20), rand(g, 20, 12, scale=0.2), rand(g, 12), rand(g, 2, 9, 12)
    c = rand(g, 2, 9, 12)

    def f(x, w, b, r):
        return (layers.linear(x, w, b, activation=act, residual=r).double() * c.double()).sum()

    ins = [t.clone().requires_grad_() for t in (x, w, b, r)]
    _directional(f, [x, w, b, r], torch.autograd.grad(f(*ins), ins), g)


def test_autograd_of_grouped_linear_and_layer_norm_against_differences():
    g = gen(52)
    off = torch.tensor([0, 4, 4, 11, 14], dtype=torch.int32, device=DEV)
    x, w, c = rand(g, 15, 16), rand(g, 4, 16, 10, scale=0.3), rand(g, 15, 10)
    f = lambda x, w: (layers.grouped_linear(x, w, off).double() * c.double()).sum()
    ins = [t.clone().requires_grad_() for t in (x, w)]
    _directional(f, [x, w], torch.autograd.grad(f(*ins), ins), g)
    x, w, b, c = rand(g, 3, 5, 24), rand(g, 24), rand(g, 24), rand(g, 3, 5, 24)
    f = lambda x, w, b: (layers.layer_norm(x, w, b).double() * c.double()).sum()
    ins = [t.clone().requires_grad_() for t in (x, w, b)]
    _directional(f, [x, w, b], torch.autograd.grad(f(*ins), ins), g)


def test_autograd_takes_expanded_gradients_and_transposed_weights():
    """The gradient of a sum is an expanded scalar; a weight kept as [out, in] gets its gradient in that layout."""
    g = gen(53)
    p = rand(g, 40, 24).requires_grad_()          # [out, in]
    x = rand(g, 6, 24).requires_grad_()
    layers.linear(x, p.t()).sum().backward()
    one = torch.ones(6, 40, device=DEV)
    want = R.linear_backward(one, x, p.t(), None, "none", torch.float32)
    R.check(x.grad, *want["dx"], "dx")
    R.check(p.grad.t(), *want["dw"], "dw")
    assert p.grad.is_contiguous()


def test_grouped_autograd_feeds_separate_parameters():
    g = gen(54)
    ws = [rand(g, 16, 24).requires_grad_(i != 1) for i in range(3)]
    x = rand(g, 10, 16).requires_grad_()
    off = torch.tensor([0, 5, 8, 8], dtype=torch.int32, device=DEV)
    layers.grouped_linear(x, ws, off).sum().backward()
    assert ws[1].grad is None and (ws[2].grad == 0).all()
    want = R.linear_backward(torch.ones(5, 24, device=DEV), x[:5], ws[0], None, "none", torch.float32)
    R.check(ws[0].grad, *want["dw"], "dw")
    assert (x.grad[8:] == 0).all()


# ----------------------------------------------------------------- refusals

def test_bad_arguments_are_refused():
    g = gen(61)
    x, w = rand(g, 4, 8), rand(g, 8, 6)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    bank = rand(g, 2, 8, 6)
    bad = [
        lambda: layers.linear_forward(x.cpu(), w.cpu()),
        lambda: layers.linear_forward(x, w.cpu()),
        lambda: layers.linear_forward(x, rand(g, 7, 6)),
        lambda: layers.linear_forward(x, w.bfloat16()),
        lambda: layers.linear_forward(x.t().contiguous().t(), w),
        lambda: layers.linear_forward(x[:1].expand(4, 8), w),
        lambda: layers.linear_forward(x, rand(g, 16, 12)[::2, ::2]),
        lambda: layers.linear_forward(x, w, bias=rand(g, 5)),
        lambda: layers.linear_forward(x, w, bias=rand(g, 12)[::2]),
        lambda: layers.linear_forward(x, w, residual=rand(g, 4, 5)),
        lambda: layers.linear_forward(x, w, activation="tanh"),
        lambda: layers.linear_forward(x, rand(g, 8, 0)),
        lambda: layers.linear_forward(rand(g, 4, 0), rand(g, 0, 6)),
        lambda: layers.linear_forward(rand(g, 8), w),
        lambda: layers.linear_backward(rand(g, 4, 6), x, w, activation="gelu"),
        lambda: layers.linear_backward(rand(g, 4, 7), x, w),
        lambda: layers.grouped_linear_forward(x, bank, off.long()),
        lambda: layers.grouped_linear_forward(x, bank, off[:2]),
        lambda: layers.grouped_linear_forward(x, bank, off.cpu()),
        lambda: layers.grouped_linear_forward(x, [bank[0], rand(g, 8, 7)], off),
        lambda: layers.grouped_linear_forward(x, [], off),
        lambda: layers.grouped_linear_forward(x, rand(g, 300, 8, 6), torch.zeros(301, dtype=torch.int32, device=DEV)),
        lambda: layers.grouped_linear_backward(rand(g, 4, 6), x, bank, off, weight_grad=[True]),
        lambda: layers.layer_norm_forward(x, rand(g, 7)),
        lambda: layers.layer_norm_forward(x, rand(g, 8).bfloat16()),
        lambda: layers.layer_norm_backward(rand(g, 4, 8), x, None, rand(g, 4).double(), rand(g, 4)),
        lambda: layers.layer_norm_backward(rand(g, 4, 8), x, None, rand(g, 3), rand(g, 4)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        layers.linear_forward(x.half(), w.half())
    with pytest.raises(MuonError, match="eps"):
        layers.layer_norm_forward(x, eps=-1.0)
    with pytest.raises(MuonError, match="eps"):
        layers.layer_norm_forward(x, eps=float("nan"))


def test_layer_norm_bias_of_another_dtype_without_a_weight():
    g = gen(71)
    x, b = rand(g, 40, 96, dtype=torch.bfloat16).requires_grad_(), rand(g, 96).requires_grad_()
    c = rand(g, 40, 96, dtype=torch.bfloat16)
    (layers.layer_norm(x, None, b) * c).sum().backward()
    assert b.grad.dtype == torch.float32
    want = R.f64(c).sum(0)
    assert ((R.f64(b.grad) - want).abs() <= 48 * R.U * R.f64(c).abs().sum(0)).all()


def test_operators_take_keywords():
    g = gen(72)
    x, w = rand(g, 3, 16), rand(g, 16, 8)
    y = layers.linear_forward(x=x, weight=w)
    assert torch.equal(y, layers.linear_forward(x, w))
    dx, dw, _ = layers.linear_backward(x=x, dy=y, weight=w)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), layers.linear_backward(y, x, w)[:2]))
    assert torch.equal(layers.layer_norm_forward(weight=None, x=x), layers.layer_norm_forward(x))
