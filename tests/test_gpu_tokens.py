"""The operators that take token or expert numbers on the GPU -- embedding, the
way to the experts and back, the loss over a vocabulary -- against plain ones in 64 bits
(tests/tokens_ref.py, which derives the bounds)."""
import pytest
import torch

import layers_ref as L
import tokens_ref as R
from paper_2606_27153_amd import layers
from paper_2606_27153_amd._lib import MuonError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16]
ids_of = lambda v: str(v).replace("torch.", "")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def numbers(g, n, *shape, dtype=torch.int64, outside=0.0):
    """Numbers below n; a share of them outside of the range, on both sides."""
    v = torch.randint(n, shape, generator=g, device=DEV)
    u = torch.rand(*shape, generator=g, device=DEV)
    far = 1 << 40 if dtype == torch.int64 else 1 << 30
    v = torch.where(u < outside / 2, torch.full_like(v, -1), torch.where(u > 1 - outside / 2, v + n + far, v))
    return v.to(dtype)


def check(got, want, what=""):
    L.check(got, want[0].cpu(), want[1].cpu(), what)


# ---------------------------------------------------------------- embedding

# rows x vocab x cols: one element, odd ones, one block of keys and beyond, two and three digits
EMBEDDINGS = [(1, 1, 1), (3, 5, 7), (0, 9, 8), (64, 1, 40), (65, 3, 130), (500, 513, 33), (777, 70000, 24), (4096, 300, 64),
              (4097, 511, 72), (9000, 512, 8), (5000, 262144, 16), (300, 1000, 2056), (140000, 40, 8)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("shape", EMBEDDINGS, ids=ids_of)
def test_embedding_both_passes(shape, dtype):
    rows, vocab, cols = shape
    g = gen(rows + vocab)
    w = rand(g, vocab, cols, dtype=dtype)
    for number, outside, scale in ((torch.int64, 0.0, 1.0), (torch.int32, 0.2, 5.7)):
        ids = numbers(g, vocab, rows, dtype=number, outside=outside)
        if rows > 600:     # a frequent token: runs of many groups
            ids[100:rows // 2] = vocab // 2
        check(layers.embedding_forward(ids, w, scale=scale), R.embedding_forward(ids, w, scale), "y")
        dy = rand(g, rows, cols, dtype=dtype)
        dw = layers.embedding_backward(dy, ids, vocab, scale=scale)
        check(dw, R.embedding_backward(dy, ids, vocab, scale), "dw")
        assert torch.equal(dw, layers.embedding_backward(dy, ids, vocab, scale=scale))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
def test_embedding_strides_shapes_and_special_values(dtype):
    g = gen(2)
    for cols, off, pad in ((64, 8, 16), (33, 3, 5), (130, 1, 2)):
        w = rand(g, 50, cols + pad, dtype=dtype)[1::2, off % pad:off % pad + cols]
        ids = numbers(g, 25, 2, 3, 7)
        y = layers.embedding_forward(ids, w, scale=0.5)
        assert y.shape == (2, 3, 7, cols)
        check(y, R.embedding_forward(ids, w, 0.5), "y")
        dy = rand(g, 42, cols + pad, dtype=dtype)[:, off % pad:off % pad + cols].view(2, 3, 7, cols)
        check(layers.embedding_backward(dy, ids, 25, scale=0.5), R.embedding_backward(dy, ids, 25, 0.5), "dw")
    # NaN and infinities stay in their rows
    ids = torch.tensor([3, 1, 3, 0], device=DEV)
    dy = torch.ones(4, 8, dtype=dtype, device=DEV)
    dy[0, 2], dy[1, 3] = float("nan"), float("inf")
    dw = layers.embedding_backward(dy, ids, 5).float()
    assert torch.isnan(dw[3, 2]) and torch.isinf(dw[1, 3]) and torch.isfinite(dw).sum() == 5 * 8 - 2
    assert (dw[2] == 0).all() and (dw[4] == 0).all() and (dw[0] == 1).all()


# ------------------------------------------------------------------ routing

# tokens, top, experts, cols
ROUTES = [(1, 1, 1, 1), (5, 2, 3, 7), (0, 2, 4, 8), (8, 6, 64, 256), (33, 8, 256, 40), (100, 3, 7, 333), (683, 6, 64, 72),
          (1366, 3, 5, 16), (3000, 8, 130, 24), (20000, 8, 64, 8), (17, 256, 200, 12)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("case", ROUTES, ids=ids_of)
def test_routing_both_passes(case, dtype):
    tokens, top, experts, cols = case
    g = gen(tokens + top)
    for number, outside in ((torch.int64, 0.0), (torch.int32, 0.3)):
        chosen = numbers(g, experts, tokens, top, dtype=number, outside=outside)
        if experts > 4:
            chosen[chosen == 2] = 3      # an expert without rows, one with twice as many
        routing = layers.sort_by_expert(chosen, experts)
        want = R.route(chosen, experts)
        for got, ref, name in zip(routing, want, ("offsets", "position", "source")):
            assert torch.equal(got.cpu(), ref), name
        position = routing.position
        x = rand(g, tokens, cols, dtype=dtype)
        rows = layers.dispatch_forward(x, routing)
        assert torch.equal(rows, R.dispatch(x, position))
        h = rand(g, tokens * top, cols, dtype=dtype)
        check(layers.dispatch_backward(h, routing), R.gather(h, position), "dx")
        for wdt in {torch.float32, dtype}:
            weights = torch.rand(tokens, top, generator=g, device=DEV).to(wdt)
            for r in (None, rand(g, tokens, cols, dtype=dtype)):
                y = layers.combine_forward(h, weights, routing, residual=r)
                check(y, R.gather(h, position, weights, r), "y")
            dy = rand(g, tokens, cols, dtype=dtype)
            ref = R.combine_backward(dy, h, weights, position)
            drows, dweights = layers.combine_backward(dy, h, weights, routing)
            check(drows, ref["drows"], "drows")
            check(dweights, ref["dweights"], "dweights")
            only = layers.combine_backward(dy, h, weights, routing, rows_grad=False)
            assert only[0] is None and torch.equal(only[1], dweights)
            only = layers.combine_backward(dy, h, weights, routing, weights_grad=False)
            assert only[1] is None and torch.equal(only[0], drows)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
def test_routing_ignores_what_lies_in_rows_of_nobody(dtype):
    g = gen(4)
    chosen = torch.tensor([[0, -1], [9, 2], [-1, -1], [2, 0]], device=DEV)
    routing = layers.sort_by_expert(chosen, 3)
    assert routing.offsets.tolist() == [0, 2, 2, 4]
    h = rand(g, 8, 24, dtype=dtype)
    h[4:] = float("nan")
    w = torch.ones(4, 2, device=DEV)
    w[2] = float("inf")
    y = layers.combine_forward(h, w, routing)
    assert torch.isfinite(y).all() and (y[2] == 0).all() and (layers.dispatch_backward(h, routing)[2] == 0).all()
    dy = rand(g, 4, 24, dtype=dtype)
    dy[2] = float("nan")
    drows, dw = layers.combine_backward(dy, h, w, routing)
    assert torch.isfinite(drows).all() and (drows[4:] == 0).all() and (dw[chosen < 0] == 0).all()
    # rows and choices that sort_by_expert would not give are nobody's either
    wild = routing._replace(position=torch.tensor([[99, -7], [1 << 30, 0], [8, 7], [-1, 3]], dtype=torch.int32, device=DEV),
                            source=torch.tensor([99, -99, 1 << 30, 3, 8, -1, 0, 6], dtype=torch.int32, device=DEV))
    x = rand(g, 4, 24, dtype=dtype)
    rows = layers.dispatch_forward(x, wild)
    assert all(torch.equal(rows[r], x[t]) for r, t in ((0, 1), (7, 2), (3, 3))) and (rows[[1, 5]] == 0).all()
    drows, _ = layers.combine_backward(dy, h, torch.ones_like(w), wild)
    assert (drows[[0, 1, 2, 4, 5]] == 0).all() and all(torch.equal(drows[r], dy[t]) for r, t in ((3, 1), (6, 0), (7, 3)))
    assert torch.equal(layers.dispatch_backward(h, wild)[0], torch.zeros_like(h[0]))


def test_combine_in_place_of_the_residual_and_strided_rows():
    g = gen(6)
    for dtype in DTYPES:
        chosen = numbers(g, 5, 40, 3, outside=0.2)
        routing = layers.sort_by_expert(chosen, 5)
        h = rand(g, 120, 70, dtype=dtype)[:, 3:53]
        r = rand(g, 40, 61, dtype=dtype)[:, 1:51]
        w = torch.rand(40, 3, generator=g, device=DEV)
        check(layers.combine_forward(h, w, routing, residual=r), R.gather(h, routing.position, w, r), "y")
        rows = layers.dispatch_forward(r, routing)
        assert torch.equal(rows, R.dispatch(r, routing.position))


# --------------------------------------------------------------------- loss

# rows x inner x vocab: one element, odd ones, few rows, one past tiles and strips
LOSSES = [(1, 1, 1), (3, 7, 13), (2, 40, 3), (5, 64, 300), (1, 4096, 1000), (16, 200, 65), (33, 72, 4100), (64, 128, 5003),
          (65, 256, 768), (129, 200, 2049), (300, 1000, 129), (257, 72, 4100), (700, 136, 1031), (100, 65, 7),
          (1030, 264, 2056), (18, 824, 4184), (0, 16, 40)]


def loss_case(g, rows, inner, vocab, dtype, transposed, outside=0.1, ignore=-100):
    x = rand(g, rows, inner, dtype=dtype)
    std = 2 * inner ** -0.5
    w = rand(g, vocab, inner, dtype=dtype, scale=std).t() if transposed else rand(g, inner, vocab, dtype=dtype, scale=std)
    t = numbers(g, vocab, rows, outside=outside)
    if rows > 2:
        t[1] = ignore
    return x, w, t


def check_loss(x, w, t, reduction, g, ignore=-100):
    ref = R.Loss(x, w, t, ignore)
    loss, lse = layers.linear_cross_entropy_forward(x, w, t, reduction=reduction, ignore_index=ignore)
    assert loss.dtype == lse.dtype == torch.float32
    check(lse, (ref.lse, ref.lse_error), "lse")
    check(loss, ref.rows() if reduction == "none" else ref.total(reduction), "loss")
    dloss = torch.rand(x.shape[0], generator=g, device=DEV) if reduction == "none" else torch.tensor(1.7, device=DEV)
    dx, dw = layers.linear_cross_entropy_backward(dloss, x, w, t, lse, reduction=reduction, ignore_index=ignore)
    want = ref.backward(dloss, reduction)
    check(dx, want["dx"], "dx")
    check(dw, want["dw"], "dw")
    assert (dx[~ref.live] == 0).all()
    assert dw.stride() == w.stride() or min(w.shape) == 1 or not w.is_contiguous() and not w.t().is_contiguous()
    return dx, dw, lse


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("shape", LOSSES, ids=ids_of)
def test_loss_both_passes(shape, dtype):
    rows, inner, vocab = shape
    g = gen(rows * 3 + inner)
    for i, transposed in enumerate((False, True)):
        x, w, t = loss_case(g, rows, inner, vocab, dtype, transposed)
        reduction = ("mean", "none", "sum")[(rows + inner + i) % 3]
        dx, dw, lse = check_loss(x, w, t.int() if i and vocab < 1 << 20 else t, reduction, g)
        if reduction != "none":
            one = torch.tensor(1.7, device=DEV)
            only = layers.linear_cross_entropy_backward(one, x, w, t, lse, reduction=reduction, weight_grad=False)
            assert only[1] is None and torch.equal(only[0], dx)
            only = layers.linear_cross_entropy_backward(one, x, w, t, lse, reduction=reduction, input_grad=False)
            assert only[0] is None and torch.equal(only[1], dw)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("rows", [1, 20, 200])
def test_loss_strided_and_unaligned_rows(rows, dtype):
    g = gen(rows)
    for inner, vocab, off, pad in ((256, 264, 8, 16), (64, 128, 1, 3), (130, 72, 4, 6), (72, 2100, 3, 8)):
        x = rand(g, rows, inner + pad, dtype=dtype)[:, off % pad:off % pad + inner]
        for transposed in (False, True):
            a, b = (vocab, inner) if transposed else (inner, vocab)
            w = rand(g, a + 1, b + pad, dtype=dtype, scale=0.1)[1:, off % pad:off % pad + b]
            w = w.t() if transposed else w
            t = numbers(g, vocab, rows, outside=0.2)
            check_loss(x, w, t, "none" if transposed else "mean", g, ignore=vocab // 2)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
def test_loss_without_targets_and_with_extreme_logits(dtype):
    g = gen(9)
    for rows, vocab in ((4, 50), (80, 300)):
        x, w, t = loss_case(g, rows, 40, vocab, dtype, False)
        for reduction in ("mean", "sum", "none"):
            none = torch.full_like(t, -100)
            loss, lse = layers.linear_cross_entropy_forward(x, w, none, reduction=reduction)
            assert (loss == 0).all() and torch.isfinite(lse).all()
            d = torch.ones_like(loss)
            dx, dw = layers.linear_cross_entropy_backward(d, x, w, none, lse, reduction=reduction)
            assert (dx == 0).all() and (dw == 0).all()
        # logits of thousands: the largest alone counts, nothing overflows
        big = x * 300
        ref = R.Loss(big, w, t)
        loss, lse = layers.linear_cross_entropy_forward(big, w, t, reduction="none")
        check(lse, (ref.lse, ref.lse_error), "lse")
        check(loss, ref.rows(), "loss")
        # a row of NaN without a target leaves the others and the weight's gradient alone
        t[2] = -100
        nan = x.clone()
        nan[2] = float("nan")
        loss, lse = layers.linear_cross_entropy_forward(nan, w, t)
        assert torch.isfinite(loss)
        dx, dw = layers.linear_cross_entropy_backward(torch.ones((), device=DEV), nan, w, t, lse)
        assert (dx[2] == 0).all() and torch.isfinite(dx).all()
        # an infinite gradient and a weight that is not finite leave such rows' gradients alone too
        inf = torch.full((), float("inf"), device=DEV)
        w9 = w.clone()
        w9[3, 7] = float("nan")
        for weight, d in ((w, inf), (w9, inf / inf)):
            dx, _ = layers.linear_cross_entropy_backward(d, x, weight, t, lse.nan_to_num())
            live = (t >= 0) & (t < vocab)
            assert (dx[~live] == 0).all() and not torch.isfinite(dx[live]).all(1).any()
        # -inf columns (a vocabulary masked through its weight) have probability 0
        x1 = torch.cat([x.abs(), torch.ones(rows, 8, device=DEV, dtype=dtype)], 1)
        w1 = torch.cat([w, torch.zeros(8, vocab, device=DEV, dtype=dtype)])
        w1[40, 5:9] = float("-inf")
        t1 = torch.where((t >= 5) & (t < 9), 1, t)
        loss, lse = layers.linear_cross_entropy_forward(x1, w1, t1, reduction="none")
        keep = torch.tensor([v for v in range(vocab) if not 5 <= v < 9], device=DEV)
        ref = R.Loss(x1, w1[:, keep], torch.where(t1 >= 9, t1 - 4, t1))
        check(lse, (ref.lse, ref.lse_error), "lse")
        check(loss, ref.rows(), "loss")


# rows, inner, vocab, transposed, dtype: more rows than a forward pass takes at once, more
# columns than a piece has, copied weights, every kernel that can be chosen
LARGE = [(33000, 24, 600, False, torch.bfloat16), (20000, 64, 40000, True, torch.bfloat16),
         (100, 72, 50001, False, torch.bfloat16), (70, 16, 270000, True, torch.float32),
         (9, 16, 270001, False, torch.bfloat16), (300, 40, 66001, False, torch.float32),
         (133, 6785, 32000, False, torch.bfloat16), (19791, 152, 6489, True, torch.bfloat16),
         (11428, 129, 12292, True, torch.bfloat16), (194, 3352, 13208, False, torch.bfloat16),
         (1982, 130, 28296, True, torch.bfloat16), (70, 2905, 15745, False, torch.float32),
         (17716, 2048, 83, False, torch.float32), (72, 2642, 13695, False, torch.bfloat16),
         (6504, 83, 3995, True, torch.float32), (13735, 2535, 70, True, torch.bfloat16),
         (270, 2, 32000, False, torch.bfloat16), (16687, 3, 281, True, torch.bfloat16),
         (54548, 160, 3, False, torch.bfloat16), (9283, 1159, 1, True, torch.bfloat16),
         (67, 8, 34914, True, torch.bfloat16), (19461, 175, 1, True, torch.bfloat16),
         (12031, 258, 1, False, torch.bfloat16), (12628, 221, 1, True, torch.float32),
         (64672, 2, 4, False, torch.bfloat16), (17, 15, 1274, True, torch.bfloat16),
         (18, 8, 1247, False, torch.bfloat16), (19, 8, 570, True, torch.float32),
         (19, 1024, 8, False, torch.bfloat16), (17, 5, 593, False, torch.float32), (19, 513, 4, True, torch.float32),
         (17, 563, 4, False, torch.float32), (41, 9, 1, False, torch.bfloat16), (34, 11, 1, True, torch.bfloat16),
         (33, 5, 1, True, torch.float32), (36, 4, 1, False, torch.float32), (19, 9, 1, True, torch.bfloat16)]


@pytest.mark.parametrize("case", LARGE, ids=ids_of)
def test_loss_large(case):
    rows, inner, vocab, transposed, dtype = case
    g = gen(11)
    x, w, t = loss_case(g, rows, inner, vocab, dtype, transposed)
    check_loss(x, w, t, "mean", g)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("rows", [1, 3, 4, 5, 8, 9, 16, 17, 32, 33])
def test_loss_of_few_rows(rows, dtype):
    """Whose weight gradient is an outer product: every number of rows that a kernel is made for."""
    g = gen(rows + 70)
    for i, (inner, vocab, pad) in enumerate(((37, 1031, 0), (264, 40, 0), (1, 3, 0), (2056, 7, 0), (40, 2056, 3), (33, 31, 1))):
        x = rand(g, rows, inner + pad, dtype=dtype)[:, :inner]
        for transposed in (False, True):
            a, b = (vocab, inner) if transposed else (inner, vocab)
            w = rand(g, a, b + pad, dtype=dtype, scale=0.1)[:, :b]
            w = w.t() if transposed else w
            check_loss(x, w, numbers(g, vocab, rows, outside=0.2), ("mean", "none", "sum")[i % 3], g, ignore=vocab // 2)


def test_loss_rows_far_apart():
    """Rows 2^23 bytes or more apart are copied before the kernels' 32-bit offsets reach them."""
    g = gen(13)
    buf = torch.empty(70 * (1 << 22) + 64, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((70, 64), (1 << 22, 1))
    x.copy_(rand(g, 70, 64))
    w = rand(g, 64, 300, dtype=torch.bfloat16, scale=0.2)
    t = numbers(g, 300, 70)
    check_loss(x, w, t, "mean", g)
    wide = buf.as_strided((64, 300), (1 << 22, 1))
    wide.copy_(w)
    check_loss(rand(g, 70, 64, dtype=torch.bfloat16), wide, t, "none", g)
    del buf, x, wide
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("cols", [1023, 1024])
def test_lookups_of_many_bytes(cols, dtype):
    """Outputs of more than 64 MB are stored by another kernel: exact, row by row."""
    g = gen(cols)
    rows = (1 << 26) // (cols * dtype.itemsize) + 2
    w = rand(g, 50, cols, dtype=dtype)
    ids = numbers(g, 50, rows, outside=0.1)
    y = layers.embedding_forward(ids, w, scale=0.5)
    live = (ids >= 0) & (ids < 50)
    assert torch.equal(y, torch.where(live[:, None], w[ids.clamp(0, 49)] * 0.5, torch.zeros_like(y)))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("shape", [(1, 8, 9), (5, 24, 40), (40, 33, 257), (300, 264, 1000)], ids=ids_of)
def test_loss_rows_without_a_target_may_hold_anything(shape, dtype):
    """(As the rows of a padded batch do: results are those of zeros in their place.)"""
    rows, inner, vocab = shape
    g = gen(rows)
    for transposed in (False, True):
        x, w, t = loss_case(g, rows, inner, vocab, dtype, transposed)
        t[::3] = -100
        t[1::5] = vocab + 3
        dead = (t < 0) | (t >= vocab)
        zeros, bad = x.clone(), x.clone()
        zeros[dead] = 0
        bad[dead] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e38], device=DEV).to(dtype).repeat(inner)[:inner]
        for reduction in ("mean", "sum", "none"):
            out = []
            for v in (zeros, bad):
                loss, lse = layers.linear_cross_entropy_forward(v, w, t, reduction=reduction)
                d = torch.full_like(loss, 0.7)
                if reduction == "none":
                    d[dead] = float("nan")
                out.append((loss, *layers.linear_cross_entropy_backward(d, v, w, t, lse, reduction=reduction)))
            for a, b in zip(*out):
                assert torch.isfinite(a).all() and torch.equal(a, b)


# ----------------------------------------------------- autograd and together

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
        # off by h^2 times the third derivative, and the fp32 loss by its own rounding over 2h
        assert abs(diff - an) <= 2e-3 * scale + 1e-3, (i, diff, an, scale)


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd_of_the_loss_against_differences(reduction):
    g = gen(31)
    x, w = rand(g, 2, 9, 20), rand(g, 20, 37, scale=0.3)
    t = numbers(g, 37, 2, 9, outside=0.2)
    c = torch.rand(2, 9, generator=g, device=DEV)

    def f(x, w):
        loss = layers.linear_cross_entropy(x, w, t, reduction=reduction)
        assert loss.shape == (t.shape if reduction == "none" else ())
        return (loss.double() * (c.double() if reduction == "none" else 3.0)).sum()

    ins = [v.clone().requires_grad_() for v in (x, w)]
    _directional(f, [x, w], torch.autograd.grad(f(*ins), ins), g)


def test_autograd_of_embedding_and_routing_against_differences():
    g = gen(32)
    ids, c = numbers(g, 11, 3, 5, outside=0.2), rand(g, 3, 5, 16)
    f = lambda w: (layers.embedding(ids, w, scale=1.5).double() * c.double()).sum()
    w = rand(g, 11, 16)
    leaf = w.clone().requires_grad_()
    _directional(f, [w], torch.autograd.grad(f(leaf), [leaf]), g)
    routing = layers.sort_by_expert(numbers(g, 4, 9, 3, outside=0.2), 4)
    c = rand(g, 9, 16)
    x, p, r = rand(g, 9, 16), torch.rand(9, 3, generator=g, device=DEV), rand(g, 9, 16)

    def route(x, p, r):
        rows = layers.dispatch(x, routing)
        return (layers.combine(rows * rows, p, routing, residual=r).double() * c.double()).sum()

    ins = [v.clone().requires_grad_() for v in (x, p, r)]
    _directional(route, [x, p, r], torch.autograd.grad(route(*ins), ins), g)


def test_gradients_only_where_they_are_wanted_and_expanded_ones():
    g = gen(33)
    x, w = rand(g, 6, 24).requires_grad_(), rand(g, 40, 24)
    t = numbers(g, 40, 6)
    layers.linear_cross_entropy(x, w.t(), t, reduction="none").sum().backward()     # an expanded gradient
    want = R.Loss(x.detach(), w.t(), t).backward(torch.ones(6, device=DEV), "none")
    check(x.grad, want["dx"], "dx")
    table = w.clone().requires_grad_()
    layers.linear_cross_entropy(x.detach(), table.t(), t).backward()
    assert table.grad.is_contiguous()
    check(table.grad.t(), R.Loss(x.detach(), w.t(), t).backward(torch.ones((), device=DEV), "mean")["dw"], "dw")
    with torch.no_grad():
        assert not layers.linear_cross_entropy(x, table.t(), t).requires_grad
    routing = layers.sort_by_expert(numbers(g, 3, 6, 2), 3)
    rows = layers.dispatch(x, routing)
    p = torch.rand(6, 2, generator=g, device=DEV, requires_grad=True)
    layers.combine(rows.detach(), p, routing).sum().backward()
    assert p.grad is not None
    layers.embedding(t, table).sum().backward()


def _model(table, norm, bank, router, ids, targets, ops):
    """A token model of one MoE layer, tied ends: its loss.  ops: the library's operators, or plain ones."""
    h = ops.embedding(ids, table, 4.0)
    n = ops.norm(h, norm)
    scores = torch.softmax((n @ router).float() if ops is Own else n @ router, -1)
    weight, chosen = torch.topk(scores, 2, dim=-1)
    h = ops.experts(n, h, weight, chosen, bank)
    return ops.loss(ops.norm(h, norm), table, targets)


class Own:
    embedding = staticmethod(lambda ids, table, s: layers.embedding(ids, table, scale=s))
    norm = staticmethod(lambda x, w: layers.layer_norm(x, w))
    loss = staticmethod(lambda x, table, t: layers.linear_cross_entropy(x, table.t(), t))

    @staticmethod
    def experts(n, h, weight, chosen, bank):
        routing = layers.sort_by_expert(chosen, len(bank))
        rows = layers.grouped_linear(layers.dispatch(n, routing), list(bank), routing.offsets)
        return layers.combine(rows, weight, routing, residual=h)


class Plain:
    embedding = staticmethod(lambda ids, table, s: s * table[ids])
    norm = staticmethod(lambda x, w: torch.nn.functional.layer_norm(x, x.shape[-1:], w))
    loss = staticmethod(lambda x, table, t: torch.nn.functional.cross_entropy(x @ table.t(), t, ignore_index=-100))

    @staticmethod
    def experts(n, h, weight, chosen, bank):
        out = h
        for j in range(chosen.shape[1]):
            out = out + weight[:, j, None] * torch.stack([n[i] @ bank[int(e)] for i, e in enumerate(chosen[:, j])])
        return out


def test_a_model_of_them_together_has_the_gradients_of_the_formulas():
    g = gen(34)
    tokens, width, vocab, experts = 60, 40, 90, 5
    ids, targets = numbers(g, vocab, tokens), numbers(g, vocab, tokens)
    targets[::7] = -100
    leaves = [rand(g, vocab, width, scale=0.3), 1 + rand(g, width, scale=0.1),
              *[rand(g, width, width, scale=0.2) for _ in range(experts)], rand(g, width, experts, scale=0.5)]

    def grads(ops, cast):
        t = [cast(v).requires_grad_() for v in leaves]
        loss = _model(t[0], t[1], t[2:-1], t[-1], ids, targets, ops)
        return [loss, *torch.autograd.grad(loss, t)]

    got, want = grads(Own, lambda v: v.clone()), grads(Plain, lambda v: v.double())
    # chains of fp32 sums of up to 90 terms, a handful deep: some hundred roundings of 2^-24
    for a, b in zip(got, want):
        assert float((a.detach().double() - b.detach()).norm() / b.detach().norm()) < 1000 * L.U


# ------------------------------------------------------------ graphs, streams

def test_operators_captured_in_a_graph_match_eager_and_other_streams():
    g = gen(41)
    rows, width, vocab = 200, 136, 3000
    x, w = rand(g, rows, width, dtype=torch.bfloat16), rand(g, vocab, width, dtype=torch.bfloat16, scale=0.1)
    ids = numbers(g, vocab, rows)
    chosen = numbers(g, 9, rows, 4, outside=0.1)
    p = torch.rand(rows, 4, generator=g, device=DEV)
    one = torch.ones((), device=DEV)

    def work():
        y = layers.embedding_forward(ids, w, scale=2.0)
        dw = layers.embedding_backward(x, ids, vocab)
        routing = layers.sort_by_expert(chosen, 9)
        h = layers.dispatch_forward(x, routing)
        out = layers.combine_forward(h, p, routing, residual=x)
        dh, dp = layers.combine_backward(x, h, p, routing)
        dx = layers.dispatch_backward(dh, routing)
        loss, lse = layers.linear_cross_entropy_forward(x, w.t(), ids)
        return [y, dw, *routing, h, out, dh, dp, dx, loss, lse,
                *layers.linear_cross_entropy_backward(one, x, w.t(), ids, lse)]

    work()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):     # two graphs of the same operators, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = work()
        graphs.append((graph, out))
    side = torch.cuda.Stream()
    for k in range(4):
        x.copy_(rand(g, rows, width))
        ids.copy_(numbers(g, vocab, rows, outside=0.1))
        chosen.copy_(numbers(g, 9, rows, 4, outside=0.1))
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        with torch.cuda.stream(side):
            want = work()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_operators_take_keywords():
    g = gen(42)
    x, w = rand(g, 5, 16), rand(g, 16, 30)
    t = numbers(g, 30, 5)
    loss, lse = layers.linear_cross_entropy_forward(targets=t, weight=w, x=x)
    assert torch.equal(lse, layers.linear_cross_entropy_forward(x, w, t)[1])
    d = torch.ones((), device=DEV)
    assert torch.equal(layers.linear_cross_entropy_backward(lse=lse, targets=t, weight=w, x=x, dloss=d)[0],
                       layers.linear_cross_entropy_backward(d, x, w, t, lse)[0])
    assert torch.equal(layers.embedding_forward(weight=w, ids=t % 16), layers.embedding_forward(t % 16, w))
    assert torch.equal(layers.embedding_backward(vocab=9, ids=t, dy=x), layers.embedding_backward(x, t, 9))
    r = layers.sort_by_expert(count=3, experts=t[:, None] % 3)
    assert torch.equal(layers.dispatch_forward(routing=r, x=x), layers.dispatch_forward(x, r))
    p = torch.ones(5, 1, device=DEV)
    assert torch.equal(layers.combine_forward(routing=r, weights=p, rows=x), layers.combine_forward(x, p, r))


# ----------------------------------------------------------------- refusals

def test_bad_arguments_are_refused():
    g = gen(61)
    x, w, t = rand(g, 4, 8), rand(g, 8, 6), numbers(g, 6, 4)
    r = layers.sort_by_expert(t[:, None], 6)
    p = torch.ones(4, 1, device=DEV)
    f, b = layers.linear_cross_entropy_forward, layers.linear_cross_entropy_backward
    lse, one = torch.zeros(4, device=DEV), torch.ones((), device=DEV)
    bad = [
        lambda: f(x.cpu(), w.cpu(), t.cpu()), lambda: f(x, w, t.cpu()), lambda: f(x, w, t[:3]), lambda: f(x, w, t[:, None]),
        lambda: f(x, rand(g, 7, 6), t), lambda: f(x, w.bfloat16(), t), lambda: f(x, w, t, reduction="max"),
        lambda: f(x, rand(g, 8, 0), t), lambda: f(x, w, torch.stack([t, t], 1)[:, 0]),
        lambda: b(one, x, w, t, lse[:3]), lambda: b(one, x, w, t, lse.double()), lambda: b(lse, x, w, t, lse),
        lambda: b(one, x, w, t, lse, reduction="none"), lambda: b(one.cpu(), x, w, t, lse),
        lambda: layers.linear_cross_entropy(x, w, t.view(2, 2)),
        lambda: layers.embedding_forward(t, x.cpu()), lambda: layers.embedding_forward(t.cpu(), x),
        lambda: layers.embedding_forward(t, x[0]), lambda: layers.embedding_forward(t, rand(g, 0, 8)),
        lambda: layers.embedding_forward(t, rand(g, 8, 4).t()), lambda: layers.embedding_forward(t[::2], x),
        lambda: layers.embedding_backward(x, t[:3], 6), lambda: layers.embedding_backward(x, t, 0),
        lambda: layers.embedding_backward(x.cpu(), t, 6),
        lambda: layers.sort_by_expert(t, 6), lambda: layers.sort_by_expert(t[:, None], 0),
        lambda: layers.sort_by_expert(t[:, None], 257), lambda: layers.sort_by_expert(t.view(1, 4)[:, ::2], 6),
        lambda: layers.sort_by_expert(torch.zeros(3, 0, dtype=torch.int64, device=DEV), 6),
        lambda: layers.sort_by_expert(t[:, None].cpu(), 6),
        lambda: layers.dispatch_forward(rand(g, 5, 8), r), lambda: layers.dispatch_forward(x.cpu(), r),
        lambda: layers.dispatch_forward(x, r._replace(source=r.source[:3])),
        lambda: layers.dispatch_forward(x, r._replace(position=r.position.long())),
        lambda: layers.dispatch_backward(rand(g, 5, 8), r),
        lambda: layers.combine_forward(x, p[:3], r), lambda: layers.combine_forward(x, p.double(), r),
        lambda: layers.combine_forward(x, p.cpu(), r), lambda: layers.combine_forward(rand(g, 5, 8), p, r),
        lambda: layers.combine_forward(x, p, r, residual=rand(g, 4, 7)),
        lambda: layers.combine_backward(rand(g, 3, 8), x, p, r), lambda: layers.combine_backward(x, x.bfloat16(), p, r),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(x, w, t.float()), lambda: layers.embedding_forward(t.short(), x), lambda: f(x.half(), w.half(), t),
                 lambda: layers.sort_by_expert(p, 6), lambda: layers.dispatch_forward(x, r.position),
                 lambda: layers.embedding_forward([1, 2], x), lambda: f(x, w, [1, 2, 3, 4])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(MuonError, match="scale"):
        layers.embedding_forward(t, x, scale=float("nan"))
    with pytest.raises(MuonError, match="2\\^20"):
        f(torch.zeros(1, (1 << 20) + 8, device=DEV), torch.zeros((1 << 20) + 8, 8, device=DEV), t[:1])


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("tokens,top,cols,experts", [(1, 1, 1, 1), (3, 2, 72, 5), (700, 6, 40, 64)])
def test_compiled_calls_and_those_in_python_are_the_same(dtype, tokens, top, cols, experts):
    """On another stream than the default one, rows of wider ones."""
    g = gen(tokens)
    fast = layers._compiled()
    wide = lambda n: torch.randn(n, cols + 3, generator=g, device=DEV).to(dtype)[:, :cols]
    choice = torch.randint(-1, experts + 1, (tokens, top), generator=g, device=DEV)
    x, h, r = wide(tokens), wide(tokens * top), wide(tokens)
    w = torch.rand(tokens, top, generator=g, device=DEV)
    ids = torch.randint(-1, tokens + 1, (2, 3), generator=g, device=DEV, dtype=torch.int32)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        route = layers._sort_by_expert(choice, experts)
        pairs = [(fast.sort_by_expert(choice, experts), route),
                 (fast.dispatch_forward(x, route), layers._dispatch_forward(x, route)),
                 (fast.dispatch_backward(h, route), layers._dispatch_backward(h, route)),
                 (fast.embedding_forward(ids, x, 1.5), layers._embedding_forward(ids, x, 1.5))]
        dy = x.new_ones(2, 3, cols) / 3
        pairs.append((fast.embedding_backward(dy, ids, tokens, 1.5), layers._embedding_backward(dy, ids, tokens, 1.5)))
        for res in (None, r):
            pairs.append((fast.combine_forward(h, w, route, res), layers._combine_forward(h, w, route, res)))
        for weights in (w, w.to(dtype)):
            for rg, wg in ((True, True), (True, False), (False, True), (False, False)):
                pairs.append((fast.combine_backward(x, h, weights, route, rg, wg),
                              layers._combine_backward(x, h, weights, route, rg, wg)))
    stream.synchronize()
    for a, b in pairs:
        a, b = (v if isinstance(v, tuple) else (v,) for v in (a, b))
        assert len(a) == len(b)
        for s, t in zip(a, b):
            assert (s is None) == (t is None)
            assert s is None or (s.dtype == t.dtype and s.shape == t.shape and s.stride() == t.stride()
                                 and torch.equal(s, t))


def test_compiled_calls_leave_what_does_not_fit_to_python():
    """(Each of these either is refused there or has nothing to do.)"""
    fast = layers._compiled()
    x, h = torch.zeros(4, 8, device=DEV), torch.zeros(8, 8, device=DEV)
    w, choice = torch.zeros(4, 2, device=DEV), torch.zeros(4, 2, device=DEV, dtype=torch.int64)
    ids = torch.zeros(3, device=DEV, dtype=torch.int64)
    r = layers.sort_by_expert(choice, 4)
    torch.cuda.synchronize()
    none = [fast.sort_by_expert(*a) for a in ((choice, 0), (choice, 1 << 20), (choice, 1 << 80), (choice, 2.0), (choice,),
                                              (choice.float(), 4), (choice.t(), 4), (choice.cpu(), 4), (choice[0], 4),
                                              (choice[:0], 4), (3, 4), (None, 4))]
    for a in ((x.half(), r), (x.t(), r), (x[:3], r), (x[:, ::2], r), (x.cpu(), r), (x[0], r), (x, r[:2]), (x, None), (7, r),
              (x, (r[0], r[1].long(), r[2])), (x, (r[0], r[1], r[2][:7])), (x, (r[0], r[1].cpu(), r[2])),
              (x[:, :0], r), (x[:1].expand(4, 8), r)):
        none += [fast.dispatch_forward(*a)]
    none += [fast.dispatch_backward(x, r), fast.dispatch_backward(h.t()[:7], r)]
    for a in ((h, w, r, x[:3]), (h, w, r, x.bfloat16()), (h, w.double(), r, None), (h, w.bfloat16(), r, None),
              (h, w.t(), r, None), (h[:7], w, r, None), (h, w, r), (h, w[:3], r, None), (h, None, r, None)):
        none += [fast.combine_forward(*a)]
    for a in ((x, h, w, r, 1, True), (x[:3], h, w, r, True, True), (x, h[:7], w, r, True, True),
              (x, h.bfloat16(), w, r, True, True)):
        none += [fast.combine_backward(*a)]
    for a in ((ids, x, 1), (ids.float(), x, 1.0), (ids, x[:0], 1.0), (ids[:0], x, 1.0), (ids[::2], x, 1.0),
              (ids.cpu(), x, 1.0), (ids, x.half(), 1.0), (ids, x, float("nan")), (ids, x, float("inf"))):
        none += [fast.embedding_forward(*a)]
    dy = x[:3]
    for a in ((dy, ids, 1.0, 1.0), (dy, ids, 0, 1.0), (dy[:2], ids, 4, 1.0), (dy.half(), ids, 4, 1.0), (dy, ids.cpu(), 4, 1.0),
              (x[:3, 1:], ids, 4, 1.0), (dy, ids, 4, float("inf")), (dy[:0], ids[:0], 4, 1.0), (dy[:, :0], ids, 4, 1.0),
              (dy, ids[0], 4, 1.0), (dy[0, 0], ids, 4, 1.0)):
        none += [fast.embedding_backward(*a)]
    assert all(v is None for v in none)
    with pytest.raises(MuonError, match="scale"):
        layers.embedding_forward(ids, x, scale=float("nan"))


def test_calls_of_two_threads_at_once():
    """Each on its own stream, with its own sizes and one refusal among its calls."""
    import threading
    bad = []

    def work(seed, tokens, experts, cols):
        g = gen(seed)
        x, w = rand(g, tokens, cols), torch.rand(tokens, 2, generator=g, device=DEV)
        choice, ids = numbers(g, experts, tokens, 2), numbers(g, tokens, 40)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            first = None
            for i in range(200):
                r = layers.sort_by_expert(choice, experts)
                h = layers.dispatch_forward(x, r)
                y = layers.combine_forward(h, w, r, residual=x)
                dh, dw = layers.combine_backward(y, h, w, r)
                e = layers.embedding_forward(ids, y)
                de = layers.embedding_backward(e, ids, tokens)
                out = (*r, h, y, dh, dw, e, de)
                if i == 50:
                    with pytest.raises(ValueError):
                        layers.dispatch_forward(x[1:], r)
                first = first or out
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(out, first)):
                    bad.append((seed, i))
                    return

    threads = [threading.Thread(target=work, args=a) for a in ((1, 300, 9, 64), (2, 41, 64, 130))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@pytest.mark.parametrize("case", [(9, 1344, 66001, torch.bfloat16), (16, 1329, 66048, torch.bfloat16),
                                  (17, 680, 66001, torch.float32), (32, 669, 66048, torch.float32)], ids=ids_of)
def test_large_weight_gradients_of_few_rows(case):
    """Of more than 160 MB: the outer products of the most rows."""
    rows, inner, vocab, dtype = case
    g = gen(rows + 170)
    for transposed in (False, True):
        x, w, t = loss_case(g, rows, inner, vocab, dtype, transposed, outside=0.2)
        check_loss(x, w, t, "none" if transposed else "sum", g)
        torch.cuda.empty_cache()


def test_calls_of_two_threads_give_what_one_gives():
    """Threads on streams of their own, with refusals among their calls: every output is that
    of the same calls made before by one thread, and what a thread raises is raised here."""
    from concurrent.futures import ThreadPoolExecutor
    from paper_2606_27153_amd import adamw
    rounds = 200

    def inputs(seed, tokens, experts, cols):
        g = gen(seed)
        return dict(x=rand(g, tokens, cols), w=torch.rand(tokens, 2, generator=g, device=DEV), experts=experts,
                    choice=numbers(g, experts, tokens, 2), ids=numbers(g, tokens, 40), t=numbers(g, tokens, tokens),
                    p=rand(g, tokens, cols), state=adamw.new_state(torch.empty(tokens, cols, device=DEV), 8))

    def calls(a):
        r = layers.sort_by_expert(a["choice"], a["experts"])
        h = layers.dispatch_forward(a["x"], r)
        y = layers.combine_forward(h, a["w"], r, residual=a["x"])
        dx = layers.dispatch_backward(h, r)
        dh, dw = layers.combine_backward(y, h, a["w"], r)
        e = layers.embedding_forward(a["ids"], y)
        de = layers.embedding_backward(e, a["ids"], len(a["x"]))
        loss, lse = layers.linear_cross_entropy_forward(a["x"], y.t(), a["t"], reduction="sum")
        grads = layers.linear_cross_entropy_backward(torch.ones_like(loss), a["x"], y.t(), a["t"], lse, reduction="sum")
        p, state = a["p"].clone(), [s.clone() for s in a["state"]]
        adamw.adamw_step([p], [dx], [state], step=1, lr=1e-3)
        return (*r, h, y, dx, dh, dw, e, de, loss, lse, *grads, p, *state)

    cases = [inputs(1, 300, 9, 64), inputs(2, 41, 64, 130)]
    want = [calls(a) for a in cases]
    torch.cuda.synchronize()

    def work(k):
        a, done = cases[k], 0
        with torch.cuda.stream(torch.cuda.Stream()):
            for i in range(rounds):
                got = calls(a)
                if i % 50 == 7:
                    with pytest.raises(ValueError):
                        layers.dispatch_forward(a["x"][1:], got[:3])
                    with pytest.raises(MuonError):
                        layers.embedding_forward(a["ids"], a["x"], scale=float("inf"))
                torch.cuda.current_stream().synchronize()
                for j, (v, w) in enumerate(zip(got, want[k])):
                    assert torch.equal(v, w), (k, i, j)
                done += 1
        return done

    with ThreadPoolExecutor(2) as pool:
        assert [f.result() for f in [pool.submit(work, k) for k in (0, 1)]] == [rounds, rounds]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids_of)
@pytest.mark.parametrize("tokens,top,cols,pad", [(1, 1, 1, 0), (40, 3, 50, 11), (300, 6, 264, 0), (65, 9, 136, 24),
                                                 (33, 17, 77, 3)])
def test_combine_writes_over_its_residual(tokens, top, cols, pad, dtype):
    """y in the residual's own buffer (same ld), as the C ABI allows: bit by bit what another
    buffer gets, and nothing beside its rows."""
    g = gen(tokens + 60)
    lib = layers._load()
    routing = layers.sort_by_expert(numbers(g, 19, tokens, top, outside=0.2), 19)
    h, w = rand(g, tokens * top, cols, dtype=dtype), torch.rand(tokens, top, generator=g, device=DEV)
    wide = rand(g, tokens + 2, cols + pad, dtype=dtype)
    y = wide[1:-1, pad // 2:pad // 2 + cols]
    want = wide.clone()
    want[1:-1, pad // 2:pad // 2 + cols] = layers.combine_forward(h, w, routing, residual=y)
    code = layers._DTYPES[dtype]
    layers.LL.check(lib.muon_combine_forward(
        h.data_ptr(), cols, w.data_ptr(), layers.MUON_F32, routing.position.data_ptr(), y.data_ptr(), cols + pad,
        y.data_ptr(), cols + pad, tokens, top, cols, code, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(wide, want)


def test_an_ignore_index_of_more_than_64_bits_is_refused():
    """(Cut to 64 bits it would be a token's.)"""
    x, w = torch.ones(2, 8, device=DEV), torch.ones(8, 6, device=DEV)
    t = torch.tensor([5, 1], device=DEV)
    loss, lse = layers.linear_cross_entropy_forward(x, w, t, ignore_index=-1 << 63)
    for index in ((1 << 64) + 5, 1 << 63, -(1 << 63) - 1):
        with pytest.raises(ValueError, match="64 bits"):
            layers.linear_cross_entropy_forward(x, w, t, ignore_index=index)
        with pytest.raises(ValueError, match="64 bits"):
            layers.linear_cross_entropy_backward(loss, x, w, t, lse, ignore_index=index)
        with pytest.raises(ValueError, match="64 bits"):
            layers.linear_cross_entropy(x, w, t, ignore_index=index)
