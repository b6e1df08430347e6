"""The operators that take token or expert numbers on the GPU -- embedding, the
way to the experts and back, the loss over a vocabulary -- against plain ones in 64 bits
(tests/tokens_ref.py, which derives the bounds)."""
import pytest
import torch

import layers_ref as L
import tokens_ref as R
from paper_2606_27153_amd import layers

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
          (1030, 264, 2056), (0, 16, 40)]


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


def test_loss_in_row_blocks_and_pieces():
    """More rows than a forward pass takes at once, more columns than a piece has."""
    g = gen(11)
    for rows, inner, vocab, transposed, dtype in (
            (33000, 24, 600, False, torch.bfloat16), (20000, 64, 40000, True, torch.bfloat16),
            (100, 72, 50001, False, torch.bfloat16), (70, 16, 270000, True, torch.float32),
            (9, 16, 270001, False, torch.bfloat16), (300, 40, 66001, False, torch.float32)):
        x, w, t = loss_case(g, rows, inner, vocab, dtype, transposed)
        check_loss(x, w, t, "mean", g)
        torch.cuda.empty_cache()
