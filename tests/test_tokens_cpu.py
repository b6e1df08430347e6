"""The token and expert operators without a GPU: the C ABI's argument checks, which
come before any device call, and what the Python entry points refuse."""
import ctypes

import pytest
import torch

from paper_2606_27153_amd import _layers_lib as LL
from paper_2606_27153_amd import _lib as L
from paper_2606_27153_amd import layers

X, Y, WS = 0x1000, 0x2000, 0x10000   # addresses that are checked, never read
BF16, F32 = L.MUON_BF16, L.MUON_F32


@pytest.fixture(scope="module")
def lay():
    return LL.load()


def refused(lay, status, word, want=L.MUON_ERR_INVALID_ARG):
    assert status == want, (status, lay.muon_layers_last_error())
    assert word in lay.muon_layers_last_error().decode(), lay.muon_layers_last_error()


def test_reductions_match_the_header():
    assert LL.REDUCTIONS == {"none": 0, "sum": 1, "mean": 2}


@pytest.mark.parametrize("kw,word", [
    (dict(ids=None), "ids"), (dict(ids=X + 4), "ids"), (dict(w=None), "w is NULL"), (dict(w=X + 1), "w is not"),
    (dict(y=None), "y is NULL"), (dict(ldw=7), "w has"), (dict(ldy=7), "y has"), (dict(rows=-1), "rows"),
    (dict(vocab=0), "vocab"), (dict(cols=0), "cols"), (dict(cols=1 << 25, ldw=1 << 25, ldy=1 << 25), "cols"),
    (dict(scale=float("inf")), "scale")])
def test_embedding_refusals(lay, kw, word):
    a = dict(ids=X, size=8, w=X, ldw=8, y=Y, ldy=8, rows=4, vocab=5, cols=8, scale=1.0, dtype=F32)
    a.update(kw)
    refused(lay, lay.muon_embedding_forward(*a.values(), None), word)
    b = dict(dy=a["y"], lddy=a["ldy"], ids=a["ids"], size=8, dw=a["w"], lddw=a["ldw"], rows=a["rows"],
             vocab=a["vocab"], cols=a["cols"], scale=a["scale"], dtype=F32, ws=WS, bytes=1 << 40)
    refused(lay, lay.muon_embedding_backward(*b.values(), None), {"y is NULL": "dy is NULL", "y has": "dy has",
                                                                 "w is NULL": "dw is NULL"}.get(word, word))


def test_embedding_types_and_workspaces(lay):
    n = ctypes.c_size_t()
    assert lay.muon_embedding_workspace_bytes(1000, 300, 64, ctypes.byref(n)) == L.MUON_OK and n.value >= 4 * 4000
    call = lambda ws, b, dt=F32, size=8: lay.muon_embedding_backward(X, 64, X, size, Y, 64, 1000, 300, 64, 1.0, dt, ws, b, None)
    refused(lay, call(None, n.value), "workspace")
    refused(lay, call(WS, n.value - 1), "workspace", L.MUON_ERR_WORKSPACE_TOO_SMALL)
    refused(lay, call(WS + 16, n.value), "256-byte")
    refused(lay, call(WS, n.value, dt=7), "dtype", L.MUON_ERR_UNSUPPORTED)
    refused(lay, call(WS, n.value, size=2), "bytes", L.MUON_ERR_UNSUPPORTED)
    refused(lay, lay.muon_embedding_workspace_bytes(1, 1, 1, None), "bytes")
    assert lay.muon_embedding_forward(None, 8, None, 8, None, 8, 0, 5, 8, 1.0, F32, None) == L.MUON_OK


@pytest.mark.parametrize("kw,word", [
    (dict(ids=None), "ids"), (dict(offsets=None), "offsets"), (dict(offsets=X + 2), "offsets"),
    (dict(position=None), "position"), (dict(source=None), "source"), (dict(tokens=-1), "tokens"),
    (dict(top=0), "top"), (dict(top=257), "top"), (dict(experts=0), "experts"), (dict(experts=257), "experts"),
    (dict(tokens=1 << 29, top=4), "2^30")])
def test_sort_refusals(lay, kw, word):
    a = dict(ids=X, size=8, tokens=4, top=2, experts=5, offsets=X, position=X, source=X, ws=WS, bytes=1 << 40)
    a.update(kw)
    refused(lay, lay.muon_sort_by_expert(*a.values(), None), word)


def test_sort_workspaces(lay):
    n = ctypes.c_size_t()
    assert lay.muon_sort_by_expert_workspace_bytes(4, 2, ctypes.byref(n)) == L.MUON_OK and n.value == 0
    assert lay.muon_sort_by_expert_workspace_bytes(5000, 2, ctypes.byref(n)) == L.MUON_OK and n.value > 0
    refused(lay, lay.muon_sort_by_expert(X, 8, 5000, 2, 5, X, X, X, WS, n.value - 1, None), "workspace",
            L.MUON_ERR_WORKSPACE_TOO_SMALL)
    refused(lay, lay.muon_sort_by_expert(X, 3, 4, 2, 5, X, X, X, None, 0, None), "bytes", L.MUON_ERR_UNSUPPORTED)


def test_dispatch_and_combine_refusals(lay):
    def dispatch(x=X, ldx=8, pos=X, src=X, rows=Y, ldr=8, tokens=4, top=2, cols=8, dt=F32):
        return lay.muon_dispatch_forward(x, ldx, pos, src, rows, ldr, tokens, top, cols, dt, None)

    for kw, word in ((dict(x=None), "x is NULL"), (dict(ldx=7), "x has"), (dict(pos=None), "position"),
                     (dict(src=None), "source"), (dict(src=X + 1), "source"), (dict(rows=None), "rows is NULL"),
                     (dict(ldr=7), "rows has"), (dict(cols=0), "cols"), (dict(top=0), "top")):
        refused(lay, dispatch(**kw), word)
    refused(lay, dispatch(dt=9), "dtype", L.MUON_ERR_UNSUPPORTED)
    assert dispatch(tokens=0, x=None, pos=None, src=None, rows=None) == L.MUON_OK
    refused(lay, lay.muon_dispatch_backward(None, 8, X, Y, 8, 4, 2, 8, F32, None), "drows")
    refused(lay, lay.muon_dispatch_backward(X, 8, X, None, 8, 4, 2, 8, F32, None), "dx")

    def combine(rows=X, ldr=8, w=X, wdt=F32, pos=X, res=None, ldres=8, y=Y, ldy=8, dt=BF16):
        return lay.muon_combine_forward(rows, ldr, w, wdt, pos, res, ldres, y, ldy, 4, 2, 8, dt, None)

    for kw, word in ((dict(rows=None), "rows"), (dict(w=None), "weights"), (dict(w=X + 2), "weights"),
                     (dict(pos=None), "position"), (dict(res=X, ldres=7), "residual"), (dict(y=None), "y is NULL"),
                     (dict(ldy=7), "y has")):
        refused(lay, combine(**kw), word)
    refused(lay, combine(wdt=BF16, dt=F32), "weight_dtype", L.MUON_ERR_UNSUPPORTED)
    refused(lay, lay.muon_combine_backward(None, 8, X, 8, X, F32, X, Y, 8, Y, 4, 2, 8, F32, None), "dy")
    refused(lay, lay.muon_combine_backward(X, 8, None, 8, X, F32, X, Y, 8, Y, 4, 2, 8, F32, None), "rows")
    refused(lay, lay.muon_combine_backward(X, 8, X, 8, X, F32, X, Y, 7, Y, 4, 2, 8, F32, None), "drows")
    refused(lay, lay.muon_combine_backward(X, 8, X, 8, X, F32, X, Y, 8, Y + 1, 4, 2, 8, F32, None), "dweights")


def _loss(lay, back=False, **kw):
    a = dict(x=X, ldx=8, w=X, ldw=6, t=0, targets=X, size=8, ignore=-100, red=2, loss=Y, lse=Y, rows=4, inner=8, outer=6,
             dtype=F32, ws=WS, bytes=1 << 40, dx=Y, lddx=8, dw=Y, lddw=6)
    a.update(kw)
    head = [a[k] for k in ("x", "ldx", "w", "ldw", "t", "targets", "size", "ignore", "red")]
    tail = [a[k] for k in ("rows", "inner", "outer", "dtype", "ws", "bytes")] + [None]
    if back:
        return lay.muon_linear_cross_entropy_backward(a["loss"], *head, a["lse"], a["dx"], a["lddx"], a["dw"], a["lddw"],
                                                      *tail)
    return lay.muon_linear_cross_entropy_forward(*head, a["loss"], a["lse"], *tail)


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "x is NULL"), (dict(w=None), "w is NULL"), (dict(ldx=7), "x has"), (dict(ldw=5), "w has"),
    (dict(t=1), "w has"), (dict(targets=None), "targets"), (dict(targets=X + 4), "targets"), (dict(red=3), "reduction"),
    (dict(red=-1), "reduction"), (dict(loss=None), "loss"), (dict(lse=None), "lse"), (dict(rows=-1), "rows"),
    (dict(inner=0), "inner"), (dict(outer=0), "outer"), (dict(ws=None), "workspace"), (dict(ws=WS + 8), "256-byte")])
def test_loss_refusals(lay, kw, word):
    refused(lay, _loss(lay, **kw), word)
    refused(lay, _loss(lay, back=True, **kw), word)


def test_loss_types_limits_and_workspaces(lay):
    for back in (False, True):
        refused(lay, _loss(lay, back, dtype=5), "dtype", L.MUON_ERR_UNSUPPORTED)
        refused(lay, _loss(lay, back, size=1), "bytes", L.MUON_ERR_UNSUPPORTED)
        refused(lay, _loss(lay, back, inner=(1 << 20) + 1, ldx=1 << 21), "2^20", L.MUON_ERR_UNSUPPORTED)
        refused(lay, _loss(lay, back, bytes=255), "workspace", L.MUON_ERR_WORKSPACE_TOO_SMALL)
    refused(lay, _loss(lay, True, lddx=7), "dx has")
    refused(lay, _loss(lay, True, lddw=5), "dw has")
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    size = lay.muon_linear_cross_entropy_workspace_bytes
    assert size(5000, 64, 50000, BF16, 1, ctypes.byref(n)) == L.MUON_OK
    assert size(5000, 64, 50000, BF16, 3, ctypes.byref(m)) == L.MUON_OK
    # not the logits of all rows and columns; room for copies on top
    assert n.value < 5000 * 50000 * 2 + (1 << 28) and m.value >= n.value
    refused(lay, size(1, 1, 1, F32, 4, ctypes.byref(n)), "flags")
    refused(lay, size(1, 1, 1, F32, 0, None), "bytes")
    # nothing to do
    assert _loss(lay, True, rows=0, x=None, w=None, targets=None, loss=None, lse=None, dx=None, dw=None) == L.MUON_OK


def test_python_refusals_without_a_gpu():
    x, w, t = torch.zeros(4, 8), torch.zeros(8, 6), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: layers.linear_cross_entropy(x, w, t), lambda: layers.embedding(t, x),
                 lambda: layers.sort_by_expert(t[:, None], 4), lambda: layers.linear_cross_entropy(x, w, t[:3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: layers.linear_cross_entropy(x, w, [0, 0, 0, 0]), lambda: layers.embedding([1], x),
                 lambda: layers.embedding(t, None), lambda: layers.combine(None, x, None),
                 lambda: layers.combine(x, None, None)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("outer", [131072, 524288, 1 << 20, 3000001, 1 << 24])
def test_the_losss_sums_over_a_very_large_vocabulary_stay_in_1_gb(lay, outer, dtype):
    """The forward pass's workspace: 2^27 sums of 8 bytes at most (their places are counted
    piece by piece, so up to 64 columns' worth more for each of the pieces), and two
    numbers a row."""
    n = ctypes.c_size_t()
    for rows in (33, 64, 300, 5000, 20000, 32768, 1 << 20):
        for inner in (64, 256):
            assert lay.muon_linear_cross_entropy_workspace_bytes(rows, inner, outer, dtype, 0, ctypes.byref(n)) == L.MUON_OK
            assert n.value <= (1 << 30) + (64 * 32768 * 8) + 8 * rows + 1024, (rows, n.value)
