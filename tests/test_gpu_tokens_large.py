"""The token and expert operators, the loss and AdamW on the GPU where indexes pass 31 and
32 bits: values whose sums are exact in fp32, so that results are known bit by bit, or
the 64-bit reference at the ends of what is too large to compare whole."""
import numpy as np
import pytest
import torch

import adamw_ref as A
import layers_ref as L
import tokens_ref as R
from paper_2606_27153_amd import adamw, layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
ids_of = lambda v: str(v).replace("torch.", "")
COLS = 2056
ROWS = (1 << 20) + 5       # by COLS: more than 2^31 elements


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def small(g, *shape):
    """-1, 0 and 1 in bf16."""
    return torch.randint(-1, 2, shape, generator=g, device=DEV, dtype=torch.int8).to(BF16)


def test_lookups_in_and_gradients_of_a_large_table():
    g = gen(1)
    table = small(g, ROWS, COLS)
    ids = torch.randint(ROWS, (3000,), generator=g, device=DEV)
    ids[:4] = torch.tensor([0, ROWS - 1, ROWS // 2, ROWS])
    y = layers.embedding_forward(ids, table)
    assert torch.equal(y[:3], table[ids[:3]]) and torch.equal(y[4:], table[ids[4:]]) and (y[3] == 0).all()
    dw = layers.embedding_backward(y, ids, ROWS)
    live, count = ids[ids < ROWS].unique(return_counts=True)
    assert torch.equal(dw[live], table[live] * count[:, None].to(BF16))
    rest = torch.ones(ROWS, dtype=torch.bool, device=DEV)
    rest[live] = False
    assert not any(dw[a:a + 65536][rest[a:a + 65536]].any() for a in range(0, ROWS, 65536))


def test_lookups_of_many_tokens_and_the_gradient_of_all_of_them():
    g = gen(2)
    table = small(g, 1000, COLS)
    ids = torch.randint(1000, (ROWS,), generator=g, device=DEV, dtype=torch.int32)
    ids[-3000:] = 999
    y = layers.embedding_forward(ids, table)
    assert torch.equal(y, table[ids])
    dw = layers.embedding_backward(y, ids, 1000)
    want = table.float() * torch.bincount(ids, minlength=1000)[:, None]
    assert torch.equal(dw, want.to(BF16))


def test_routing_of_many_rows():
    g = gen(3)
    tokens, top, experts = ROWS // 4 + 1, 4, 64
    x = small(g, tokens, COLS)
    choice = torch.rand(tokens, experts, generator=g, device=DEV).topk(top, 1).indices
    choice[::5, 3] = experts      # of no expert
    routing = layers.sort_by_expert(choice, experts)
    n = int(routing.offsets[-1])
    source, live = routing.source, choice < experts
    assert n == int(live.sum()) and torch.equal(routing.position >= 0, live)
    rows = layers.dispatch_forward(x, routing)
    for a in range(0, n, 1 << 18):
        b = min(n, a + (1 << 18))
        assert torch.equal(rows[a:b], x[(source[a:b] // top).long()])
    assert not rows[n:].any()
    count = live.sum(1, keepdim=True).to(BF16)
    assert torch.equal(layers.dispatch_backward(rows, routing), x * count)
    w = torch.tensor([0.5, 0.25, 0.125, 0.125], device=DEV).expand(tokens, top).contiguous()
    y = layers.combine_forward(rows, w, routing, residual=x)
    assert torch.equal(y, (x.float() * (1 + (w * live).sum(1, keepdim=True))).to(BF16))
    drows, dw = layers.combine_backward(x, rows, w, routing)
    for a in range(0, n, 1 << 18):
        b = min(n, a + (1 << 18))
        s = source[a:b].long()
        assert torch.equal(drows[a:b], (x[s // top].float() * w.view(-1)[s, None]).to(BF16))
    assert not drows[n:].any()
    assert torch.equal(dw, x.float().square().sum(1, keepdim=True) * live)


def test_loss_of_many_rows():
    """97 different rows with their targets, over and over: dz has more than 2^31 elements."""
    g = gen(4)
    inner, vocab, period = 8, 2048, 97
    base = torch.randn(period, inner, generator=g, device=DEV).to(BF16)
    which = torch.arange(ROWS, device=DEV) % period
    x, at = base[which], torch.randint(vocab, (period,), generator=g, device=DEV)
    at[5] = -100
    w = (torch.randn(inner, vocab, generator=g, device=DEV) * 0.5).to(BF16)
    loss, lse = layers.linear_cross_entropy_forward(x, w, at[which], reduction="none")
    for name, v in (("loss", loss), ("lse", lse)):
        assert torch.equal(v, v[:period][which]), name
    ref = R.Loss(base, w, at)
    L.check(lse[:period], ref.lse.cpu(), ref.lse_error.cpu(), "lse")
    L.check(loss[:period], *(v.cpu() for v in ref.rows()), "loss")
    dx, dw = layers.linear_cross_entropy_backward(torch.ones(ROWS, device=DEV), x, w, at[which], lse, reduction="none")
    assert torch.equal(dx, dx[:period][which])
    one = ref.backward(torch.ones(period, device=DEV), "none")
    L.check(dx[:period], *(v.cpu() for v in one["dx"]), "dx")
    # the weight's gradient is linear in the rows' factors: how often each comes
    often = torch.bincount(which).double()
    value, bound = ref.backward(often, "none")["dw"]
    # (sums of ROWS terms: 12 and the period's are in the bound already)
    terms = ref.x.abs().t() @ (often[:, None] * (ref.p + 1))
    L.check(dw, value.cpu(), (bound + ROWS * L.U * terms).cpu(), "dw")


@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("transposed", [False, True])
def test_loss_over_a_large_weight(rows, transposed):
    """[inner, vocab] of more than 2^31 elements: compared at its ends and around its middle."""
    g = gen(5)
    inner, vocab = 8200, (1 << 18) + 8
    w = torch.empty((vocab, inner) if transposed else (inner, vocab), dtype=BF16, device=DEV)
    for part in w.split(4096):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * (2 * inner ** -0.5))
    w = w.t() if transposed else w
    x = torch.randn(rows, inner, generator=g, device=DEV).to(BF16)
    t = torch.randint(vocab, (rows,), generator=g, device=DEV)
    t[:2] = torch.tensor([vocab - 1, -100])
    loss, lse = layers.linear_cross_entropy_forward(x, w, t)
    dx, dw = layers.linear_cross_entropy_backward(torch.tensor(1.7, device=DEV), x, w, t, lse)
    ref = R.Loss(x, w, t)
    L.check(lse, ref.lse.cpu(), ref.lse_error.cpu(), "lse")
    L.check(loss, *(v.cpu() for v in ref.total("mean")), "loss")
    want = ref.backward(torch.tensor(1.7, device=DEV), "mean")
    L.check(dx, *(v.cpu() for v in want["dx"]), "dx")
    for a in (0, vocab // 2 - 150, vocab - 300):
        L.check(dw[:, a:a + 300], *(v[:, a:a + 300].cpu() for v in want["dw"]), f"dw from column {a}")
    for a in (0, inner // 2, inner - 2):
        L.check(dw[a:a + 2], *(v[a:a + 2].cpu() for v in want["dw"]), f"dw from row {a}")


HOW = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def test_adamw_of_a_large_tensor():
    n = (1 << 31) + 4099
    p, g = torch.full((n,), 0.5, dtype=BF16, device=DEV), torch.full((n,), 0.25, dtype=BF16, device=DEV)
    state = adamw.new_state(p)
    at = [slice(0, 9000), slice((1 << 31) - 5000, (1 << 31) + 1000), slice(n - 5000, n)]
    r = gen(6)
    for s in at:
        p[s] = torch.randn(p[s].shape, generator=r, device=DEV).to(BF16)
        g[s] = torch.randn(p[s].shape, generator=r, device=DEV).to(BF16)
    parts = [(p[s].clone(), g[s].clone(), adamw.new_state(p[s])) for s in at]
    adamw.adamw_step([p], [g], [state], step=1, **HOW)
    adamw.adamw_step([v[0] for v in parts], [v[1] for v in parts], [v[2] for v in parts], step=1, **HOW)
    for s, (q, _, (m, v)) in zip(at, parts):
        assert torch.equal(p[s], q) and torch.equal(state[0][s], m) and torch.equal(state[1][s], v)
    assert (p[9000:(1 << 31) - 5000] == p[9000]).all()


def test_adamw_of_a_large_tensor_with_8_bit_states():
    """More than 2^32 elements: the rounding of those behind has a key of its own."""
    n, tail, seed, step = (1 << 32) + 4099, 1 << 32, 7, 3
    p, g = torch.full((n,), 0.5, dtype=BF16, device=DEV), torch.full((n,), 0.25, dtype=BF16, device=DEV)
    r = gen(7)
    state = adamw.new_state(p, 8)
    ends = [slice(0, 8192), slice(tail, n)]
    for s in ends:
        g[s] = (torch.randn(p[s].shape, generator=r, device=DEV) * 1e-3).to(BF16)
        p[s] = torch.randn(p[s].shape, generator=r, device=DEV).to(BF16)
    old = [(p[s].float().cpu().numpy(), g[s].float().cpu().numpy()) for s in ends]
    adamw.adamw_step([p], [g], [state], step=step, seed=seed, **HOW)
    values = adamw.state_values(state)
    u = lambda v: np.uint32(v & 0xFFFFFFFF)
    key = A.mix(u(int(A.mix(u(seed + step * 0x9E3779B9))) + 0))
    for s, (w, d), k in zip(ends, old, (key, A.mix(u(int(key) + 1)))):
        zero = np.zeros_like(d)
        mn, vn = A.averages(d, zero, zero, HOW["betas"])
        with np.errstate(over="ignore"):
            h = A.mix((np.arange(d.size, dtype=np.uint32) * np.uint32(0x9E3779B1)) ^ k)
        for i, (new, bits, signed) in enumerate(((mn, h & np.uint32(0xFFFF), True), (vn, h >> np.uint32(16), False))):
            codes, bases = A.encode(new, bits << np.uint32(4), signed)
            assert np.array_equal(state[i][s].cpu().numpy(), codes), (s, i)
            rows = slice(s.start // 256, -(-s.stop // 256))
            assert np.array_equal(state[2][rows, i].cpu().numpy(), bases), (s, i)
            held = torch.from_numpy(A.decode(codes, bases, signed)).to(BF16)
            assert torch.equal(values[i][s].cpu(), held), (s, i)
        L.check(p[s], *A.param(w, d, zero, zero, step, HOW["lr"], HOW["betas"], HOW["eps"], HOW["weight_decay"], BF16),
                "param")
    assert (p[8192:tail] == p[8192]).all()
