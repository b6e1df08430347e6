"""The AdamW step on the GPU against plain ones (tests/adamw_ref.py)."""
import numpy as np
import pytest
import torch

import adamw_ref as R
import layers_ref as L
from paper_2606_27153_amd import AdamW, adamw
from paper_2606_27153_amd._lib import MuonError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
ids_of = lambda v: str(v).replace("torch.", "")
HOW = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def f32(t):
    return t.detach().float().cpu().numpy().reshape(-1).copy()


def make(g, shape, pdt, gdt, bits, offset=0):
    """(param, grad, state) as views `offset` elements into their buffers."""
    n = int(np.prod(shape))

    def rand(scale, dtype):
        return (torch.randn(n + offset, generator=g, device=DEV) * scale).to(dtype)[offset:].view(shape)

    p, d = rand(0.1, pdt), rand(1e-3, gdt)
    if bits == 32:
        return p, d, (rand(5e-4, F32), rand(1e-3, F32).square_())
    state = adamw.new_state(p, 8)
    state[0].copy_(torch.randint(0, 256, (n,), generator=g, device=DEV))
    state[1].copy_(torch.randint(0, 256, (n,), generator=g, device=DEV))
    state[2][:, 0] = 117 * 8 - 127      # the largest about 2^-10
    state[2][:, 1] = 107 * 8 - 255
    return p, d, state


def old_averages(state):
    if len(state) == 2:
        return f32(state[0]), f32(state[1])
    base = state[2].cpu().numpy()
    return (R.decode(state[0].cpu().numpy(), base[:, 0], True), R.decode(state[1].cpu().numpy(), base[:, 1], False))


def expect(p, g, state, step, seed, index, how=HOW):
    """What a step leaves: (param, bound), then the averages or the codes and bases."""
    m, v = old_averages(state)
    new = R.param(f32(p), f32(g), m, v, step, how["lr"], how["betas"], how["eps"], how["weight_decay"], p.dtype)
    mn, vn = R.averages(f32(g), m, v, how["betas"])
    if len(state) == 2:
        return new, (mn, vn)
    rm, rv = R.random_bits(mn.size, seed, step, index)
    cm, bm = R.encode(mn, rm, True)
    cv, bv = R.encode(vn, rv, False)
    return new, (cm, cv, np.stack([bm, bv], 1))


def check(p, state, want, what=""):
    new, held = want
    L.check(p.reshape(-1), *new, f"param {what}")
    for name, got, ref in zip(("exp_avg", "exp_avg_sq", "bases"), state, held):
        assert np.array_equal(got.cpu().numpy().reshape(-1), ref.reshape(-1)), (name, what)


SHAPES = [(1,), (7,), (8,), (255,), (256,), (257,), (3, 5), (4095,), (4096,), (4097,), (2049,), (100, 333), (70001,)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt,gdt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)], ids=ids_of)
def test_step_of_tensors_of_all_sizes(pdt, gdt, bits):
    g = gen(bits)
    for step, offset in ((1, 0), (7, 3), (100000, 0)):
        rows = [make(g, s, pdt, gdt, bits, offset) for s in SHAPES]
        want = [expect(*r, step, 5, i) for i, r in enumerate(rows)]
        adamw.adamw_step(*zip(*rows), step=step, seed=5, **HOW)
        for s, r, w in zip(SHAPES, rows, want):
            check(r[0], r[2], w, f"{s} step {step}")


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_of_mixed_types_steps_and_missing_gradients(bits):
    g = gen(3)
    types = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]
    rows = [list(make(g, (17 * i % 700,), *types[i % 4], bits)) for i in range(250)]   # some are empty
    steps = [1 + i % 5 for i in range(250)]
    want = []
    for i, r in enumerate(rows):
        if i % 7 == 3:
            r[1] = None
        want.append(expect(*r, steps[i], 9, i) if r[1] is not None and r[0].numel() else None)
    before = [(r[0].clone(), [t.clone() for t in r[2]]) for r in rows]
    adamw.adamw_step(*zip(*rows), step=steps, seed=9, **HOW)
    for i, (r, w) in enumerate(zip(rows, want)):
        if w is None:
            assert torch.equal(r[0], before[i][0]) and all(torch.equal(a, b) for a, b in zip(r[2], before[i][1]))
        else:
            check(r[0], r[2], w, str(i))


@pytest.mark.parametrize("bits", [32, 8])
def test_nothing_beside_the_tensors_is_written(bits):
    g = gen(8)
    for n in (5, 300, 4100):
        bufs = [torch.full((n + 64,), 7, dtype=d, device=DEV) for d in ((F32, F32, F32) if bits == 32 else
                                                                      (BF16, torch.uint8, torch.uint8))]
        views = [b[32:32 + n] for b in bufs]
        views[0].normal_(generator=g)
        for t in views[1:]:
            t.zero_()
        state = tuple(views[1:])
        if bits == 8:
            pad = torch.full((n // 256 + 9, 2), 7, dtype=torch.int16, device=DEV)
            blocks = -(-n // 256)
            state += (pad[4:4 + blocks],)
            state[2].zero_()
        adamw.adamw_step([views[0]], [torch.randn(n, generator=g, device=DEV)], [state], step=1, **HOW)
        for b in bufs:
            assert (b[:32] == 7).all() and (b[32 + n:] == 7).all()
        if bits == 8:
            assert (pad[:4] == 7).all() and (pad[4 + blocks:] == 7).all()


def test_eight_bit_extremes():
    """Zeros, values out of the block's range, infinities and NaN: the codes are those of the formula."""
    n = 2048
    g = torch.zeros(n, device=DEV)
    g[0:256:3] = 1.0
    g[1:256:3] = 1e-12                      # far below the block's largest
    g[256] = float("inf")
    g[513] = float("nan")
    g[768:1024] = 1e-42                     # fp32's smallest
    g[1024:1280] = -3.4e38
    g[1300] = 1e-30
    p = torch.randn(n, generator=gen(1), device=DEV)
    state = adamw.new_state(p, 8)
    with np.errstate(all="ignore"):
        want = expect(p, g, state, 1, 0, 0)
    adamw.adamw_step([p], [g], [state], step=1, **HOW)
    for name, got, ref in zip(("exp_avg", "exp_avg_sq", "bases"), state, want[1]):
        got = got.cpu().numpy()
        keep = np.ones(n, bool)
        keep[513] = name == "bases"         # (a NaN's sign is its own)
        assert np.array_equal(got.reshape(-1)[keep[:got.size]], ref.reshape(-1)[keep[:got.size]]), name
    m, v = adamw.state_values(state)
    assert m.dtype == v.dtype == BF16 and torch.equal(m[2:256:3], torch.zeros_like(m[2:256:3]))
    assert (v[1:256:3] > 0).all() and torch.isinf(m[256]) and torch.isnan(m[513].abs())
    fine = torch.isfinite(g) & (g.abs() < 1e30)
    assert torch.isfinite(p[fine]).all()


def test_eight_bit_rounding_keeps_the_mean():
    """An average that moves by less than a code's step moves on average: of n elements of one
    value, half as far as between two codes, the share that is rounded up is within 6 standard
    deviations, sqrt(n) / 2 each, of what keeps the mean; also over the steps of one element."""
    n = 1 << 20
    p = torch.zeros(n, device=DEV)
    state = adamw.new_state(p, 8)
    state[1].fill_(250)
    state[2][:, 1] = 800
    value = float(R.decode(np.array([250], np.uint8), np.array([800], np.int16), False)[0])
    g = torch.zeros(n, device=DEV)
    for step in range(1, 4):
        state[1].fill_(250)
        state[2][:, 1] = 800
        adamw.adamw_step([p], [g], [state], step=step, lr=0.0, betas=(0.9, 0.999))
        _, v = adamw.state_values(state)
        # 0.999 of it lies between its code and the one below, which the block's base keeps
        below = float(R.decode(np.array([249], np.uint8), np.array([800], np.int16), False)[0])
        up = int((v.float() == value).sum())
        assert up + int((v.float() == below).sum()) == n
        share = (np.float32(value) * np.float32(0.999) - below) / (value - below)
        assert abs(up - n * share) < 6 * (n * share * (1 - share)) ** 0.5 + n * 2.0 ** -16


@pytest.mark.parametrize("bits", [32, 8])
def test_step_in_a_graph_and_on_another_stream(bits):
    g = gen(12)
    rows = [make(g, s, BF16, BF16, bits) for s in ((300,), (64, 40), (5000,))]
    other = [(r[0].clone(), r[1].clone(), tuple(t.clone() for t in r[2])) for r in rows]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adamw.adamw_step(*zip(*rows), step=4, seed=2, **HOW)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            adamw.adamw_step(*zip(*other), step=4, seed=2, **HOW)
        torch.cuda.synchronize()
        for a, b in zip(rows, other):
            assert torch.equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(a[2], b[2]))


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_steps_as_the_function_and_survives_its_state_dict(bits):
    g = gen(20)
    shapes = [(40, 24), (33,), (300,)]
    dts = [BF16, F32, BF16]
    start = [torch.randn(*s, generator=g, device=DEV).to(d) for s, d in zip(shapes, dts)]
    grads = [[torch.randn(*s, generator=g, device=DEV).to(d) for s, d in zip(shapes, dts)] for _ in range(4)]

    def run(reload):
        ps = [torch.nn.Parameter(t.clone()) for t in start]
        groups = [dict(params=ps[:2]), dict(params=ps[2:], weight_decay=0.0, lr=1e-2)]
        opt = AdamW(groups, lr=1e-3, state_bits=bits, seed=4)
        for k, ds in enumerate(grads):
            for i, (p, d) in enumerate(zip(ps, ds)):
                p.grad = None if (k, i) == (1, 1) else d.t().contiguous().t() if d.dim() == 2 else d
            if reload and k == 2:
                fresh = AdamW([dict(params=ps[:2]), dict(params=ps[2:], weight_decay=0.0, lr=1e-2)], lr=1e-3,
                              state_bits=bits, seed=4)
                fresh.load_state_dict(opt.state_dict())
                opt = fresh
            opt.step()
        return ps, opt

    ps, opt = run(False)
    qs, _ = run(True)
    assert all(torch.equal(a, b) for a, b in zip(ps, qs))
    assert [opt.state[p]["step"] for p in ps] == [4, 3, 4]
    # the same by the function
    rs = [t.clone() for t in start]
    states = [adamw.new_state(t, bits) for t in rs]
    for k, ds in enumerate(grads):
        live = [0] if k == 1 else [0, 1]
        steps = [k + 1, k + 1 if k < 1 else k]
        adamw.adamw_step([rs[i] for i in live], [ds[i] for i in live], [states[i] for i in live],
                         step=[steps[i] for i in live], lr=1e-3, seed=4)
        adamw.adamw_step(rs[2:], ds[2:], states[2:], step=k + 1, lr=1e-2, weight_decay=0.0, seed=4 + 0x632BE5AB)
    assert all(torch.equal(a, b) for a, b in zip(ps, rs))


def test_bad_tensors_are_refused():
    g = gen(30)
    p, d, st = make(g, (40,), F32, BF16, 32)
    q, e, s8 = make(g, (300,), BF16, BF16, 8)
    call = lambda ps, gs, ss, **kw: adamw.adamw_step(ps, gs, ss, **{**dict(step=1, lr=1e-3), **kw})
    half = torch.zeros(40, device=DEV, dtype=torch.float16)
    bad = [([p, p], [d, d], [st, st]), ([p], [d[:39]], [st]), ([p], [d], [st[::-1] + st]), ([p], [d], [(st[0], st[1][:3])]),
           ([p], [d], [(st[0].double(), st[1])]), ([p], [d], [(st[0].cpu(), st[1])]), ([p], [d.cpu()], [st]),
           ([p[::2]], [d[::2]], [st]), ([p.view(8, 5).t()], [d.view(8, 5).t()], [st]), ([p, q], [d, e], [st, s8]),
           ([q], [e], [(s8[0], s8[1], s8[2][:1])]), ([q], [e], [(s8[0], s8[1], s8[2].int())]),
           ([q], [e], [(s8[0], s8[1].float(), s8[2])]), ([half], [d], [st]), ([p], [half], [st]), ([p], [3], [st]),
           ([p], [d], [None]), ([p.view(8, 5)], [d], [st])]
    for ps, gs, ss in bad:
        with pytest.raises((ValueError, TypeError)):
            call(ps, gs, ss)
    with pytest.raises(ValueError, match="again"):
        call([p, p], [d, d], [st, adamw.new_state(p)])
    for kw in (dict(step=0), dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(eps=float("nan")), dict(weight_decay=-1)):
        with pytest.raises(MuonError):
            call([p], [d], [st], **kw)
    with pytest.raises(ValueError, match="steps"):
        call([p], [d], [st], step=[1, 2])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_state_in_two_places_is_refused(bits):
    g = gen(31)
    p, d, st = make(g, (600,), BF16, BF16, bits)
    q, e, other = make(g, (600,), BF16, BF16, bits)
    before = [t.clone() for t in (p, q, *st, *other)]
    for k in range(len(st)):
        shared = (*other[:k], st[k], *other[k + 1:])
        with pytest.raises(ValueError, match="again"):
            adamw.adamw_step([p, q], [d, e], [st, shared], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="again"):
        adamw.adamw_step([p], [d], [(st[0], st[0], *st[2:])], step=1, lr=1e-3)
    assert all(torch.equal(a, b) for a, b in zip(before, (p, q, *st, *other)))


@pytest.mark.parametrize("bits", [32, 8])
def test_backward_passes_over_stepped_parameters_are_refused(bits):
    """A step writes in place: what autograd saved of a parameter before it is gone."""
    g = gen(40)
    ps = [torch.nn.Parameter(torch.randn(300, generator=g, device=DEV).to(d)) for d in (F32, BF16)]
    idle = torch.nn.Parameter(torch.randn(300, generator=g, device=DEV))
    losses = [(p * p).sum() for p in (*ps, idle)]
    opt = AdamW([*ps, idle], state_bits=bits)
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    for loss in losses[:2]:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    losses[2].backward()      # (no gradient, no step)
    assert torch.equal(idle.grad, 2 * idle.detach())
    # by the function: params of any kind, states too; a refused step writes nothing
    p, d, st = make(g, (40,), F32, F32, bits)
    with torch.inference_mode():
        q, e, other = make(g, (40,), F32, F32, bits)
    kept = [t._version for t in (p, d, *st)]
    with pytest.raises(MuonError):
        adamw.adamw_step([p], [d], [st], step=0, lr=1e-3)
    assert [t._version for t in (p, d, *st)] == kept
    adamw.adamw_step([p, q], (d, e), [st, list(other)], step=1, lr=1e-3)
    assert d._version == kept[1]
    assert all(t._version > k for t, k in zip((p, *st), [kept[0], *kept[2:]]))


def test_the_versions_of_parameters_by_one_check_after_the_other():
    """The same where the tensors are not read by compiled code (a gradient is None)."""
    g = gen(41)
    p, d, st = make(g, (40,), F32, F32, 32)
    q, _, other = make(g, (40,), F32, F32, 32)
    kept = [t._version for t in (p, *st, q, *other)]
    adamw.adamw_step([p, q], [d, None], [st, other], step=1, lr=1e-3)
    now = [t._version for t in (p, *st, q, *other)]
    assert all(a > b for a, b in zip(now[:3], kept[:3])) and now[3:] == kept[3:]


def test_steps_of_more_than_64_bits_are_refused():
    """(Cut to 64 bits they would be others.)"""
    g = gen(42)
    p, d, st = make(g, (40,), F32, F32, 32)
    q, e, other = make(g, (40,), F32, F32, 32)
    before = [t.clone() for t in (p, q, *st, *other)]
    for step in ((1 << 64) + 1, [1, 1 << 63], [-(1 << 63) - 1, 1]):
        with pytest.raises(ValueError, match="64 bits"):
            adamw.adamw_step([p, q], [d, e], [st, other], step=step, lr=1e-3)
    assert all(torch.equal(a, b) for a, b in zip(before, (p, q, *st, *other)))
