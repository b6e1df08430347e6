"""Performance cases of the operators at the two ends of a model and between
its experts: what a program that trains or serves with them has them do.

* ``loss``    softmax cross entropy of x W over a vocabulary, with its gradients
* ``embed``   lookup of a table's rows by token, scaled, and the table's gradient
* ``route``   tokens sorted by expert, handed to the experts and brought back
              weighted, and the gradients of both ways
* ``adamw``   an AdamW step over the parameters that the Muon step leaves out
              (tables, norms, biases), with states in 32 bits or in 8

Widths, experts and row counts are those of ``paper_2606_27153_amd/workloads.py``
(a tiny transformer, Llama-style 1B and 8B layers, an MoE expert bank) or generic
odd ones; vocabularies are generic (the workloads have none).  Directions:
"forward" as served, "backward", and "step" for both.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_IGNORE = -100
_BLOCK = 256          # elements of an 8-bit state that share a scale
_LR, _BETAS, _ADAM_EPS, _DECAY = 1e-3, (0.9, 0.95), 1e-8, 0.1


def _loss(name, rows, width, vocab, **kw):
    """``ignored``: share of the rows without a target; ``tied``: the weight is
    the transposed view of an embedding table."""
    c = {"op": "loss", "rows": rows, "width": width, "vocab": vocab, "dtype": "bf16", "direction": "step",
         "reduction": "mean", "ignored": 0.1, "tied": False}
    return _named(c, name, kw)


def _embed(name, rows, width, vocab, **kw):
    """``skew``: the exponent by which tokens grow rarer with their rank."""
    c = {"op": "embed", "rows": rows, "width": width, "vocab": vocab, "dtype": "bf16", "direction": "step",
         "skew": 1.0}
    return _named(c, name, kw)


def _route(name, tokens, top, experts, width, **kw):
    """``skew``: how uneven the experts' shares are; ``dropped``: share of the
    tokens' choices that go to no expert."""
    c = {"op": "route", "tokens": tokens, "top": top, "experts": experts, "width": width, "dtype": "bf16",
         "direction": "step", "skew": 0.5, "dropped": 0.0, "residual": True}
    return _named(c, name, kw)


def _adamw(name, tables, vocab, width, layers, **kw):
    """``tables`` matrices of vocab x width, and per layer ``vectors`` vectors of
    width elements and, with ``biases``, one of 4 width + 1."""
    c = {"op": "adamw", "tables": tables, "vocab": vocab, "width": width, "layers": layers, "vectors": 2,
         "biases": False, "params": "bf16", "grads": "bf16", "bits": 32}
    return _named(c, name, kw)


def _named(c, name, kw):
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # serving: the log probability of one given token under an 8B model's head
        _loss("loss_token", 1, 4096, 128000, direction="forward", reduction="none", ignored=0.0, tied=True),
        # a small odd model in fp32, rows weighted one by one: a whole training step
        _loss("loss_odd_f32_step", 777, 200, 5003, dtype="f32", reduction="none"),
        # a 1B model's head that shares its table with the embedding, two sequences of 2048
        _loss("loss_1b_step", 4096, 2048, 32000, tied=True),
        # an 8B model's head over a batch of long sequences
        _loss("loss_8b_step", 16384, 4096, 128000),
        # serving: the embedding of a decode batch
        _embed("embed_token", 8, 4096, 128000, direction="forward"),
        # an 8B model's table in training, a batch of long sequences
        _embed("embed_8b_step", 32768, 4096, 128000),
        # serving: 8 tokens routed to 6 of 64 experts each
        _route("route_decode", 8, 6, 64, 2048, direction="forward", skew=0.0),
        # small odd experts in fp32 with choices that capacity dropped: a whole training step
        _route("route_odd_f32_step", 1001, 3, 7, 333, dtype="f32", dropped=0.2, residual=False),
        # an MoE layer in training, 4 sequences of 4096 on 6 of 64 experts each
        _route("route_moe_step", 16384, 6, 64, 2048),
        # the tiny transformer's norms and biases in fp32
        _adamw("adamw_tiny_f32", 0, 0, 256, 4, vectors=4, biases=True, params="f32", grads="f32"),
        # a 1B model's embedding, head and norms
        _adamw("adamw_1b", 2, 32000, 2048, 16),
        # an 8B model's embedding and norms, states in 8 bits
        _adamw("adamw_8b_8bit", 1, 128000, 4096, 32, bits=8),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(step, lo, min(hi // step * step, v))


# the model widths of the workloads
_WIDTHS = (256, 768, 1024, 1152, 1408, 2048, 4096)
_VOCABS = (32000, 50001, 65536, 128000)


def draw(rng):
    """A case of the same ranges: operator, sizes, type, direction, options."""
    while True:
        op = rng.choice(["loss", "loss", "embed", "route", "adamw"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        width = rng.choice([rng.choice(_WIDTHS), _log(rng, 64, 4096, 8), _log(rng, 17, 4000)])
        vocab = rng.choice([rng.choice(_VOCABS), _log(rng, 300, 128000)])
        if op == "loss":
            c = _loss(None, _log(rng, 1, 16384), width, vocab, dtype=dtype, direction=rng.choice(["forward", "step"]),
                      reduction=rng.choice(["mean", "sum", "none"]), ignored=rng.choice([0.0, 0.1, 0.6]),
                      tied=rng.random() < 0.5)
            # fp32 matrix products run at a tenth of the bf16 rate or less
            if work(c)["flops"] * (8 if dtype == "f32" else 1) < 4e13:
                return c
        elif op == "embed":
            c = _embed(None, _log(rng, 1, 65536), width, vocab, dtype=dtype, skew=rng.choice([0.0, 1.0, 1.5]),
                       direction=rng.choice(["forward", "backward", "step"]))
            if work(c)["bytes"] < 1.9e9:
                return c
        elif op == "route":
            experts = rng.choice([4, 7, 8, 16, 64, 64, 128])
            c = _route(None, _log(rng, 1, 32768), rng.randint(1, min(8, experts)), experts, width, dtype=dtype,
                       skew=rng.choice([0.0, 0.5, 1.5]), dropped=rng.choice([0.0, 0.0, 0.2]),
                       residual=rng.random() < 0.5, direction=rng.choice(["forward", "step"]))
            if work(c)["bytes"] < 3e9:
                return c
        else:
            tables = rng.choice([0, 1, 2])
            c = _adamw(None, tables, vocab if tables else 0, width, rng.randint(1, 40), vectors=rng.randint(1, 6),
                       biases=rng.random() < 0.5, params=dtype, grads=rng.choice(["bf16", dtype]),
                       bits=rng.choice([8, 32]))
            if work(c)["bytes"] < 6e9:
                return c


# ------------------------------------------------------------------- inputs

def _shapes(case):
    """The tensors of an AdamW step."""
    s = [(case["vocab"], case["width"])] * case["tables"]
    for _ in range(case["layers"]):
        s += [(case["width"],)] * case["vectors"]
        if case["biases"]:
            s.append((4 * case["width"] + 1,))
    return s


def _starts(shapes):
    """Where each tensor starts in one flat buffer, whole blocks each, and its elements."""
    at, out = 0, []
    for s in shapes:
        n = math.prod(s)
        out.append((at, n))
        at += -(-n // _BLOCK) * _BLOCK
    return out, at


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 17)

    def rand(*shape, dtype, scale=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev)

    st = {"case": case}
    d = case.get("direction")
    if case["op"] == "adamw":
        return _prepare_adamw(case, st, seed, rand, dev)
    dt = _DT[case["dtype"]]
    if case["op"] == "loss":
        rows, width, vocab = case["rows"], case["width"], case["vocab"]
        # logits of a model in training: a few units wide
        st["x"] = rand(rows, width, dtype=dt)
        std = 2.0 * width ** -0.5
        st["w"] = rand(vocab, width, dtype=dt, scale=std).t() if case["tied"] else rand(width, vocab, dtype=dt, scale=std)
        t = torch.randint(vocab, (rows,), generator=g, device=dev)
        st["t"] = torch.where(uniform(rows) < case["ignored"], torch.full_like(t, _IGNORE), t)
        if d == "step":
            # the upstream gradient: one number, or a weight for each row
            st["dloss"] = torch.ones((), device=dev) if case["reduction"] != "none" else uniform(rows) + 0.5
        return st
    if case["op"] == "embed":
        rows, width, vocab = case["rows"], case["width"], case["vocab"]
        # tokens by rank: u^(1 / (1 - s)) grows rarer as rank^-s; s = 1 is the limit vocab^u
        u, s = uniform(rows).double(), case["skew"]
        rank = vocab * u if s == 0 else vocab ** u - 1 if s == 1 else (u * (vocab ** (1 - s) - 1) + 1) ** (1 / (1 - s)) - 1
        rank = rank.long().clamp_(0, vocab - 1)
        # ranks lie anywhere in the table, as in a vocabulary that is not sorted by frequency
        st["ids"] = torch.randperm(vocab, generator=g, device=dev)[rank]
        st["scale"] = float(width) ** 0.5
        if d != "backward":
            st["w"] = rand(vocab, width, dtype=dt, scale=0.02)
        if d != "forward":
            st["dy"] = rand(rows, width, dtype=dt, scale=0.05)
        return st
    tokens, top, experts, width = case["tokens"], case["top"], case["experts"], case["width"]
    score = torch.randn(tokens, experts, generator=g, device=dev) + \
        case["skew"] * torch.randn(experts, generator=g, device=dev)
    weight, expert = torch.topk(torch.softmax(score, dim=-1), top, dim=-1)
    st["experts"] = torch.where(uniform(tokens, top) < case["dropped"], torch.full_like(expert, -1), expert)
    st["weights"] = weight / weight.sum(-1, keepdim=True)
    st["x"] = rand(tokens, width, dtype=dt)
    st["h"] = rand(tokens * top, width, dtype=dt)       # what the experts make of their rows
    st["r"] = rand(tokens, width, dtype=dt) if case["residual"] else None
    if d == "step":
        st["dy"] = rand(tokens, width, dtype=dt, scale=0.05)
        st["drows"] = rand(tokens * top, width, dtype=dt, scale=0.05)   # what comes back through the experts
    return st


def _prepare_adamw(case, st, seed, rand, dev):
    shapes = _shapes(case)
    where, total = _starts(shapes)
    cut = lambda t: [t[a:a + n].view(s) for (a, n), s in zip(where, shapes)]
    st["seed"], st["step"] = seed % 100000 + 1, 1000
    # between the tensors, up to whole blocks, everything is 0 and stays so
    used = torch.cat([torch.arange(-(-n // _BLOCK) * _BLOCK, device=dev, dtype=torch.int32) < n for _, n in where])
    st["p"] = rand(total, dtype=_DT[case["params"]], scale=0.02).mul_(used)
    st["g"] = rand(total, dtype=_DT[case["grads"]], scale=1e-3).mul_(used)
    m = rand(total, dtype=torch.float32, scale=3e-4).mul_(used)
    v = rand(total, dtype=torch.float32, scale=1e-3).square_().add_(1e-8).mul_(used)
    st["params"], st["grads"] = cut(st["p"]), cut(st["g"])
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
        st["states"] = list(zip(cut(m), cut(v)))
        return st
    half = torch.full((), 1 << 19, dtype=torch.int32, device=dev)
    st["m"], bm = _encode(m, half, 127, True)
    st["v"], bv = _encode(v, half, 255, False)
    st["scales"] = torch.stack([bm, bv], 1).contiguous()
    flat = lambda t: [t[a:a + n] for a, n in where]
    blocks = [(a // _BLOCK, -(-n // _BLOCK)) for a, n in where]
    st["states"] = list(zip(flat(st["m"]), flat(st["v"]), [st["scales"][a:a + n] for a, n in blocks]))
    # where each element lies in its own tensor, and which tensor that is
    st["index"] = torch.cat([torch.arange(-(-n // _BLOCK) * _BLOCK, device=dev, dtype=torch.int32) for _, n in where])
    st["tensor"] = torch.cat([torch.full((n,), i, device=dev, dtype=torch.int32) for i, (_, n) in enumerate(blocks)])
    return st


# --------------------------------------------------------------- plain forms

def _plain_loss(st):
    c = st["case"]
    dt = _DT[c["dtype"]]
    x, w, t = st["x"].float(), st["w"].float(), st["t"]
    live = (t >= 0) & (t < c["vocab"]) & (t != _IGNORE)
    at = torch.where(live, t, torch.zeros_like(t))[:, None]
    z = x @ w
    top = z.max(1, keepdim=True).values
    e = (z - top).exp_()
    total = e.sum(1, keepdim=True)
    rows = torch.where(live, (top + total.log() - z.gather(1, at))[:, 0], torch.zeros_like(top[:, 0]))
    count = live.sum().clamp(min=1)
    out = {"loss": rows if c["reduction"] == "none" else rows.sum() / (count if c["reduction"] == "mean" else 1)}
    if c["direction"] == "step":
        del z
        dloss = st["dloss"] / (count if c["reduction"] == "mean" else 1)
        dz = e.div_(total)
        dz.scatter_add_(1, at, torch.full_like(top, -1.0))
        dz *= torch.where(live, dloss, torch.zeros_like(rows))[:, None]
        out["dx"] = (dz @ w.t()).to(dt)
        out["dw"] = (dz.t() @ x).t().to(dt) if c["tied"] else (x.t() @ dz).to(dt)
    return out


def _plain_embed(st):
    c = st["case"]
    dt, d, ids = _DT[c["dtype"]], c["direction"], st["ids"]
    out = {}
    if d != "backward":
        out["y"] = (st["w"][ids].float() * st["scale"]).to(dt)
    if d != "forward":
        dw = torch.zeros(c["vocab"], c["width"], dtype=torch.float32, device=ids.device)
        dw.index_add_(0, ids, st["dy"].float())
        out["dw"] = (dw * st["scale"]).to(dt)
    return out


def _plain_route(st):
    c = st["case"]
    dt, top, experts = _DT[c["dtype"]], c["top"], c["experts"]
    e, weights = st["experts"].flatten(), st["weights"]
    n = e.numel()
    # choices sorted by expert, in the tokens' order within each; those of no expert come last
    key = torch.where(e >= 0, e, torch.full_like(e, experts))
    order = torch.sort(key, stable=True).indices
    bounds = torch.arange(experts + 1, device=e.device)
    offsets = (key[None, :] < bounds[:, None]).sum(1).to(torch.int32)
    place = torch.empty_like(order)
    place[order] = torch.arange(n, device=e.device)
    live = e >= 0
    out = {"offsets": offsets, "position": torch.where(live, place, torch.full_like(place, -1)).to(torch.int32)}
    used = (torch.arange(n, device=e.device) < offsets[-1])[:, None]
    token = order // top
    zero = torch.zeros((), dtype=torch.float32, device=e.device)
    out["rows"] = torch.where(used, st["x"][token].float(), zero).to(dt)

    def back(rows, scale):
        r = torch.where(live[:, None], rows[place].float() * scale.reshape(-1, 1), zero)
        return r.view(c["tokens"], top, -1).sum(1)

    y = back(st["h"], weights)
    out["y"] = (y if st["r"] is None else y + st["r"].float()).to(dt)
    if c["direction"] == "step":
        dy = st["dy"].float()
        out["dh"] = torch.where(used, dy[token] * weights.flatten()[order][:, None], zero).to(dt)
        dots = (st["h"][place].float() * dy.repeat_interleave(top, 0)).sum(1)
        out["dweights"] = torch.where(live, dots, zero).view(weights.shape)
        out["dx"] = back(st["drows"], torch.ones_like(weights)).to(dt)
    return out


def _mix(h):
    """A hash of 32 bits in the low half of int64."""
    m = 0xFFFFFFFF
    h = h ^ (h >> 16)
    h = (h * 0x6A09E667) & m
    h = h ^ (h >> 15)
    h = (h * 0xBB67AE85) & m
    return h ^ (h >> 16)


def _decode(code, base, signed):
    """The values that codes of 8 bits stand for: with a block's base, the upper 12
    bits of a number in fp32 (code 0 is 0)."""
    c = code.int()
    size = c & 127 if signed else c
    bits = torch.where(size > 0, (size + base.int().repeat_interleave(_BLOCK)) << 20, torch.zeros_like(size))
    value = bits.view(torch.float32)
    return torch.where(c > 127, -value, value) if signed else value


def _encode(value, add, top, signed):
    """(codes, bases) of values: ``add`` (below 2^20) to the bits, then the upper 12
    of them.  The block's largest value gets one of the two topmost codes, what is
    too small for code 1 gets 0; a square's average that is not 0 gets 1."""
    bits = value.view(torch.int32) & 0x7FFFFFFF
    base = ((bits.view(-1, _BLOCK).max(1).values >> 20) + 1 - top).clamp_(0, 2047 - top)
    size = ((bits + add) >> 20) - base.repeat_interleave(_BLOCK)
    size = size.clamp_(max=top)
    size = size.clamp_(min=0) if signed else torch.maximum(size, (bits != 0).int())
    if signed:
        size = size + torch.where((value < 0) & (size > 0), 128, 0)
    return size.to(torch.uint8), base.to(torch.int16)


def _plain_adamw(st):
    c = st["case"]
    (b1, b2), step = _BETAS, st["step"]
    p, g = st["p"].float(), st["g"].float()
    small = c["bits"] == 8
    m = _decode(st["m"], st["scales"][:, 0], True) if small else st["m"]
    v = _decode(st["v"], st["scales"][:, 1], False) if small else st["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    denom = v.sqrt() / math.sqrt(1 - b2 ** step) + _ADAM_EPS
    st["p"].copy_(p * (1 - _LR * _DECAY) - (_LR / (1 - b1 ** step)) * m / denom)
    if not small:
        st["m"].copy_(m)
        st["v"].copy_(v)
        return {"p": st["p"], "m": st["m"], "v": st["v"]}
    del p, g, denom
    first = torch.full((), (st["seed"] + step * 0x9E3779B9) & 0xFFFFFFFF, dtype=torch.int64, device=m.device)
    key = _mix((_mix(first) + st["tensor"].long()) & 0xFFFFFFFF).repeat_interleave(_BLOCK)
    h = _mix(((st["index"].long() * 0x9E3779B1) & 0xFFFFFFFF) ^ key)
    del key
    code, bm = _encode(m, ((h & 0xFFFF) << 4).int(), 127, True)
    st["m"].copy_(code)
    code, bv = _encode(v, ((h >> 16) << 4).int(), 255, False)
    st["v"].copy_(code)
    st["scales"].copy_(torch.stack([bm, bv], 1))
    del h, m, v, code
    return {"p": st["p"], "m": _decode(st["m"], bm, True).to(torch.bfloat16),
            "v": _decode(st["v"], bv, False).to(torch.bfloat16)}


# ----------------------------------------------------------- the framework's

def _own_loss(st):
    from paper_2606_27153_amd import layers
    c = st["case"]
    loss, lse = layers.linear_cross_entropy_forward(st["x"], st["w"], st["t"], reduction=c["reduction"],
                                                    ignore_index=_IGNORE)
    out = {"loss": loss}
    if c["direction"] == "step":
        out["dx"], out["dw"] = layers.linear_cross_entropy_backward(
            st["dloss"], st["x"], st["w"], st["t"], lse, reduction=c["reduction"], ignore_index=_IGNORE)
    return out


def _own_embed(st):
    from paper_2606_27153_amd import layers
    c = st["case"]
    out = {}
    if c["direction"] != "backward":
        out["y"] = layers.embedding_forward(st["ids"], st["w"], scale=st["scale"])
    if c["direction"] != "forward":
        out["dw"] = layers.embedding_backward(st["dy"], st["ids"], c["vocab"], scale=st["scale"])
    return out


def _own_route(st):
    from paper_2606_27153_amd import layers
    c = st["case"]
    routing = layers.sort_by_expert(st["experts"], c["experts"])
    out = {"offsets": routing.offsets, "position": routing.position.view(-1)}
    out["rows"] = layers.dispatch_forward(st["x"], routing)
    out["y"] = layers.combine_forward(st["h"], st["weights"], routing, residual=st["r"])
    if c["direction"] == "step":
        out["dh"], out["dweights"] = layers.combine_backward(st["dy"], st["h"], st["weights"], routing)
        out["dx"] = layers.dispatch_backward(st["drows"], routing)
    return out


def _own_adamw(st):
    from paper_2606_27153_amd import adamw
    c = st["case"]
    adamw.adamw_step(st["params"], st["grads"], st["states"], step=st["step"], lr=_LR, betas=_BETAS, eps=_ADAM_EPS,
                     weight_decay=_DECAY, seed=st["seed"])
    if c["bits"] == 32:
        return {"p": st["p"], "m": st["m"], "v": st["v"]}
    m, v = adamw.state_values((st["m"], st["v"], st["scales"]))
    return {"p": st["p"], "m": m, "v": v}


_PLAIN = {"loss": _plain_loss, "embed": _plain_embed, "route": _plain_route, "adamw": _plain_adamw}
_OWN = {"loss": _own_loss, "embed": _own_embed, "route": _own_route, "adamw": _own_adamw}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once; of a table only the rows that are looked up."""
    step = case.get("direction") == "step"
    if case["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        # parameter and gradient; both states read and written, the scales of 8-bit
        # ones too, and their values as they are returned
        state = 16 if case["bits"] == 32 else 4 + 4 + 8 / _BLOCK
        return {"bytes": int(n * (2 * _SIZE[case["params"]] + _SIZE[case["grads"]] + state)),
                "flops": n * (14 if case["bits"] == 32 else 40)}
    s = _SIZE[case["dtype"]]
    if case["op"] == "loss":
        rows, width, vocab = case["rows"], case["width"], case["vocab"]
        el = rows * width + width * vocab
        return {"bytes": s * el * (2 if step else 1) + 12 * rows,
                "flops": rows * vocab * ((6 if step else 2) * width + (8 if step else 5))}
    if case["op"] == "embed":
        rows, width, vocab, d = case["rows"], case["width"], case["vocab"], case["direction"]
        el = (2 * rows * width if d != "backward" else 0) + ((rows + vocab) * width if d != "forward" else 0)
        return {"bytes": s * el + 8 * rows, "flops": rows * width * ((d != "backward") + (d != "forward"))}
    tokens, top, width = case["tokens"], case["top"], case["width"]
    t, n = tokens * width, tokens * top * width
    el = t + n + n + t + (t if case["residual"] else 0)
    if step:
        el += t + n + n + t     # dy, dh, drows, dx (the experts' outputs are read above)
    return {"bytes": int(s * el + tokens * top * (8 + 4 + 4 + (4 if step else 0))),
            "flops": 2 * n + (4 * n if step else 0)}


# --------------------------------------------------------------------- exact

def exact(case, seed):
    """The outputs in 64 bits, from the definitions."""
    st = prepare(case, seed)
    step = case.get("direction") == "step"
    out = {}
    if case["op"] == "loss":
        x, w, t = st["x"].double(), st["w"].double(), st["t"]
        live = t != _IGNORE
        z = x.mm(w)
        lse = torch.logsumexp(z, 1)
        row = torch.arange(case["rows"], device=t.device)[live]
        loss = torch.zeros_like(lse)
        loss[row] = lse[row] - z[row, t[row]]
        n = max(1, int(live.sum())) if case["reduction"] == "mean" else 1
        out["loss"] = loss if case["reduction"] == "none" else loss.sum() / n
        if step:
            dz = z.sub_(lse[:, None]).exp_()
            dz[row, t[row]] -= 1
            dz *= (live.double() * st["dloss"].double() / n)[:, None]
            out["dx"] = dz.mm(w.t())
            out["dw"] = x.t().mm(dz)
        return out
    if case["op"] == "embed":
        ids = st["ids"]
        if case["direction"] != "backward":
            out["y"] = st["scale"] * torch.index_select(st["w"], 0, ids).double()
        if case["direction"] != "forward":
            dw = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device=ids.device)
            out["dw"] = dw.index_put_((ids,), st["scale"] * st["dy"].double(), accumulate=True)
        return out
    if case["op"] == "route":
        return _exact_route(case, st, step)
    (b1, b2), k = _BETAS, st["step"]
    small = case["bits"] == 8
    g = st["g"].double()
    m = (_decode(st["m"], st["scales"][:, 0], True) if small else st["m"]).double()
    v = (_decode(st["v"], st["scales"][:, 1], False) if small else st["v"]).double()
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g.square(), v, b2)
    # which of two codes an average gets is decided by rounding, which 64 bits do not have
    out["m"], out["v"] = (None, None) if small else (m, v)
    p = st["p"].double()
    out["p"] = p - _LR * (_DECAY * p + (m / (1 - b1 ** k)) / ((v / (1 - b2 ** k)).sqrt() + _ADAM_EPS))
    return out


def _exact_route(case, st, step):
    """One expert's choices after another's."""
    tokens, top = case["tokens"], case["top"]
    e, w = st["experts"].reshape(-1), st["weights"].double().reshape(-1)
    slots = torch.cat([torch.nonzero(e == i)[:, 0] for i in range(case["experts"])])
    n, token = slots.numel(), slots // top
    counts = torch.bincount(e[slots], minlength=case["experts"])
    out = {"offsets": torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()}
    out["position"] = torch.full_like(e, -1, dtype=torch.int32)
    out["position"][slots] = torch.arange(n, device=e.device, dtype=torch.int32)
    grown = lambda r: torch.cat([r, r.new_zeros(tokens * top - n, r.shape[1])])
    gathered = lambda r: torch.zeros(tokens, case["width"], dtype=torch.float64, device=e.device).index_add_(0, token, r)
    out["rows"] = grown(st["x"].double()[token])
    h = st["h"].double()[:n]
    out["y"] = gathered(h * w[slots][:, None])
    if st["r"] is not None:
        out["y"] += st["r"].double()
    if step:
        dy = st["dy"].double()[token]
        out["dh"] = grown(dy * w[slots][:, None])
        out["dweights"] = torch.zeros_like(w)
        out["dweights"][slots] = (dy * h).sum(1)
        out["dweights"] = out["dweights"].view(tokens, top)
        out["dx"] = gathered(st["drows"].double()[:n])
    return out
