"""Performance cases of the layer operators: what a program that trains or
serves with them has them do.

Three operators, those of the layers that hold the matrices the Muon step
updates (sizes from ``paper_2606_27153_amd/workloads.py``: a tiny transformer,
a vision tower, Llama-style 1B and 8B layers, an MoE expert bank; and generic
odd ones):

* ``linear``   y = act(x W + b) + r over [rows, inner] activations
* ``experts``  y_t = x_t W_e, rows sorted by expert, ragged counts per expert
* ``norm``     layer norm over the last dimension

Directions: "forward" as served, "keep" the forward pass of a training step
(with what its backward pass needs), "backward", and "step" for both.
Weights are [in, out], as in the workloads.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_EPS = 1e-5


def _linear(name, rows, inner, outer, **kw):
    c = {"op": "linear", "rows": rows, "inner": inner, "outer": outer, "dtype": "bf16", "direction": "forward",
         "act": "none", "bias": False, "residual": False, "transposed": False}
    return _named(c, name, kw)


def _experts(name, rows, experts, inner, outer, **kw):
    """``idle``: share of the experts that get no row; ``skew``: how uneven
    the others' shares are (0: rows fall on them alike)."""
    c = {"op": "experts", "rows": rows, "experts": experts, "inner": inner, "outer": outer, "dtype": "bf16",
         "direction": "forward", "idle": 0.25, "skew": 0.5}
    return _named(c, name, kw)


def _norm(name, rows, cols, **kw):
    c = {"op": "norm", "rows": rows, "cols": cols, "dtype": "bf16", "direction": "forward", "bias": True}
    return _named(c, name, kw)


def _named(c, name, kw):
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # serving: one token through an 8B layer's gate projection
        _linear("linear_token", 1, 4096, 14336, act="silu"),
        # the tiny transformer in fp32, 8 sequences of 64: a whole training step of its up projection
        _linear("linear_tiny_f32_step", 512, 256, 1024, dtype="f32", direction="step", act="gelu", bias=True),
        # the vision tower's first MLP product in training, 8 images of 27 x 27 patches
        _linear("linear_vision_fc1", 5832, 1152, 4304, direction="keep", act="gelu_tanh", bias=True),
        # the backward pass of the same product
        _linear("linear_vision_fc1_backward", 5832, 1152, 4304, direction="backward", act="gelu_tanh", bias=True),
        # an 8B layer's down projection over a batch of long sequences, added to the residual stream
        _linear("linear_down_8b", 16384, 14336, 4096, residual=True),
        # serving: 8 tokens routed to 6 of 64 experts each
        _experts("experts_decode", 48, 64, 2048, 1408, idle=0.0, skew=0.0),
        # small odd experts in fp32: a whole training step
        _experts("experts_odd_f32_step", 777, 7, 200, 65, dtype="f32", direction="step"),
        # an MoE layer's gate (or up) projection in training, 4096 tokens on 6 of 64 experts each
        _experts("experts_gate", 24576, 64, 2048, 1408),
        # the backward pass of its down projection: input gradient and every expert's weight gradient
        _experts("experts_down_backward", 24576, 64, 1408, 2048, direction="backward"),
        # serving: the norm of one token
        _norm("norm_token", 1, 4096),
        # the vision tower's norm, backward
        _norm("norm_vision_backward", 5832, 1152, direction="backward"),
        # an 8B layer's norm over a batch of long sequences, forward and backward
        _norm("norm_8b_step", 16384, 4096, direction="step"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(step, lo, min(hi // step * step, v))


# the model widths of the workloads
_WIDTHS = (256, 768, 1024, 1152, 1408, 2048, 3456, 4096, 4304, 5632, 14336)
_LARGEST = 1.9e12  # flops of the largest listed case, a little under


def draw(rng):
    """A case of the same ranges: operator, sizes, type, direction, options."""
    while True:
        op = rng.choice(["linear", "linear", "experts", "experts", "norm"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if op == "norm":
            cols = rng.choice([rng.choice(_WIDTHS), _log(rng, 17, 9000)])
            c = _norm(None, _log(rng, 1, 20000), cols, dtype=dtype, bias=rng.random() < 0.8,
                      direction=rng.choice(["forward", "keep", "backward", "step"]))
            if c["rows"] * c["cols"] > 16384 * 4096:
                continue
            return c
        shape = rng.random()
        if shape < 0.55:
            inner, outer = rng.choice(_WIDTHS), rng.choice(_WIDTHS)
        elif shape < 0.8:
            inner, outer = _log(rng, 64, 6000, 8), _log(rng, 64, 6000, 8)
        else:
            inner, outer = _log(rng, 17, 4000), _log(rng, 17, 4000)
        if op == "linear":
            d = rng.choice(["forward", "forward", "keep", "backward", "step"])
            act = rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"])
            if act == "relu" and d == "step":
                act = "silu"   # a step's relu mask hangs on the sign of sums that are zero but for rounding
            c = _linear(None, _log(rng, 1, 16384), inner, outer, dtype=dtype, bias=rng.random() < 0.6,
                        residual=rng.random() < 0.4 and d != "backward", act=act, transposed=rng.random() < 0.25,
                        direction=d)
        else:
            experts = rng.choice([4, 7, 8, 16, 32, 64, 64])
            if experts * inner * outer > 64 * 2048 * 1408:
                continue
            c = _experts(None, _log(rng, 1, 32768), experts, inner, outer, dtype=dtype,
                         idle=rng.choice([0.0, 0.25, 0.5]), skew=rng.choice([0.0, 0.5, 1.5]),
                         direction=rng.choice(["forward", "forward", "backward", "step"]))
        # fp32 matrix products run at a tenth of the bf16 rate or less
        if work(c)["flops"] * (8 if dtype == "f32" else 1) < _LARGEST:
            return c


# ------------------------------------------------------------------- inputs

def _counts(case, seed=0):
    """Rows of each expert: a fixed draw, so that ``work`` can tell which
    experts have rows; the seed permutes the experts."""
    import random
    e, rows = case["experts"], case["rows"]
    rng = random.Random(case["rows"] * 131 + e)
    idle = int(e * case["idle"])
    share = [0.0] * idle + [math.exp(case["skew"] * rng.gauss(0, 1)) for _ in range(e - idle)]
    total = sum(share)
    counts = [0] * e
    pick, acc = [], 0.0
    for s in share:
        acc += s / total
        pick.append(acc)
    for _ in range(rows):
        u = rng.random()
        lo, hi = 0, e - 1
        while lo < hi:
            mid = (lo + hi) // 2
            if pick[mid] > u:
                hi = mid
            else:
                lo = mid + 1
        counts[lo] += 1
    random.Random(seed).shuffle(counts)
    return counts


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 17)
    dt = _DT[case["dtype"]]

    def rand(*shape, scale=1.0, shift=0.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device=dev) * scale + shift).to(dtype)

    d = case["direction"]
    rows = case["rows"]
    st = {"case": case}
    if case["op"] == "norm":
        cols = case["cols"]
        # activations of a residual stream: rows of different scales and offsets
        row = torch.exp(0.5 * torch.randn(rows, 1, generator=g, device=dev))
        st["x"] = (torch.randn(rows, cols, generator=g, device=dev) * row
                   + 0.3 * torch.randn(rows, 1, generator=g, device=dev)).to(dt)
        st["w"] = rand(cols, scale=0.1, shift=1.0)
        st["b"] = rand(cols, scale=0.1) if case["bias"] else None
        if d in ("backward", "step"):
            st["dy"] = rand(rows, cols, scale=0.05)
        if d == "backward":
            xf = st["x"].float()
            st["mean"] = xf.mean(1)
            st["rstd"] = torch.rsqrt((xf - st["mean"][:, None]).pow(2).mean(1) + _EPS)
        return st
    inner, outer = case["inner"], case["outer"]
    st["x"] = rand(rows, inner)
    if d in ("backward", "step"):
        st["dy"] = rand(rows, outer, scale=0.05)
    std = inner ** -0.5
    if case["op"] == "linear":
        # a weight kept as [out, in] comes as its transposed view
        st["w"] = rand(outer, inner, scale=std).t() if case["transposed"] else rand(inner, outer, scale=std)
        st["b"] = rand(outer, scale=0.5) if case["bias"] else None
        st["r"] = rand(rows, outer) if case["residual"] and d != "backward" else None
        if d == "backward":
            st["z"] = rand(rows, outer) if case["act"] != "none" else None
        return st
    st["w"] = rand(case["experts"], inner, outer, scale=std)
    ends = [0]
    for n in _counts(case, seed):
        ends.append(ends[-1] + n)
    st["ends"] = ends
    st["offsets"] = torch.tensor(ends, dtype=torch.int32, device=dev)
    return st


# --------------------------------------------------------------- plain forms

_GELU_C = math.sqrt(2.0 / math.pi)


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(_GELU_C * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_GELU_C * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _GELU_C * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _f(t):
    return None if t is None else t.float()


def _plain_linear(st):
    c = st["case"]
    dt, d, act = _DT[c["dtype"]], c["direction"], c["act"]
    x, w, b = _f(st["x"]), _f(st["w"]), _f(st["b"])
    out = {}
    z = _f(st.get("z"))
    if d != "backward":
        z = x @ w
        if b is not None:
            z = z + b
        y = _act(z, act)
        if st["r"] is not None:
            y = y + st["r"].float()
        out["y"] = y.to(dt)
        if d != "forward" and act != "none":
            out["z"] = z.to(dt)
            z = out["z"].float()
    if d in ("backward", "step"):
        dz = st["dy"].float()
        if act != "none":
            dz = dz * _act_grad(z, act)
        out["dx"] = (dz @ w.t()).to(dt)
        out["dw"] = (x.t() @ dz).to(dt)
        if b is not None:
            out["db"] = dz.sum(0).to(dt)
    return out


def _plain_experts(st):
    c = st["case"]
    dt, d = _DT[c["dtype"]], c["direction"]
    x, w, ends = st["x"], st["w"], st["ends"]
    out = {}
    if d != "backward":
        out["y"] = torch.zeros(c["rows"], c["outer"], dtype=dt, device=x.device)
    if d != "forward":
        out["dx"] = torch.zeros_like(x)
        out["dw"] = torch.zeros_like(w)
    for e in range(c["experts"]):
        lo, hi = ends[e], ends[e + 1]
        if lo == hi:
            continue
        xe, we = x[lo:hi].float(), w[e].float()
        if d != "backward":
            out["y"][lo:hi] = (xe @ we).to(dt)
        if d != "forward":
            dye = st["dy"][lo:hi].float()
            out["dx"][lo:hi] = (dye @ we.t()).to(dt)
            out["dw"][e] = (xe.t() @ dye).to(dt)
    return out


def _plain_norm(st):
    c = st["case"]
    dt, d = _DT[c["dtype"]], c["direction"]
    x, w, b = _f(st["x"]), _f(st["w"]), _f(st["b"])
    out = {}
    if d == "backward":
        mean, rstd = st["mean"], st["rstd"]
    else:
        mean = x.mean(1)
        rstd = torch.rsqrt((x - mean[:, None]).pow(2).mean(1) + _EPS)
    xh = (x - mean[:, None]) * rstd[:, None]
    if d != "backward":
        y = xh * w
        if b is not None:
            y = y + b
        out["y"] = y.to(dt)
        if d != "forward":
            out["mean"], out["rstd"] = mean, rstd
    if d in ("backward", "step"):
        dy = st["dy"].float()
        gx = dy * w
        dx = rstd[:, None] * (gx - gx.mean(1, keepdim=True) - xh * (gx * xh).mean(1, keepdim=True))
        out["dx"] = dx.to(dt)
        out["dw"] = (dy * xh).sum(0).to(dt)
        if b is not None:
            out["db"] = dy.sum(0).to(dt)
    return out


# ----------------------------------------------------------- the framework's

def _own_linear(st):
    from paper_2606_27153_amd import layers
    c = st["case"]
    d, act = c["direction"], c["act"]
    out = {}
    z = st.get("z")
    if d == "forward":
        out["y"] = layers.linear_forward(st["x"], st["w"], bias=st["b"], residual=st["r"], activation=act)
    elif d != "backward":
        out["y"], z = layers.linear_forward(st["x"], st["w"], bias=st["b"], residual=st["r"], activation=act,
                                            keep_preactivation=True)
        if act != "none":
            out["z"] = z
    if d in ("backward", "step"):
        dx, dw, db = layers.linear_backward(st["dy"], st["x"], st["w"], preactivation=z, activation=act,
                                            bias_grad=st["b"] is not None)
        out["dx"], out["dw"] = dx, dw
        if db is not None:
            out["db"] = db
    return out


def _own_experts(st):
    from paper_2606_27153_amd import layers
    d = st["case"]["direction"]
    out = {}
    if d != "backward":
        out["y"] = layers.grouped_linear_forward(st["x"], st["w"], st["offsets"])
    if d != "forward":
        out["dx"], out["dw"] = layers.grouped_linear_backward(st["dy"], st["x"], st["w"], st["offsets"])
    return out


def _own_norm(st):
    from paper_2606_27153_amd import layers
    d = st["case"]["direction"]
    out = {}
    mean, rstd = st.get("mean"), st.get("rstd")
    if d == "forward":
        out["y"] = layers.layer_norm_forward(st["x"], st["w"], st["b"], eps=_EPS)
    elif d != "backward":
        out["y"], mean, rstd = layers.layer_norm_forward(st["x"], st["w"], st["b"], eps=_EPS, keep_stats=True)
        out["mean"], out["rstd"] = mean, rstd
    if d in ("backward", "step"):
        dx, dw, db = layers.layer_norm_backward(st["dy"], st["x"], st["w"], mean, rstd,
                                                bias_grad=st["b"] is not None)
        out["dx"], out["dw"] = dx, dw
        if db is not None:
            out["db"] = db
    return out


_PLAIN = {"linear": _plain_linear, "experts": _plain_experts, "norm": _plain_norm}
_OWN = {"linear": _own_linear, "experts": _own_experts, "norm": _own_norm}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once; an expert's weight only if it has rows."""
    s, d, rows = _SIZE[case["dtype"]], case["direction"], case["rows"]
    fwd, bwd = d != "backward", d in ("backward", "step")
    if case["op"] == "norm":
        n, cols = rows * case["cols"], case["cols"]
        byts = s * ((n if fwd else 0) + (2 * n if bwd else 0) + (n if fwd and not bwd else 0) + (n if d == "step" else 0))
        byts += s * cols * (4 if bwd else 2) + (8 * rows if d != "forward" else 0)
        return {"bytes": byts, "flops": n * ((7 if fwd else 0) + (12 if bwd else 0))}
    k, n = case["inner"], case["outer"]
    flops = 2 * rows * k * n * (int(fwd) + 2 * int(bwd))
    el = rows * k + (rows * n if fwd else 0) + (rows * n + rows * k if bwd else 0)
    if case["op"] == "linear":
        el += k * n * (1 + int(bwd))
        el += n * (1 + int(bwd)) if case["bias"] else 0
        el += rows * n if case["residual"] and fwd else 0
        el += rows * n if case["act"] != "none" and d != "forward" else 0   # the pre-activation, written or read
        return {"bytes": s * el, "flops": flops}
    routed = sum(c > 0 for c in _counts(case))
    el += k * n * (routed + (case["experts"] if bwd else 0))
    return {"bytes": s * el + 4 * (case["experts"] + 1), "flops": flops}


# --------------------------------------------------------------------- exact

def exact(case, seed):
    """The outputs in 64 bits, from the definitions."""
    st = prepare(case, seed)
    d = case["direction"]
    f = {k: v.double() for k, v in st.items() if torch.is_tensor(v) and v.is_floating_point()}
    out = {}
    if case["op"] == "norm":
        x, w = f["x"], f["w"]
        # the statistics a backward pass is handed are inputs
        mu = f["mean"][:, None] if d == "backward" else x.sum(1, keepdim=True) / x.shape[1]
        c = x - mu
        sd = 1.0 / f["rstd"][:, None] if d == "backward" else torch.sqrt((c * c).sum(1, keepdim=True) / x.shape[1] + _EPS)
        h = c / sd
        if d != "backward":
            out["y"] = torch.addcmul(f["b"] if "b" in f else torch.zeros_like(w), h, w)
            if d != "forward":
                out["mean"], out["rstd"] = mu[:, 0], 1.0 / sd[:, 0]
        if d in ("backward", "step"):
            p = f["dy"] * w
            n = x.shape[1]
            out["dx"] = (p - (p.sum(1, keepdim=True) + h * (p * h).sum(1, keepdim=True)) / n) / sd
            out["dw"] = (f["dy"] * h).sum(0)
            if "b" in f:
                out["db"] = f["dy"].sum(0)
        return out
    if case["op"] == "linear":
        x, w = f["x"], f["w"]
        z = f.get("z")
        act = case["act"]
        if d != "backward":
            z = torch.addmm(f["b"], x, w) if "b" in f else x.mm(w)
            y = _exact_act(z, act)[0]
            out["y"] = y + f["r"] if "r" in f else y
            if d != "forward" and act != "none":
                out["z"] = z
                # the backward pass reads the pre-activation as it is kept
                z = z.to(_DT[case["dtype"]]).double()
        if d in ("backward", "step"):
            dz = f["dy"] if act == "none" else f["dy"] * _exact_act(z, act)[1]
            out["dx"] = dz.mm(w.t())
            out["dw"] = x.t().mm(dz)
            if "b" in f:
                out["db"] = dz.sum(0)
        return out
    x, w = f["x"], f["w"]
    if d != "backward":
        out["y"] = torch.zeros(case["rows"], case["outer"], dtype=torch.float64, device=x.device)
    if d != "forward":
        out["dx"], out["dw"] = torch.zeros_like(x), torch.zeros_like(w)
    for e, (lo, hi) in enumerate(zip(st["ends"][:-1], st["ends"][1:])):
        if d != "backward":
            out["y"][lo:hi] = x[lo:hi].mm(w[e])
        if d != "forward":
            out["dx"][lo:hi] = f["dy"][lo:hi].mm(w[e].t())
            out["dw"][e] = x[lo:hi].t().mm(f["dy"][lo:hi])
    return out


def _exact_act(z, act):
    """The activation and its derivative."""
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        s = torch.special.expit(2 * _GELU_C * (z + 0.044715 * z ** 3))
        return z * s, s + z * s * (1 - s) * 2 * _GELU_C * (1 + 0.134145 * z ** 2)
    if act == "silu":
        s = torch.special.expit(z)
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)
