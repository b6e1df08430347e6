"""Reference in 64 bits of the operators that take token or expert numbers, with
bounds on how far fp32 arithmetic and the roundings may be from it.

As in layers_ref: a sum of n terms in fp32, in any order, is within n u S of the
exact one (u = 2^-24, S the sum of the absolute values), a few more roundings
are covered by n + 8, and rounding to a type of p significant bits adds 2^-p.
"""
import torch

from layers_ref import ROUND, U

# exp on the GPU: its argument is rounded after the factor log2(e), which a result
# passes on |argument| times, and the instruction is good to a few units
EXP = 2.0 ** -21


def exp_error(arg):
    """Relative error of exp(arg), arg an exact difference of two fp32 numbers of the logits' size."""
    return EXP + arg.abs() * 2.0 ** -22


def rounded(value, err, dtype):
    return value, err + ROUND[dtype] * (value.abs() + err) + 1e-300


def embedding_forward(ids, w, scale):
    live = (ids >= 0) & (ids < w.shape[0])
    y = w.double()[torch.where(live, ids, 0).long()] * scale * live[..., None]
    return rounded(y, 2 * U * y.abs(), w.dtype)     # the scale's own rounding, the product's


def embedding_backward(dy, ids, vocab, scale):
    cols = dy.shape[-1]
    ids, g = ids.reshape(-1).long(), dy.reshape(-1, cols).double()
    live = (ids >= 0) & (ids < vocab)
    ids, g = ids[live], g[live]
    add = lambda v: torch.zeros(vocab, cols, dtype=torch.float64, device=g.device).index_put_((ids,), v, accumulate=True)
    n = torch.bincount(ids, minlength=vocab)[:, None].double()
    dw, s = add(g) * scale, add(g.abs()) * abs(scale)
    return rounded(dw, (n + 8) * U * s, dy.dtype)


def route(experts, count):
    """(offsets, position, source) on the CPU, one choice after another."""
    e = experts.cpu().reshape(-1).tolist()
    lists = [[i for i, v in enumerate(e) if v == x] for x in range(count)]
    order = [i for l in lists for i in l]
    offsets = [0]
    for l in lists:
        offsets.append(offsets[-1] + len(l))
    position = [-1] * len(e)
    for r, i in enumerate(order):
        position[i] = r
    nobody = [~i for i, v in enumerate(e) if not 0 <= v < count]
    as_int = lambda v: torch.tensor(v, dtype=torch.int32)
    return as_int(offsets), as_int(position).view(experts.shape), as_int(order + nobody)


def dispatch(x, position):
    tokens, top = position.shape
    rows = torch.zeros(tokens * top, x.shape[1], dtype=x.dtype, device=x.device)
    live = position >= 0
    rows[position[live].long()] = x.repeat_interleave(top, 0).view(tokens, top, x.shape[1])[live]
    return rows


def gather(rows, position, weights=None, residual=None):
    """(value, bound) of y[t] = residual[t] + sum of weights[t, j] rows[position[t, j]]."""
    tokens, top = position.shape
    live = position >= 0
    r = torch.where(live[..., None], rows.double()[position.clamp(min=0).long()], 0.0)   # [tokens, top, cols]
    if weights is not None:
        r = r * torch.where(live, weights.double(), 0.0)[..., None]
    y, s = r.sum(1), r.abs().sum(1)
    if residual is not None:
        y, s = y + residual.double(), s + residual.double().abs()
    return rounded(y, (top + 8) * U * s, rows.dtype)


def combine_backward(dy, rows, weights, position):
    """{"drows", "dweights"}: (value, bound)."""
    tokens, top = position.shape
    live = position >= 0
    g = dy.double()[:, None].expand(tokens, top, -1)
    w = torch.where(live, weights.double(), 0.0)[..., None]
    drows = torch.zeros(tokens * top, dy.shape[1], dtype=torch.float64, device=dy.device)
    drows[position[live].long()] = (g * w)[live]
    r = rows.double()[position.clamp(min=0).long()]
    dots = torch.where(live[..., None], g * r, 0.0)
    return {"drows": rounded(drows, U * drows.abs(), dy.dtype),
            "dweights": rounded(dots.sum(-1), (dy.shape[1] + 8) * U * dots.abs().sum(-1), weights.dtype)}


class Loss:
    """Softmax cross entropy of x w in 64 bits; targets None of which count where ``live`` is false."""

    def __init__(self, x, w, targets, ignore=-100):
        self.x, self.w = x.double(), w.double()
        self.dtype = x.dtype
        k, v = w.shape
        self.live = (targets >= 0) & (targets < v) & (targets != ignore)
        self.at = torch.where(self.live, targets, 0).long()[:, None]
        self.z = self.x @ self.w
        self.ez = (k + 8) * U * (self.x.abs() @ self.w.abs())          # of the logits
        self.lse = torch.logsumexp(self.z, 1)
        p = torch.exp(self.z - self.lse[:, None])
        # sums of V exponentials: each thread's, the lanes', the waves', then the strips of at least 64 columns
        chain = (128 + v / 64) * U
        far = (self.z.max(1, keepdim=True).values - self.z)
        self.lse_error = (p * (self.ez + exp_error(far))).sum(1) + self.ez.max(1).values + chain + 4 * U * (1 + self.lse.abs())
        # (the largest logit's own error moves the reference and the terms alike; it is counted once more)
        self.p = p
        self.count = int(self.live.sum())

    def rows(self):
        loss = torch.where(self.live, self.lse - self.z.gather(1, self.at)[:, 0], 0.0)
        err = torch.where(self.live, self.lse_error + self.ez.gather(1, self.at)[:, 0] + 2 * U * loss.abs(), 0.0)
        return loss, err + 1e-300

    def total(self, reduction):
        loss, err = self.rows()
        n = max(1, self.count) if reduction == "mean" else 1
        return loss.sum() / n, (err.sum() + (loss.numel() + 8) * U * loss.abs().sum()) / n + 1e-300

    def backward(self, dloss, reduction):
        """{"dx", "dw"}: (value, bound)."""
        q = ROUND[self.dtype]
        dz = self.p.clone()
        dz.scatter_add_(1, self.at, torch.full_like(self.lse[:, None], -1.0))
        e = self.p * (self.ez + self.lse_error[:, None] + exp_error(self.z - self.lse[:, None])) + 2 * U * dz.abs()
        live = self.live.double()[:, None]
        scale = dloss.double()
        if reduction == "none":
            dz, e, f = dz * scale[:, None], e * scale.abs()[:, None], 1.0
        else:
            f = float(scale) / (max(1, self.count) if reduction == "mean" else 1)
        dz, e = dz * live, e * live
        e = e + q * (dz.abs() + e)                      # rounded to the operands' type

        def close(v, s, err, terms):
            err = abs(f) * (err + (terms + 12) * U * s)
            return rounded(f * v, err, self.dtype)

        full = dz.abs() + e
        return {"dx": close(dz @ self.w.t(), full @ self.w.abs().t(), e @ self.w.abs().t(), dz.shape[1]),
                "dw": close(self.x.t() @ dz, self.x.abs().t() @ full, self.x.abs().t() @ e, dz.shape[0])}
