"""Reference of the AdamW step: the parameter in 64 bits with a bound on what fp32
arithmetic and its rounding may add, the averages and the codes of 8-bit states in
fp32 (numpy), operation by operation, which the GPU's have to equal.
"""
import numpy as np
import torch

from layers_ref import ROUND, U

BLOCK = 256
M32 = np.uint32(0xFFFFFFFF)


def mix(x):
    x = np.asarray(x, dtype=np.uint32)
    with np.errstate(over="ignore"):
        x = x ^ (x >> np.uint32(16))
        x = x * np.uint32(0x6A09E667)
        x = x ^ (x >> np.uint32(15))
        x = x * np.uint32(0xBB67AE85)
        return x ^ (x >> np.uint32(16))


def random_bits(n, seed, step, tensor):
    """What is added below the kept bits of element 0 .. n - 1: (of exp_avg, of exp_avg_sq)."""
    u = lambda v: np.uint32(v & 0xFFFFFFFF)
    key = mix(u(int(mix(u(seed + step * 0x9E3779B9))) + tensor))
    with np.errstate(over="ignore"):
        h = mix((np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B1)) ^ key)
    return (h & np.uint32(0xFFFF)) << np.uint32(4), (h >> np.uint32(16)) << np.uint32(4)


def decode(code, base, signed):
    code = code.astype(np.uint32)
    size = code & 127 if signed else code
    base = np.repeat(base.astype(np.uint32), BLOCK)[:code.size]
    bits = np.where(size > 0, (size + base) << np.uint32(20), np.uint32(0)).astype(np.uint32)
    if signed:
        bits |= (code & 128) << np.uint32(24)
    return bits.view(np.float32)


def encode(value, add, signed):
    """(codes, bases)."""
    top = 127 if signed else 255
    bits = value.view(np.uint32) & np.uint32(0x7FFFFFFF)
    blocks = -(-value.size // BLOCK)
    padded = np.zeros(blocks * BLOCK, np.uint32)
    padded[:value.size] = bits
    base = np.clip((padded.reshape(blocks, BLOCK).max(1) >> 20).astype(np.int64) + 1 - top, 0, 2047 - top)
    size = ((bits + add) >> np.uint32(20)).astype(np.int64) - np.repeat(base, BLOCK)[:value.size]
    size = np.minimum(size, top)
    size = np.maximum(size, 0 if signed else (bits != 0).astype(np.int64))
    if signed:
        size = np.where(size > 0, size | ((value.view(np.uint32) >> 31).astype(np.int64) << 7), size)
    return size.astype(np.uint8), base.astype(np.int16)


def averages(g, m, v, betas):
    """The new averages in fp32, each operation rounded by itself."""
    f = np.float32
    (b1, b2), g = betas, g.astype(f)
    with np.errstate(all="ignore"):
        return m * f(b1) + g * f(1 - b1), v * f(b2) + (g * g) * f(1 - b2)


def param(p, g, m, v, step, lr, betas, eps, decay, dtype):
    """(value, bound) of the new parameter in 64 bits, from fp32 arrays of p, g and the old averages."""
    p, g, m, v = (t.astype(np.float64) for t in (p, g, m, v))
    b1, b2 = betas
    mn, vn = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    sm = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    den = np.sqrt(vn / (1 - b2 ** step)) + eps
    rate = lr / (1 - b1 ** step)
    new = p * (1 - lr * decay) - rate * mn / den
    # m: two products with rounded factors and their sum (5 u S); v and its root the same relative to
    # itself; the quotient, the rate and the last sum
    err = rate * (5 * U * sm + 12 * U * np.abs(mn)) / den + 4 * U * np.abs(p) + 2 * U * np.abs(new)
    q = ROUND[dtype]
    t = torch.from_numpy
    return t(new), t(err + q * (np.abs(new) + err) + 1e-300)
