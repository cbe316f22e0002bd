"""Plain double-precision forms of a block's and a training step's further operators (numpy, written from their definitions)."""
import numpy as np

import training_ref

BLOCK, TOP, NONE = 256, 448.0, 2.0 ** -100


def e4m3_step(size):
    """Distance of e4m3's numbers around magnitudes of `size`."""
    return 2.0 ** (np.floor(np.log2(np.maximum(size, 2.0 ** -6))) - 3)


def e4m3(t):
    """To nearest, ties to even."""
    step = e4m3_step(np.abs(t))
    return np.rint(t / step) * step


def e4m3_by(t, bits):
    """t >= 0 to a neighbour, up where the 16 bits reach what is missing (cut to 16 bits); not from above zero to zero."""
    step = e4m3_step(t)
    low = np.floor(t / step)
    up = np.floor((t / step - low) * 65536) + bits >= 65536
    return np.where(t > 0, np.maximum(np.minimum((low + up) * step, TOP), 2.0 ** -9), 0.0)


def halves(n, number, step, seed):
    """The 16 bits of elements 0 to n - 1 of tensor `number`."""
    i = np.arange(n, dtype=np.uint64)
    block = i // np.uint64(8) + np.uint64(number << 40)
    low, seed = 0xFFFFFFFF, seed % 2 ** 64
    words = training_ref.philox([block & np.uint64(low), block >> np.uint64(32), np.full(n, step & low, np.uint64), np.full(n, step >> 32, np.uint64)],
                                (seed & low, seed >> 32))
    e = (i % np.uint64(8)).astype(np.int64)
    return (np.choose(e // 2, words) >> (np.uint64(16) * (e % 2).astype(np.uint64)) & np.uint64(0xFFFF)).astype(np.float64)


def blocks(v):
    out = np.zeros((-(-v.size // BLOCK), BLOCK))
    out.reshape(-1)[:v.size] = v
    return out


def scaled(v):
    """(v in units of its block's scale, scales [blocks])."""
    b = blocks(v)
    top = np.abs(b).max(-1)
    top = np.where(top >= NONE, top, 0.0)
    t = b * np.divide(TOP, top, out=np.zeros_like(top), where=top > 0)[:, None]
    return np.clip(t, -TOP, TOP).reshape(-1)[:v.size], top / TOP


def adamw(p, g, m, v, lr, wd, betas, eps, t, factors=(1.0, 1.0)):
    """(p, m, v, the magnitude of the move) of one tensor, all in 64 bits."""
    p, g, m, v = (a.astype(np.float64) for a in (p, g, m, v))
    g = g * factors[0]
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    lr = lr * factors[1]
    move = lr / (1 - betas[0] ** t) * m / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
    return p * (1 - lr * wd) - move, m, v, np.abs(move)
