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


E24 = 2.0 ** -24


def norm(x, gamma, beta, eps):
    mean = x.mean(-1)
    rstd = 1 / np.sqrt(((x - mean[..., None]) ** 2).mean(-1) + eps)
    return (x - mean[..., None]) * rstd[..., None] * gamma + beta, mean, rstd


def norm_backward(x, mean, rstd, g, dg, k):
    """The gradient at x for g at the unit rows, xhat, and how far fp32 sums of k terms in a chain, and dg of g, may take them."""
    mean, rstd = mean[..., None], rstd[..., None]
    xh, dxh = (x - mean) * rstd, 4 * E24 * (np.abs(x) + np.abs(mean)) * np.abs(rstd)
    avg = lambda v: v.mean(-1, keepdims=True)
    a, b = avg(g), avg(g * xh)
    da = avg(dg) + k * E24 * avg(np.abs(g))
    db = avg(np.abs(xh) * dg + np.abs(g) * dxh) + k * E24 * avg(np.abs(g * xh))
    gx = rstd * (g - a - xh * b)
    dgx = rstd * (dg + da + np.abs(xh) * db + dxh * np.abs(b)) + 8 * E24 * rstd * (np.abs(g) + np.abs(a) + np.abs(xh * b))
    return gx, dgx, xh, dxh


def end(x, residual, scale, gate, first, eps):
    """z, and what it is made of: b.  scale, gate [N] and first = (gamma, beta) are arrays or None."""
    x = x.astype(np.float64)
    b = x if first is None else norm(x, *first, eps)[0]
    by = np.ones(x.shape[:1]) if gate is None else gate.astype(np.float64)
    by = by.reshape(-1, *[1] * (x.ndim - 1)) * (1.0 if scale is None else scale)
    return residual.astype(np.float64) + np.where(by == 0, 0.0, by * b), b


def end_backward(x, z, scale, gate, first, second, stats, gy, gz, k=64, rows=256):
    """{name: (gradient, how far fp32 sums may take it)}; k, rows: terms in a chain of a row's sum and of one over rows."""
    f = lambda a: None if a is None else np.asarray(a, dtype=np.float64)
    x, z, gy, gz, scale, gate = map(f, (x, z, gy, gz, scale, gate))
    pixels = tuple(range(x.ndim - 1))
    out = {}
    add = lambda v, dv: (v.sum(pixels), dv.sum(pixels) + rows * E24 * np.abs(v).sum(pixels))
    g, dg = (np.zeros(x.shape) if gz is None else gz), np.zeros(x.shape)
    if second is not None:
        gx, dgx, zh, dzh = norm_backward(z, stats[2], stats[3], gy * second[0], 2 * E24 * np.abs(gy * second[0]), k)
        g, dg = g + gx, dgx + 2 * E24 * (np.abs(g) + np.abs(gx))
        out["grad_gamma2"] = add(gy * zh, np.abs(gy) * dzh + 2 * E24 * np.abs(gy * zh))
        out["grad_beta2"] = add(gy, 0 * gy)
    out["grad_residual"] = g, dg
    by = np.ones(x.shape[:1]) if gate is None else gate
    by = np.broadcast_to(by.reshape(-1, *[1] * (x.ndim - 1)), x.shape)
    sc = np.ones(x.shape[-1]) if scale is None else scale
    if first is not None:
        xh = (x - stats[0][..., None]) * stats[1][..., None]
        dxh = 4 * E24 * (np.abs(x) + np.abs(stats[0][..., None])) * stats[1][..., None]
        gamma, beta = first
    else:
        xh, dxh, gamma, beta = x, 0 * x, np.ones(x.shape[-1]), np.zeros(x.shape[-1])
    b, db = xh * gamma + beta, dxh * np.abs(gamma) + 2 * E24 * (np.abs(xh * gamma) + np.abs(beta))
    image = tuple(range(1, x.ndim))
    t, dt = g * sc * b, np.abs(sc) * (np.abs(g) * db + dg * np.abs(b)) + 4 * E24 * np.abs(g * sc * b)
    out["grad_gate"] = t.sum(image), dt.sum(image) + (k + rows) * E24 * np.abs(t).sum(image)
    on = by != 0
    q, dq = np.where(on, by * g, 0), np.where(on, np.abs(by) * dg + 2 * E24 * np.abs(by * g), 0)
    xz, dxz = np.where(on, xh, 0), np.where(on, dxh, 0)
    s1, ds1 = add(q * xz, np.abs(q) * dxz + dq * np.abs(xz) + 2 * E24 * np.abs(q * xz))
    s0, ds0 = add(q, dq)
    if first is None:
        out["grad_scale"] = s1, ds1
    else:
        out["grad_scale"] = gamma * s1 + beta * s0, np.abs(gamma) * ds1 + np.abs(beta) * ds0 + 4 * E24 * (np.abs(gamma * s1) + np.abs(beta * s0))
        out["grad_gamma1"] = sc * s1, np.abs(sc) * ds1 + 2 * E24 * np.abs(sc * s1)
        out["grad_beta1"] = sc * s0, np.abs(sc) * ds0 + 2 * E24 * np.abs(sc * s0)
    h, dh = q * sc * gamma, np.abs(sc * gamma) * dq + 4 * E24 * np.abs(q * sc * gamma)
    if first is None:
        out["grad_x"] = h, dh
    else:
        xs, m, r = (np.where(on, a, 0) for a in (x, np.broadcast_to(stats[0][..., None], x.shape), np.broadcast_to(stats[1][..., None], x.shape)))
        gx, dgx, _, _ = norm_backward(xs, m[..., 0], r[..., 0], h, dh, k)
        out["grad_x"] = np.where(on, gx, 0), np.where(on, dgx, 0)
    return out




def activation(a, act):
    """act(a) and its derivative."""
    from scipy.special import expit, ndtr
    if act == "silu":
        s = expit(a)
        return a * s, s * (1 + a * expit(-a))
    return a * ndtr(a), ndtr(a) + a * np.exp(-a * a / 2) / np.sqrt(2 * np.pi)


def products_off(terms, size, f16):
    """How far a sum of products on the matrix units may be off: 16 at a time, one after the other, `size` being the sum of magnitudes; fp32 operands as three
    bf16 numbers take six passes and leave out 2^-22 of each."""
    return (terms / 16 + 32) * E24 * size if f16 else (6 * (terms / 16) + 64) * E24 * size + 2.0 ** -22 * size


def gated(x, w, b, act, f16):
    """h, how far fp32 arithmetic may take it, and what the backward pass needs."""
    x, w = x.astype(np.float64), w.astype(np.float64)
    b = np.zeros(w.shape[:2]) if b is None else b.astype(np.float64)
    a, u = x @ w[0].T + b[0], x @ w[1].T + b[1]
    size = [np.abs(x) @ np.abs(w[i]).T + np.abs(b[i]) for i in (0, 1)]
    da, du = (products_off(x.shape[-1], s, f16) for s in size)
    value, slope = activation(a, act)
    # the functions: fp16's results by exp2 and a reciprocal of an argument that was rounded (a or a^2 / 2 times 2^-24 and a few steps)
    off = (a * a + np.abs(a) + 16) * E24
    dv, ds = (np.abs(slope) + da) * da + off * (np.abs(value) + 2.0 ** -30), 1.2 * da + off * (np.abs(slope) + np.abs(a))
    return value * u, np.abs(u) * dv + np.abs(value) * du + dv * du + 2 * E24 * np.abs(value * u), (a, u, da, du, value, slope, dv, ds)


def gated_backward(x, w, gh, parts, f16):
    """{name: (gradient, how far it may be off before its own rounding)}."""
    x, w, gh = x.astype(np.float64), w.astype(np.float64), gh.astype(np.float64)
    a, u, da, du, value, slope, dv, ds = parts
    d = np.concatenate([gh * u * slope, gh * value], -1)
    off = np.concatenate([np.abs(gh) * (np.abs(u) * ds + np.abs(slope) * du + du * ds), np.abs(gh) * dv], -1) + 4 * E24 * np.abs(d)
    top = np.abs(gh).max()
    rounded = off + (2.0 ** -11 * np.abs(d) + 2.0 ** -25 * top / 2 if f16 else 2.0 ** -23 * np.abs(d))
    both = w.reshape(-1, w.shape[-1])
    lead = (-1, d.shape[-1])
    d2, r2, o2, x2 = d.reshape(lead), rounded.reshape(lead), off.reshape(lead), x.reshape(-1, x.shape[-1])
    gx = (d2 @ both, r2 @ np.abs(both) + products_off(both.shape[0], np.abs(d2) @ np.abs(both), f16))
    gw = (d2.T @ x2, r2.T @ np.abs(x2) + products_off(x2.shape[0], np.abs(d2).T @ np.abs(x2), f16))
    gb = (d2.sum(0), o2.sum(0) + (x2.shape[0] / 32 + 64) * E24 * np.abs(d2).sum(0))
    return {"grad_x": tuple(v.reshape(x.shape) for v in gx), "grad_w": tuple(v.reshape(w.shape) for v in gw), "grad_b": tuple(v.reshape(w.shape[:2]) for v in gb)}


def linear_backward(x, w, gy, f16):
    x, w, gy = (v.astype(np.float64) for v in (x, w, gy))
    x2, g2 = x.reshape(-1, x.shape[-1]), gy.reshape(-1, gy.shape[-1])
    gx = (g2 @ w, products_off(w.shape[0], np.abs(g2) @ np.abs(w), f16))
    gw = (g2.T @ x2, products_off(x2.shape[0], np.abs(g2).T @ np.abs(x2), f16))
    return {"grad_x": tuple(v.reshape(x.shape) for v in gx), "grad_w": gw,
            "grad_b": (g2.sum(0), (x2.shape[0] / 256 + 320) * E24 * np.abs(g2).sum(0))}
