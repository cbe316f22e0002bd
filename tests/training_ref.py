"""Plain double-precision forms of the operators around the module (numpy, written from their definitions)."""
import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
MASK = 0xFFFFFFFF


def philox(counter, key):
    """Philox 4x32 with ten rounds, word by word: counter of four words (arrays or ints), key of two ints."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k0, k1 = key
    for _ in range(10):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & np.uint64(MASK),
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & np.uint64(MASK)]
        k0, k1 = (k0 + W0) & MASK, (k1 + W1) & MASK
    return c


def dropped(n, p, seed, offset, first=0):
    """Truth of 'element first + i is dropped', i < n."""
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    i = np.arange(first, first + n, dtype=np.uint64)
    block = i // np.uint64(8)
    words = philox([block & np.uint64(MASK), block >> np.uint64(32), np.full(n, offset & MASK, np.uint64),
                    np.full(n, offset >> 32, np.uint64)], (seed & MASK, seed >> 32))
    e = (i % np.uint64(8)).astype(np.int64)
    word = np.choose(e // 2, words)
    half = (word >> (np.uint64(16) * (e % 2).astype(np.uint64))) & np.uint64(0xFFFF)
    return half < np.uint64(limit(p))


def limit(p):
    """p as the library takes it: a float, to the nearest multiple of 2^-16."""
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def dropout(x, p, seed, offset, residual=None):
    gone = dropped(x.size, p, seed, offset).reshape(x.shape)
    y = np.zeros(x.shape) if limit(p) == 65536 else x.astype(np.float64) / (1 - limit(p) / 65536)
    y = np.where(gone, 0.0, y)
    return y if residual is None else y + residual.astype(np.float64)


def layer_norm(x, gamma, beta, eps):
    x = x.astype(np.float64)
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    y = (x - mean) * rstd
    if gamma is not None:
        y = y * gamma.astype(np.float64)
    if beta is not None:
        y = y + beta.astype(np.float64)
    return y, mean[..., 0], rstd[..., 0]


def layer_norm_backward(x, gamma, mean, rstd, grad_y):
    """grad_x, grad_gamma, grad_beta, and for each the sum of the magnitudes that it was added up from."""
    x, gy = x.astype(np.float64), grad_y.astype(np.float64)
    mean, rstd = mean.astype(np.float64)[..., None], rstd.astype(np.float64)[..., None]
    xhat = (x - mean) * rstd
    g = gy if gamma is None else gy * gamma.astype(np.float64)
    gx = rstd * (g - g.mean(-1, keepdims=True) - xhat * (g * xhat).mean(-1, keepdims=True))
    size = rstd * (np.abs(g) + np.abs(g).mean(-1, keepdims=True) + np.abs(xhat) * np.abs(g * xhat).mean(-1, keepdims=True))
    rows = tuple(range(x.ndim - 1))
    return (gx, (gy * xhat).sum(rows), gy.sum(rows)), (size, np.abs(gy * xhat).sum(rows), np.abs(gy).sum(rows))
