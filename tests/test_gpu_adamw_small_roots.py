"""AdamW's second state of 8 bits where squares are below fp32's least number: a root above zero stays above zero, beside much larger ones too.

Tolerances.  States have to be the definition's, made in 64 bits throughout, but where the scaled number is within two fp32 steps of a border between two of
them.  The move as in test_gpu_adamw.py, 8 halves of fp32's steps, and two more of the root, which below 2^-126 is off by half of fp32's least step and then
meets an eps of 2^-126; m and rate * m are off by that half step, 2^-150, as well, which is divided by root and eps."""
import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
LEAST_ROOT = 2.0 ** -75                                      # of a block's largest


def numbers(rng, n, low, high):
    """Of either sign, magnitudes spread over the powers of two from low to high."""
    return 2.0 ** rng.uniform(low, high, n) * rng.choice([-1.0, 1.0], n)


def gradients(seed):
    rng = np.random.default_rng(seed)
    g = np.concatenate([numbers(rng, 256, -140, -57),        # a block of tiny numbers, most of which have no square in fp32
                        numbers(rng, 256, -110, -72),        # one whose largest root is stored as zero
                        numbers(rng, 256, -140, -100),       # one large number beside them (below)
                        0.02 * rng.standard_normal(256),
                        numbers(rng, 77, -100, -20)])
    g[256 * 2 + 100] = 2.0 ** 62
    g[7::50] = 0
    return g.astype(np.float32)


def h(t):
    return t.float().double().cpu().numpy()


def test_roots_of_squares_below_fp32():
    n, eps, betas, lr, seed = 256 * 4 + 77, 2.0 ** -126, (0.9, 0.999), 1e-3, 11
    rng = np.random.default_rng(0)
    p = torch.from_numpy((0.1 * rng.standard_normal(n)).astype(np.float32)).cuda()
    g = torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    s = torch.zeros((-(-n // 256), 2), device="cuda")
    plan = dcn.dcnv4_adamw_plan([p], [g], [m], [v], lr, scales=[s])
    near = (1 - 2.0 ** -22, 1.0, 1 + 2.0 ** -22)
    for t in (1, 2, 3):
        g.copy_(torch.from_numpy(gradients(t)))
        scale = np.repeat(h(s), 256, axis=0)[:n]
        p0, g0, m0, v0 = h(p), h(g), h(m) * scale[:, 0], (h(v) * scale[:, 1]) ** 2
        dcn.dcnv4_adamw_step(plan, t, betas=betas, eps=eps, seed=seed)
        torch.cuda.synchronize()
        wp, wm, wv, move = ref.adamw(p0, g0, m0, v0, lr, 0.0, betas, eps, t)
        wr = np.sqrt(wv)
        below = wr / np.sqrt(1 - betas[1] ** t) + eps
        lim = 3 * E * (np.abs(p0) + move) + 10 * E * move + 2 * 2.0 ** -150 / below
        assert np.all(np.abs(h(p) - wp) <= lim), (t, np.nanmax(np.abs(h(p) - wp) / lim))
        top = np.abs(ref.blocks(wr)).max(-1)
        tr = ref.scaled(wr)[0] * np.repeat(top >= LEAST_ROOT, 256)[:n]
        tm = ref.scaled(wm)[0]
        bits = ref.halves(n, 0, t, seed)
        assert np.all(np.any([h(m) == ref.e4m3(np.clip(tm * k, -448, 448)) for k in near], axis=0)), t
        assert np.all(np.any([h(v) == ref.e4m3_by(np.minimum(tr * k, 448), bits) for k in near], axis=0)), t
        # (the blocks are what they are meant to be: zeros in one, and above zero wherever there was a gradient in the others)
        got = h(v)
        assert np.all(got[256:512] == 0) and top[0] > LEAST_ROOT > top[1]
        there = (wv > 0) & (np.arange(n) // 256 != 1)
        assert np.all(got[there] > 0) and there.sum() > 800 and (t > 1 or np.sum(wv[there] < 2.0 ** -150) > 300)
