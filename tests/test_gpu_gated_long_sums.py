"""The gated layer in fp32 over many features and few rows: roundings of the small parts' products do not add to those of the large ones.

Tolerance, for 2-norms.  A sum of n additions of either sign is off by 0.29 of a step at each (uniform), a step being 0.72 * 2^-23 of the sum on average, and the
sum after k of them sqrt(k / n) of the last: 0.21 * 2^-23 * sqrt(n / 2).  2048 features are 128 products of 16, each added in two halves at most: n = 256,
2.4 * 2^-23.  h has that of u and, by act'(a) a / act(a), 1.3 times that of a: 3.9 * 2^-23, and half as much again for what is not uniform.  (Six products
added one after the other are n = 768 at least, twice that.)"""
import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

LIMIT = 6 * 2.0 ** -23


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("P,K,F", [(1, 2048, 512), (48, 1952, 56), (300, 2048, 200)])
def test_forward(P, K, F, act):
    rng = np.random.default_rng(P + K)
    r = lambda *s: rng.standard_normal(s).astype(np.float32)
    x, w, b = r(P, K), (r(2, F, K) / np.sqrt(K)).astype(np.float32), (0.3 * r(2, F)).astype(np.float32)
    h = dcn.dcnv4_gated_linear(*(torch.from_numpy(t).cuda() for t in (x, w, b)), activation=act).double().cpu().numpy()
    want = ref.gated(x, w, b, act, False)[0]
    off = np.linalg.norm(h - want) / np.linalg.norm(want)
    assert off <= LIMIT, off / 2.0 ** -23
