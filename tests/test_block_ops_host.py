"""Host-side checks of a block's and a training step's further operators: refusals before any launch, and the plain forms themselves."""
import ctypes

import numpy as np
import pytest

import block_ref as ref
from paper_2401_06197_amd import binding as dcn

A = 4096                                                     # aligned, never dereferenced


def adam(count=1, beta1=0.9, beta2=0.999, eps=1e-8, step=1, more=None, factors=None, bits=32, dtype=0, **fields):
    t = (dcn.AdamwTensor * max(count, 1))()
    for r in t:
        for k, v in {"n": 10, "param": A, "grad": A, "m": A, "v": A, "scales": None, "copy": None, "lr": 1e-3, "weight_decay": 0.1, **fields}.items():
            setattr(r, k, v)
    return dcn.load_library().dcnv4_adamw(t, count, beta1, beta2, eps, step, more, factors, 0, bits, dtype, None)


def test_adamw_validates_on_the_host():
    lib, nan, inf = dcn.load_library(), float("nan"), float("inf")
    assert lib.dcnv4_adamw(None, 1, 0.9, 0.999, 1e-8, 1, None, None, 0, 32, 0, None) == 1
    for name in ("param", "grad", "m", "v"):
        assert adam(**{name: None}) == 1 and adam(**{name: A + 8}) == 4
    assert adam(bits=8) == 1 and adam(bits=8, scales=A + 4) == 4 and adam(dtype=1, copy=A + 8) == 4
    assert adam(count=0) == 2 and adam(count=-1) == 2 and adam(n=0) == 2 and adam(n=-5) == 2
    assert adam(n=(1 << 36) + 1) == 3 and adam(bits=16) == 3 and adam(dtype=2) == 3 and adam(copy=A) == 3
    for bad in (-0.1, 1.0, nan):
        assert adam(beta1=bad) == 3 and adam(beta2=bad) == 3
    for bad in (0.0, -1e-8, nan, inf, 1e-40):
        assert adam(eps=bad) == 3
    assert adam(lr=nan) == 3 and adam(lr=inf) == 3 and adam(weight_decay=inf) == 3
    assert adam(step=0) == 3 and adam(step=-1) == 3 and adam(step=-1, more=A) == 3
    assert adam(more=A + 4) == 4 and adam(factors=A + 4) == 4
    # the last of several
    t = (dcn.AdamwTensor * 2)()
    for r in t:
        r.n, r.param, r.grad, r.m, r.v, r.lr = 10, A, A, A, A, 1e-3
    t[1].v = None
    assert lib.dcnv4_adamw(t, 2, 0.9, 0.999, 1e-8, 1, None, None, 0, 32, 0, None) == 1
    assert ctypes.sizeof(dcn.AdamwTensor) == 72


def test_adamw_refuses_host_tensors():
    import torch
    z = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU tensors"):
        dcn.dcnv4_adamw_plan([z], [z], [z], [z], 1e-3)


def test_plain_8_bit_numbers_are_the_types():
    import torch
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    every = every[np.isfinite(every)]
    assert np.array_equal(ref.e4m3(every), every) and every.max() == ref.TOP
    rng = np.random.default_rng(0)
    t = np.concatenate([rng.uniform(-448, 448, 4000), rng.uniform(-0.1, 0.1, 4000), (every[:-1] + every[1:]) / 2])
    assert np.array_equal(ref.e4m3(t), torch.from_numpy(t).float().to(torch.float8_e4m3fn).double().numpy())
    u = np.abs(t)
    a, b = ref.e4m3_by(u, np.zeros(u.size)), ref.e4m3_by(u, np.full(u.size, 65535.0))
    assert np.all(np.isin(a, every)) and np.all(np.isin(b, every)) and np.all((a <= u) | (a == 2.0 ** -9)) and np.all(b >= u - ref.e4m3_step(u) / 65536)
    # and keeps the mean
    x = np.full(200000, 3.3)
    assert abs(ref.e4m3_by(x, rng.integers(0, 65536, x.size).astype(float)).mean() - 3.3) < 5 * 0.125 / np.sqrt(x.size)
