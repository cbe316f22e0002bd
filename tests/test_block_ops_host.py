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
    assert adam(n=(1 << 34) + 1) == 3 and adam(bits=16) == 3 and adam(dtype=2) == 3 and adam(copy=A) == 3
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


def without(count, i, value=None):
    ptrs = [A] * count
    ptrs[i] = value
    return tuple(ptrs)


def end(ptrs=(A,) * 14, P=6, C=16, gates=2, norms=3, eps=1e-6, dtype=0):
    return dcn.load_library().dcnv4_norm_scale_add_norm(*ptrs, P, C, gates, norms, eps, dtype, None)


def end_back(ptrs=(A,) * 22, size=1 << 30, P=6, C=16, gates=2, norms=3, dtype=0):
    return dcn.load_library().dcnv4_norm_scale_add_norm_backward(*ptrs, size, P, C, gates, norms, dtype, None)


def test_block_end_validates_on_the_host():
    for i in (0, 1, 5, 8, 9):
        assert end(without(14, i)) == 1
    for i in (0, 1, 7, 8, 9, 10, 11, 13, 14, 5, 21):
        assert end_back(without(22, i)) == 1, i
    assert end_back(without(22, 12), norms=1) == 1                # without a second norm, grad_z is the gradient
    for i in range(14):
        assert end(without(14, i, A + 8)) == 4
    for i in range(22):
        assert end_back(without(22, i, A + 8)) == 4
    for call in (end, end_back):
        assert call(P=0) == 2 and call(C=0) == 2 and call(P=-1) == 2 and call(gates=-1) == 2 and call(gates=4) == 2
        assert call(C=8193) == 3 and call(dtype=2) == 3 and call(norms=4) == 3 and call(norms=-1) == 3
        assert call(P=1 << 31) == 3 and call(P=(1 << 20) + 1, gates=(1 << 20) + 1) == 3
    assert end(eps=-1.0) == 3 and end(eps=float("nan")) == 3 and end(eps=float("inf")) == 3
    need = dcn.dcnv4_norm_scale_add_norm_workspace_bytes
    assert end_back(size=need(6, 16, 2) - 1) == 2 and end_back(gates=0) == 2
    assert need(0, 16, 0) == -1 and need(5, 16, 2) == -1 and need(4, 9000, 0) == -1 and need(6, 16, 2) > need(6, 16, 0) > 0
    assert need(10 ** 9, 8192, 0) < 1 << 30


@pytest.mark.parametrize("form", ["", "f", "s", "fs"])
def test_gradient_of_the_plain_block_end_against_differences(form):
    rng = np.random.default_rng(1)
    r = lambda *s: rng.standard_normal(s)
    shape, eps = (2, 3, 5), 1e-3
    v = {"x": r(*shape), "residual": r(*shape), "scale": r(5), "gate": np.array([0.0, 1.3]), "gamma1": r(5), "beta1": r(5), "gamma2": r(5), "beta2": r(5)}
    gy, gz = r(*shape), r(*shape)

    def forward(v):
        z, _ = ref.end(v["x"], v["residual"], v["scale"], v["gate"], (v["gamma1"], v["beta1"]) if "f" in form else None, eps)
        return z, ref.norm(z, v["gamma2"], v["beta2"], eps)[0] if "s" in form else None

    def value(v):
        z, y = forward(v)
        return (z * gz).sum() + (0 if y is None else (y * gy).sum())

    z, _ = forward(v)
    _, m1, r1 = ref.norm(v["x"], 1.0, 0.0, eps)
    _, m2, r2 = ref.norm(z, 1.0, 0.0, eps)
    got = ref.end_backward(v["x"], z, v["scale"], v["gate"], (v["gamma1"], v["beta1"]) if "f" in form else None,
                           (v["gamma2"], v["beta2"]) if "s" in form else None, (m1, r1, m2, r2), gy, gz)
    step = 1e-6
    for name, (grad, _) in got.items():
        at = name[len("grad_"):]
        for i in range(grad.size):
            moved = []
            for sign in (1, -1):
                w = {k: a.copy() for k, a in v.items()}
                w[at].reshape(-1)[i] += sign * step
                moved.append(value(w))
            assert abs((moved[0] - moved[1]) / (2 * step) - grad.reshape(-1)[i]) < 1e-6, (name, i)


def gated(ptrs=(A,) * 5, size=1 << 40, P=5, K=32, F=16, act=0, dtype=0):
    return dcn.load_library().dcnv4_gated_linear(*ptrs, size, P, K, F, act, dtype, None)


def gated_back(ptrs=(A,) * 8, size=1 << 40, P=5, K=32, F=16, act=0, dtype=0):
    return dcn.load_library().dcnv4_gated_linear_backward(*ptrs, size, P, K, F, act, dtype, None)


def linear_back(ptrs=(A,) * 7, size=1 << 40, P=5, K=32, F=16, act=0, dtype=0):
    return dcn.load_library().dcnv4_linear_backward(*ptrs, size, P, K, F, dtype, None)


def test_layers_validate_on_the_host():
    for call, count, needed in ((gated, 5, (0, 1, 3, 4)), (gated_back, 8, (0, 1, 3, 7)), (linear_back, 7, (0, 1, 2, 6))):
        for i in range(count):
            if i in needed:
                assert call(without(count, i)) == 1, (call, i)
            assert call(without(count, i, A + 8)) == 4
        assert call(P=0) == 2 and call(K=0) == 2 and call(F=0) == 2 and call(F=-8) == 2
        assert call(K=12) == 3 and call(K=20, dtype=1) == 3 and call(F=12) == 3 and call(dtype=2) == 3
        assert call(P=(1 << 24) + 1) == 3 and call(K=1 << 21) == 3 and call(F=1 << 21) == 3
    assert gated(act=2) == 3 and gated_back(act=-1) == 3
    assert gated(K=1 << 14, F=1 << 15, dtype=1) == 3 and gated(K=1 << 14, F=1 << 14, dtype=0) == 3       # weights past 32-bit offsets
    none = lambda count, *at: tuple(None if i in at else A for i in range(count))
    assert gated_back(none(8, 4, 5, 6)) == 1 and linear_back(none(7, 3, 4, 5)) == 1
    bytes_of = dcn.dcnv4_gated_linear_workspace_bytes
    assert bytes_of(5, 32, 16, 1, False) == 0 and bytes_of(5, 32, 16, 0, False) > 0 and bytes_of(0, 32, 16, 0, True) == -1
    for dtype in (0, 1):
        assert gated_back(size=bytes_of(5, 32, 16, dtype, True) - 1, dtype=dtype) == 2
        assert linear_back(size=dcn.dcnv4_linear_backward_workspace_bytes(5, 32, 16, dtype) - 1, dtype=dtype) == 2
    assert gated(size=bytes_of(5, 32, 16, 0, False) - 1) == 2
    for key, bad in (("layer_tile", 5), ("layer_splits", 65), ("layer_tile", -1)):
        with pytest.raises(dcn.Dcnv4Error):
            dcn.dcnv4_set_option(key, bad)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_of_the_plain_gated_layer_against_differences(act):
    rng = np.random.default_rng(2)
    v = {"x": rng.standard_normal((3, 4)), "w": rng.standard_normal((2, 5, 4)), "b": rng.standard_normal((2, 5))}
    gh = rng.standard_normal((3, 5))
    _, _, parts = ref.gated(v["x"], v["w"], v["b"], act, True)
    step = 1e-6
    for name, (grad, _) in ref.gated_backward(v["x"], v["w"], gh, parts, True).items():
        for i in range(grad.size):
            moved = []
            for sign in (1, -1):
                u = {k: a.copy() for k, a in v.items()}
                u[name[5:]].reshape(-1)[i] += sign * step
                moved.append((ref.gated(u["x"], u["w"], u["b"], act, True)[0] * gh).sum())
            assert abs((moved[0] - moved[1]) / (2 * step) - grad.reshape(-1)[i]) < 1e-7, (name, i)


def test_layers_refuse_host_tensors():
    import torch
    x, w, g = torch.zeros((3, 8)), torch.zeros((2, 8, 8)), torch.zeros((3, 8))
    for call in (lambda: dcn.dcnv4_gated_linear(x, w), lambda: dcn.dcnv4_gated_linear_backward(x, w, g), lambda: dcn.dcnv4_linear_backward(x, w[0], g),
                 lambda: dcn.dcnv4_norm_scale_add_norm(x, x), lambda: dcn.dcnv4_norm_scale_add_norm_backward(x, x, None, None, None, None, (None,) * 4, None, x)):
        with pytest.raises(ValueError, match="x must be a GPU tensor"):
            call()
