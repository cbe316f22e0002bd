"""The end of a residual block with its norms, scale and gate, and its gradient, against plain double-precision forms, through the C ABI.

Tolerances.  A result is rounded once: half a step of its type, in fp16 at least half of the smallest step, 2^-25.  Before that, fp32: a row's sum has
8 terms a lane, 6 exchanges and 16 waves, with a handful of operations around it: less than 64 in a chain.  A sum over rows has P / (workgroups * rows
side by side) + 64 + 16 + 64 in a chain: the cases here keep that below 256.  block_ref carries both through the formulas."""
import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

NP = {"f32": np.float32, "f16": np.float16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11}
LEAST = {"f32": 0.0, "f16": 2.0 ** -25}
E = 2.0 ** -24
NAMES = ("grad_x", "grad_residual", "grad_scale", "grad_gate", "grad_gamma1", "grad_beta1", "grad_gamma2", "grad_beta2")


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def h(t):
    return None if t is None else t.cpu().numpy().astype(np.float64)


def close(name, got, want, slack, dtype):
    got = h(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    lim = (1 + U[dtype]) * slack + U[dtype] * np.abs(want) + LEAST[dtype]
    bad = ~(np.abs(got - want) <= lim)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / np.maximum(lim, 1e-300), 0)), bad.shape)
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} off; at {at} got {got[at]!r}, want {want[at]!r}, limit {lim[at]!r}")


def draw(shape, dtype, form, seed, gate=True, scale=True, affine=True):
    rng = np.random.default_rng(seed)
    r = lambda s, size=1.0, shift=0.0: (rng.standard_normal(s) * size + shift).astype(NP[dtype])
    C = shape[-1]
    d = {"x": r(shape, 1.5, 0.3), "residual": r(shape), "grad_z": r(shape), "grad_y": r(shape) if "s" in form else None,
         "scale": r(C, 0.3, 0.5) if scale else None, "gate": None, "first": None, "second": None}
    if gate:
        d["gate"] = (rng.random(shape[0]) * 2).astype(np.float32)
        d["gate"][::3] = 0.0
    vectors = lambda: (r(C, 0.2, 1.0), r(C, 0.2)) if affine else (None, None)
    if "f" in form:
        d["first"] = vectors()
    if "s" in form:
        d["second"] = vectors()
    return d


def pair(p):
    return None if p is None else tuple(gpu(v) for v in p)


def plain(p, C):
    return None if p is None else tuple((np.full(C, o) if v is None else v.astype(np.float64)) for v, o in zip(p, (1.0, 0.0)))


def run(d, eps, grad_z=True, **kw):
    x, scale, gate, first, second = gpu(d["x"]), gpu(d["scale"]), gpu(d["gate"]), pair(d["first"]), pair(d["second"])
    z, y, *stats = dcn.dcnv4_norm_scale_add_norm(x, gpu(d["residual"]), scale, gate, first, second, eps=eps)
    back = dcn.dcnv4_norm_scale_add_norm_backward(x, z, scale, gate, first, second, stats, gpu(d["grad_y"]), gpu(d["grad_z"]) if grad_z else None, **kw)
    return z, y, stats, dict(zip(NAMES, back))


def norm_slack(x, gamma, beta, mean, rstd):
    big = (np.abs(x).max(-1, keepdims=True) + np.abs(mean)[..., None]) * rstd[..., None] + 1
    return 64 * E * (big * np.abs(gamma) + np.abs(beta))


def check(d, dtype, eps, grad_z=True):
    C = d["x"].shape[-1]
    first, second = plain(d["first"], C), plain(d["second"], C)
    z, y, stats, back = run(d, eps, grad_z)
    x64 = d["x"].astype(np.float64)
    wz, b = ref.end(d["x"], d["residual"], d["scale"], d["gate"], first, eps)
    by = np.ones(x64.shape[0]) if d["gate"] is None else d["gate"].astype(np.float64)
    by = np.abs(by.reshape(-1, *[1] * (x64.ndim - 1)) * (1.0 if d["scale"] is None else d["scale"].astype(np.float64)))
    slack = 4 * E * (by * np.abs(b) + np.abs(d["residual"]))
    if first is not None:
        _, m, r = ref.norm(x64, *first, eps)
        slack = slack + by * norm_slack(x64, *first, m, r)
        close("mean1", stats[0], m, 64 * E * np.abs(x64).mean(-1), "f32")
        close("rstd1", stats[1], r, 64 * E * r * (1 + np.abs(x64).max(-1) * r), "f32")
    else:
        assert stats[0] is None and stats[1] is None
    close("z", z, wz, slack, dtype)
    if second is not None:
        zs = h(z)
        wy, m, r = ref.norm(zs, *second, eps)
        close("y", y, wy, norm_slack(zs, *second, m, r), dtype)
        close("mean2", stats[2], m, 64 * E * np.abs(zs).mean(-1), "f32")
        close("rstd2", stats[3], r, 64 * E * r * (1 + np.abs(zs).max(-1) * r), "f32")
    else:
        assert y is None and stats[2] is None and stats[3] is None
    want = ref.end_backward(d["x"], h(z), d["scale"], d["gate"], first, second, [h(s) for s in stats], d["grad_y"], d["grad_z"] if grad_z else None)
    for name in NAMES:
        there = {"grad_scale": d["scale"] is not None, "grad_gate": d["gate"] is not None, "grad_gamma1": d["first"] and d["first"][0] is not None,
                 "grad_beta1": d["first"] and d["first"][1] is not None, "grad_gamma2": d["second"] and d["second"][0] is not None,
                 "grad_beta2": d["second"] and d["second"][1] is not None}.get(name, True)
        if not there:
            assert back[name] is None, name
            continue
        close(name, back[name], *want[name], "f32" if name == "grad_gate" else dtype)


# every lane count and its borders, odd widths, one row, one channel, one image and many
SHAPES = [(1, 1, 1), (3, 1, 1), (2, 5, 7), (1, 2, 8), (4, 3, 9), (1, 37, 16), (5, 60, 32), (3, 20, 33), (3, 41, 64), (2, 9, 127), (2, 50, 128), (7, 700, 96), (3, 11, 255), (4, 10, 256),
          (1, 7, 257), (3, 7, 321), (2, 32, 512), (1, 11, 513), (4, 300, 1024), (1, 5, 1025), (2, 3, 2048), (1, 3, 2049), (1, 5, 4096), (2, 1, 4099), (1, 3, 8192), (2, 2, 8191),
          (2, 20000, 16)]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("form", ["f", "s", "fs"])
def test_block_end(shape, form, dtype):
    check(draw(shape, dtype, form, sum(shape)), dtype, 1e-3 if shape[-1] < 3 else 1e-6)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("form", ["", "f", "s", "fs"])
@pytest.mark.parametrize("gate,scale,affine", [(False, True, True), (True, False, True), (True, True, False), (False, False, False)])
def test_what_may_be_left_out(form, gate, scale, affine, dtype):
    for shape in ((2, 9, 100), (3, 5, 7, 136)):
        check(draw(shape, dtype, form, 3, gate, scale, affine), dtype, 1e-5)


def test_one_of_gamma_and_beta():
    for keep in (0, 1):
        d = draw((2, 9, 100), "f32", "fs", 4)
        for n in ("first", "second"):
            d[n] = tuple(v if i == keep else None for i, v in enumerate(d[n]))
        check(d, "f32", 1e-5)


def test_no_gradient_down_the_residual_path():
    check(draw((2, 30, 72), "f16", "fs", 5), "f16", 1e-5, grad_z=False)
    check(draw((2, 30, 72), "f32", "s", 6), "f32", 1e-5, grad_z=False)


@pytest.mark.parametrize("form", ["", "f", "s", "fs"])
@pytest.mark.parametrize("C", [64, 100])
def test_a_gate_of_zero_hides_what_the_branch_holds(form, C):
    """NaN and infinities in images that are left out: results and gradients of all others are those without them."""
    d = draw((3, 7, C), "f16", form, 7)
    d["gate"][:] = [0.0, 1.5, 0.0]
    clean = run(d, 1e-5, grad_gate=False)
    d["x"][0] = np.nan
    d["x"][2, :, ::3] = np.inf
    dirty = run(d, 1e-5, grad_gate=False)
    assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[0][0], gpu(d["residual"])[0])
    assert clean[1] is None or torch.equal(clean[1], dirty[1])
    for name in NAMES:
        a, b = clean[3][name], dirty[3][name]
        assert a is None and b is None or torch.equal(a, b), name
    assert bool((dirty[3]["grad_x"][0] == 0).all()) and bool((dirty[3]["grad_x"][2] == 0).all()) and dirty[3]["grad_gate"] is None


def test_constant_rows_and_large_offsets():
    d = draw((2, 6, 200), "f32", "fs", 8)
    d["x"][0, :3] = 7.0
    d["x"][1] += 3000.0
    d["residual"][0, 1] = -1.0
    check(d, "f32", 1e-5)


def test_same_bits_from_run_to_run_and_with_a_stream():
    d = draw((5, 301, 200), "f16", "fs", 9)
    z, y, stats, back = run(d, 1e-6)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    x, scale, gate, first, second = gpu(d["x"]), gpu(d["scale"]), gpu(d["gate"]), pair(d["first"]), pair(d["second"])
    res, gy, gz = gpu(d["residual"]), gpu(d["grad_y"]), gpu(d["grad_z"])
    torch.cuda.synchronize()
    z2, y2, *stats2 = dcn.dcnv4_norm_scale_add_norm(x, res, scale, gate, first, second, stream=s)
    back2 = dcn.dcnv4_norm_scale_add_norm_backward(x, z2, scale, gate, first, second, stats2, gy, gz, stream=s)
    s.synchronize()
    assert torch.equal(z, z2) and torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(back.values(), back2))
    light = dcn.dcnv4_norm_scale_add_norm(x, res, scale, gate, first, second, stats=False)
    assert torch.equal(light[0], z) and torch.equal(light[1], y) and light[2:] == (None,) * 4


def test_nothing_is_written_behind_the_rows():
    for C in (20, 64, 321):
        d = draw((2, 13, C), "f16", "fs", 10)
        n, shape = 26 * C, (2, 13, C)
        room = {k: torch.full((n + 512,), 5.0, dtype=torch.float16, device="cuda") for k in ("z", "y", "grad_x", "grad_residual")}
        part = {k: v[:n].view(shape) for k, v in room.items()}
        f32 = lambda *s: torch.empty(s, device="cuda")
        x, scale, gate, first, second = gpu(d["x"]), gpu(d["scale"]), gpu(d["gate"]), pair(d["first"]), pair(d["second"])
        z, y, *stats = dcn.dcnv4_norm_scale_add_norm(x, gpu(d["residual"]), scale, gate, first, second,
                                                     out=[part["z"], part["y"]] + [f32(2, 13) for _ in range(4)])
        vec = lambda: torch.empty(C, dtype=torch.float16, device="cuda")
        dcn.dcnv4_norm_scale_add_norm_backward(x, z, scale, gate, first, second, stats, gpu(d["grad_y"]), gpu(d["grad_z"]),
                                               out=[part["grad_x"], part["grad_residual"], vec(), f32(2)] + [vec() for _ in range(4)])
        for k, v in room.items():
            assert bool((v[n:] == 5.0).all()), k
            assert bool((v[:n] != 5.0).any()), k


def test_captured_training_step_replays():
    d = draw((3, 50, 136), "f32", "fs", 11)
    t = {k: gpu(d[k]) for k in ("x", "residual", "scale", "gate", "grad_y", "grad_z")}
    first, second = pair(d["first"]), pair(d["second"])
    work = torch.empty(dcn.dcnv4_norm_scale_add_norm_workspace_bytes(150, 136, 3), dtype=torch.uint8, device="cuda")

    def step(work=None):
        z, y, *stats = dcn.dcnv4_norm_scale_add_norm(t["x"], t["residual"], t["scale"], t["gate"], first, second)
        return (z, y, *dcn.dcnv4_norm_scale_add_norm_backward(t["x"], z, t["scale"], t["gate"], first, second, stats, t["grad_y"], t["grad_z"], workspace=work))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(work)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step(work)
    for k in range(3):
        torch.cuda.synchronize()
        t["x"].normal_()
        t["gate"].fill_(0.5 * k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, step())), k


def test_refusals():
    x = torch.zeros((2, 3, 16), device="cuda")
    v, g, st = torch.zeros(16, device="cuda"), torch.ones(2, device="cuda"), torch.zeros((2, 3), device="cuda")
    end, back = dcn.dcnv4_norm_scale_add_norm, dcn.dcnv4_norm_scale_add_norm_backward
    for bad in (lambda: end(x, x[:, :2]), lambda: end(x, x.half()), lambda: end(x, x, v[:15]), lambda: end(x, x, v, g[:1]), lambda: end(x, x, v, g.half()),
                lambda: end(x, x, v, None, (v[:3], v)), lambda: end(x.transpose(0, 1), x), lambda: end(x[0, 0], x[0, 0], v, g),
                lambda: back(x, x, v, g, None, None, (None,) * 4, None), lambda: back(x, x, v, g, None, None, (None,) * 4, x, x),
                lambda: back(x, x, v, g, None, (v, v), (None, None, st, st), None, x), lambda: back(x, None, v, g, None, (v, v), (None, None, st, st), x, x),
                lambda: back(x, x, v, g, (v, v), None, (st, st[:1], None, None), None, x), lambda: end(x, x, out=[x.clone(), x.clone(), None, None, None, None])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(dcn.Dcnv4Error):
        end(torch.zeros((2, 8200), device="cuda"), torch.zeros((2, 8200), device="cuda"))
    with pytest.raises(dcn.Dcnv4Error):
        end(x, x, eps=-1.0)
    with pytest.raises(dcn.Dcnv4Error):
        back(x, x, v, g, None, None, (None,) * 4, None, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
