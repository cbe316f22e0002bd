"""Calls of the layers, the block's end and AdamW at the edges of what they take: tensors past 2^32 bytes, gradients asked for one by one, results on a
stream that is handed over, a workspace that two captured graphs share, parameters that autograd knows.

Tolerances.  Where a part of a call is the same call on a part of the rows, its bits are the same.  Sums over all rows are compared with 64 bits as 2-norms: two
roundings of half a step each (d, and the result), uniform ones of 0.58 of that, leave what fp32 sums of 2^24 numbers of either sign need: sixteen at once, they are
off by at most sqrt(2^24 / 16 / 2) * 2^-24 < 2^-14 of the sum's size."""
import ctypes

import pytest
import torch

from paper_2401_06197_amd import binding as dcn
from test_gpu_streams_of_results import check

pytestmark = pytest.mark.gpu

U16 = 2.0 ** -11


def normal(*shape, dtype=torch.float16, seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", dtype=dtype, generator=gen).mul_(size)


def near(got, want, limit=2 * U16):
    got = got.double()
    assert bool(torch.isfinite(got).all())
    assert float((got - want).norm() / want.norm()) <= limit


def pieces(P, at=1 << 20):
    return [slice(i, min(i + at, P)) for i in range(0, P, at)]


def test_linear_backward_past_32_bit_offsets():
    P, K, N = 2 ** 24, 136, 16
    x, w, gy = normal(P, K, seed=1), normal(N, K, seed=2, size=0.1), normal(P, N, seed=3, size=0.05)
    assert x.nbytes > 2 ** 32
    gx, gw, gb = dcn.dcnv4_linear_backward(x, w, gy, torch.zeros(N, device="cuda", dtype=torch.float16))
    for rows in (slice(0, 1000), slice(2 ** 24 - 1000, 2 ** 24)):
        near(gx[rows], gy[rows].double() @ w.double())
    near(gw, sum(gy[c].double().t().contiguous() @ x[c].double() for c in pieces(P)))
    near(gb, gy.double().sum(0))


def test_gated_layer_past_32_bit_offsets():
    P, K, F = 2 ** 24, 16, 136
    x, w, b, gh = normal(P, K, seed=1), normal(2, F, K, seed=2, size=0.25), normal(2, F, seed=3, size=0.3), normal(P, F, seed=4, size=0.05)
    assert gh.nbytes > 2 ** 32
    h = dcn.dcnv4_gated_linear(x, w, b)
    gx, gw, gb = dcn.dcnv4_gated_linear_backward(x, w, gh, b)
    wd, bd = w.double(), b.double()
    sum_w, sum_b = torch.zeros_like(wd), torch.zeros_like(bd)
    for c in pieces(P):
        xd, g = x[c].double(), gh[c].double()
        a, u = xd @ wd[0].t().contiguous() + bd[0], xd @ wd[1].t().contiguous() + bd[1]
        s = torch.sigmoid(a)
        d = torch.stack((g * u * s * (1 + a * (1 - s)), g * a * s))
        sum_w += torch.stack([t.t().contiguous() @ xd for t in d])
        sum_b += d.sum(1)
        if c.start == 0 or c.stop == P:
            near(h[c], a * s * u)
            near(gx[c], d[0] @ wd[0] + d[1] @ wd[1])
    near(gw, sum_w)
    near(gb, sum_b)


def test_block_end_past_32_bit_offsets():
    images, rows, C = 8, 2 ** 18, 1032
    shape = (images, rows, C)
    x, res, gy, gz = (normal(*shape, seed=i) for i in range(4))
    scale, gate = normal(C, seed=5), torch.tensor([1.25, 0.0, 1.25, 1.0, 0.5, 1.25, 0.0, 1.25], device="cuda")
    first, second = (normal(C, seed=6), normal(C, seed=7)), (normal(C, seed=8), normal(C, seed=9))
    assert x.nbytes > 2 ** 32 and x.numel() > 2 ** 31

    def both(i):
        by = gate[i].clone()                                   # (pointers are aligned to 16 bytes)
        z, y, *stats = dcn.dcnv4_norm_scale_add_norm(x[i], res[i], scale, by, first, second)
        return (z, y), dcn.dcnv4_norm_scale_add_norm_backward(x[i], z, scale, by, first, second, stats, gy[i], gz[i])

    (z, y), back = both(slice(0, images))
    totals, sizes = [0.0] * 8, [0.0] * 8
    for i in range(images):
        (z1, y1), one = both(slice(i, i + 1))
        if i in (0, images - 1):
            assert torch.equal(z1[0], z[i]) and torch.equal(y1[0], y[i]) and torch.equal(one[0][0], back[0][i]) and torch.equal(one[1][0], back[1][i])
        for k in range(2, 8):
            if k != 3:
                totals[k], sizes[k] = totals[k] + one[k].double(), sizes[k] + one[k].double().abs()
    for k in (2, 4, 5, 6, 7):
        # (each image's sum is rounded once, and the total)
        assert bool(((back[k].double() - totals[k]).abs() <= 1.1 * U16 * (sizes[k] + back[k].double().abs()) + 2.0 ** -20).all()), k


def test_gate_of_an_image_of_nearly_2_to_31_rows():
    P = 2 ** 31 - 1
    x, gz = normal(1, P, 1, seed=1), normal(1, P, 1, seed=2, size=0.5)
    gate = torch.tensor([0.75], device="cuda")
    z = dcn.dcnv4_norm_scale_add_norm(x, gz, None, gate)[0]
    for c in pieces(P, 2 ** 27):
        assert torch.equal(z[0, c], gz[0, c].float().add_(x[0, c].float(), alpha=0.75).half())   # (0.75 x is exact)
    del z
    grad_x, _, _, grad_gate, *_ = dcn.dcnv4_norm_scale_add_norm_backward(x, None, None, gate, None, None, (None,) * 4, None, gz)
    want = 0.0
    for c in pieces(P, 2 ** 27):
        want += float((x[0, c].double() * gz[0, c].double()).sum())
        assert torch.equal(grad_x[0, c], (gz[0, c].float() * 0.75).half())
    # (products are exact in fp32; sums in 64 bits, one rounding to fp32)
    assert abs(float(grad_gate[0]) - want) <= 2.0 ** -24 * abs(want) + 1e-3


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_past_32_bit_offsets(bits):
    n, part = 2 ** 31 + 256 * 3 + 77, 2 ** 20
    at = n // 256 * 256 - part
    p, g = normal(n, dtype=torch.float32, seed=1, size=0.1), normal(n, seed=2, size=0.02)
    if bits == 32:
        m, v, scales = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), None
    else:
        m, v = (torch.zeros(n, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2))
        scales = torch.zeros((-(-n // 256), 2), device="cuda")
    few = scales[at // 256:].clone() if bits == 8 else None
    end = [t[at:].clone() for t in (p, g, m.view(torch.uint8) if bits == 8 else m, v.view(torch.uint8) if bits == 8 else v)]
    if bits == 8:
        end[2:] = [t.view(torch.float8_e4m3fn) for t in end[2:]]
    large = dcn.dcnv4_adamw_plan([p], [g], [m], [v], 1e-2, 0.1, scales=None if few is None else [scales])
    small = dcn.dcnv4_adamw_plan(*[[t] for t in end], 1e-2, 0.1, scales=None if few is None else [few])
    dcn.dcnv4_adamw_step(large, 1)
    dcn.dcnv4_adamw_step(small, 1)
    assert torch.equal(end[0], p[at:]) and bool(torch.isfinite(p[-77:]).all()) and float((p[:4096] - normal(4096, dtype=torch.float32)).abs().max()) > 0
    if bits == 32:
        assert torch.equal(end[2], m[at:]) and torch.equal(end[3], v[at:])
    else:
        # (the roots of v are rounded by other random numbers, to one of the same two neighbours)
        code = lambda t: t.view(torch.uint8).int()
        assert torch.equal(code(end[2]), code(m[at:])) and torch.equal(few, scales[at // 256:])
        assert int((code(end[3]) - code(v[at:])).abs().max()) == 1


def ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gradients_one_by_one(dtype):
    """Each gradient alone, and each pair, through the C entry points: the bits that all three together have."""
    lib, code = dcn.load_library(), 1 if dtype is torch.float16 else 0
    for P, K, N in ((37, 48, 40), (700, 136, 264), (5000, 64, 96)):
        x, w, gy = normal(P, K, dtype=dtype, seed=1), normal(2, N, K, dtype=dtype, seed=2), normal(P, N, dtype=dtype, seed=3)
        b = normal(2, N, dtype=dtype, seed=4)
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        for gated in (False, True):
            if gated:
                want = dcn.dcnv4_gated_linear_backward(x, w, gy, b)
                need = dcn.dcnv4_gated_linear_workspace_bytes(P, K, N, code, True)
            else:
                want = dcn.dcnv4_linear_backward(x, w[0], gy, b[0].contiguous())
                need = dcn.dcnv4_linear_backward_workspace_bytes(P, K, N, code)
            space = torch.empty(need, dtype=torch.uint8, device="cuda")
            for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1)):
                got = [torch.full_like(t, 9.0) if a else None for t, a in zip(want, asked)]
                space.fill_(255)                               # (NaN, whatever it is read as)
                if gated:
                    rc = lib.dcnv4_gated_linear_backward(ptr(x), ptr(w), ptr(b), ptr(gy), *map(ptr, got), ptr(space), need, P, K, N, 0, code, stream)
                else:
                    rc = lib.dcnv4_linear_backward(ptr(x) if asked[1] else None, ptr(w) if asked[0] else None, ptr(gy), *map(ptr, got), ptr(space), need, P, K, N,
                                                   code, stream)
                assert rc == 0
                assert all(torch.equal(a, t) for a, t in zip(got, want) if a is not None), (P, gated, asked)


def calls():
    r = lambda *s: torch.randn(s, device="cuda")
    P, C, F = 1500, 264, 120
    x, res, gh, gy = r(4, P // 4, C), r(4, P // 4, C), r(4, P // 4, F), r(4, P // 4, C)
    w, b, scale, first, second, gate = r(2, F, C) / 16, r(2, F), r(C), (r(C), r(C)), (r(C), r(C)), torch.rand(4, device="cuda")
    z, _, *stats = dcn.dcnv4_norm_scale_add_norm(x, res, scale, gate, first, second)
    return {
        "gated layer": lambda **kw: dcn.dcnv4_gated_linear(x, w, b, **kw),
        "gated layer's gradient": lambda **kw: dcn.dcnv4_gated_linear_backward(x, w, gh, b, **kw),
        "linear layer's gradient": lambda **kw: dcn.dcnv4_linear_backward(x, w[0], gh, b[0].contiguous(), **kw),
        "block's end": lambda **kw: dcn.dcnv4_norm_scale_add_norm(x, res, scale, gate, first, second, **kw),
        "block's end's gradient": lambda **kw: dcn.dcnv4_norm_scale_add_norm_backward(x, z, scale, gate, first, second, stats, gy, res, **kw),
    }


@pytest.mark.parametrize("name", ["gated layer", "gated layer's gradient", "linear layer's gradient", "block's end", "block's end's gradient"])
def test_results_are_of_the_stream_of_the_call(name):
    check(calls()[name])


def test_two_graphs_with_one_workspace():
    """Two captured backward passes of other sizes in one workspace, replayed in turn on one stream."""
    sizes = ((600, 96, 136), (4100, 64, 72))
    ins = [(normal(P, K, seed=P), normal(2, F, K, seed=K, size=0.1), normal(P, F, seed=F)) for P, K, F in sizes]
    need = max(dcn.dcnv4_gated_linear_workspace_bytes(P, K, F, 1, True) for P, K, F in sizes)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for x, w, gh in ins:
        dcn.dcnv4_gated_linear_backward(x, w, gh)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(dcn.dcnv4_gated_linear_backward(x, w, gh, workspace=space))
        graphs.append(graph)
    for k in range(3):
        for x, _, gh in ins:
            x.normal_()
            gh.normal_().mul_(10.0 ** -k)
        torch.cuda.synchronize()
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        got = [[o.clone() for o in out[:2]] for out in outs]
        for (x, w, gh), g in zip(ins, got):
            assert all(torch.equal(a, c) for a, c in zip(g, dcn.dcnv4_gated_linear_backward(x, w, gh)))


def test_parameters_that_autograd_knows():
    """Leaves that require gradients: results are plain tensors, and a plan works on the leaves' memory, also after they are given other memory."""
    par = lambda *s: torch.nn.Parameter(torch.randn(s, device="cuda"))
    x, w, b, scale, gamma, beta = par(20, 64), par(2, 40, 64), par(2, 40), par(64), par(64), par(64)
    for r in (dcn.dcnv4_gated_linear(x, w, b), *dcn.dcnv4_gated_linear_backward(x, w, torch.ones((20, 40), device="cuda"), b),
              *dcn.dcnv4_norm_scale_add_norm(x, x, scale, None, (gamma, beta), (gamma, beta))):
        assert not r.requires_grad and r.grad_fn is None and type(r) is torch.Tensor
    before = w.detach().clone()
    held = w.data
    plan = dcn.dcnv4_adamw_plan([w], [torch.ones_like(w)], [torch.zeros_like(w)], [torch.zeros_like(w)], 0.1)
    with torch.no_grad():
        w.data = before.clone()
    dcn.dcnv4_adamw_step(plan, 1)
    torch.cuda.synchronize()
    assert torch.equal(w.detach(), before) and bool(((before.detach() - held - 0.1).abs() < 1e-5).all())
