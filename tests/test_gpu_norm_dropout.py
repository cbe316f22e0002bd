"""Layer norm, dropout and the fused end of a residual branch against plain double-precision forms, through the C ABI.

Tolerances.  A result is rounded once: half a step, u = 2^-11 (fp16) or 2^-24 (fp32) of its size, and in fp16 at least half of the
smallest step, 2^-25.  Before that, fp32 sums: a sum of n terms in a chain of k additions is off by at most k * 2^-24 of the sum of their
magnitudes.  A row's sum has at most 32 terms a lane, 3 + 3 exchanges and 8 waves: k <= 32 + 6 + 8 = 46; with the handful of
operations around it 64 is more than any result can collect.  A sum over rows has at most P / (workgroups * rows side by side) + 32
+ 16 + 64 terms in a chain; the cases here keep that below 256."""
import numpy as np
import pytest
import torch

import training_ref as ref
from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

NP = {"f32": np.float32, "f16": np.float16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11}
LEAST = {"f32": 0.0, "f16": 2.0 ** -25}
E = 2.0 ** -24


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.cpu().numpy().astype(np.float64)


def close(name, got, want, dtype, slack):
    """|got - want| <= one rounding of the type + slack (elementwise)."""
    got, want = host(got), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    err, lim = np.abs(got - want), U[dtype] * (np.abs(want) + slack) + LEAST[dtype] + slack
    bad = ~(err <= lim)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, err, 0)), err.shape)
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} off; at {at} got {got[at]!r}, want {want[at]!r}, limit {lim[at]!r}")


def rows(rng, shape, dtype, shift=0.3):
    return (rng.standard_normal(shape) * 1.5 + shift).astype(NP[dtype])


# rows, channels: every width class and its borders, odd widths, one row, one channel, more rows than workgroups side by side
SIZES = [(1, 1), (3, 1), (5, 7), (2, 8), (1, 9), (37, 64), (300, 65), (9, 127), (50, 128), (5883, 96), (33, 255), (40, 256), (7, 257),
         (21, 321), (64, 512), (11, 513), (2500, 1024), (5, 1025), (6, 2048), (3, 2049), (5, 4096), (2, 4099), (3, 8192), (2, 8193),
         (2, 16384), (1, 16383), (70000, 16)]


def slack_of_norm(x, gamma, beta, mean, rstd):
    """64 roundings of what (x - mean) * rstd is made of, and of gamma and beta around it."""
    big = (np.abs(x).max(-1, keepdims=True) + np.abs(mean)[..., None]) * rstd[..., None] + 1
    g = 1.0 if gamma is None else np.abs(gamma.astype(np.float64))
    b = 0.0 if beta is None else np.abs(beta.astype(np.float64))
    return 64 * E * (big * g + b)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("P,C", SIZES)
def test_layer_norm_and_its_gradient(P, C, dtype):
    rng = np.random.default_rng(P * 3 + C)
    x, gy = rows(rng, (P, C), dtype), rows(rng, (P, C), dtype, 0.0)
    gamma, beta = rows(rng, C, dtype, 1.0), rows(rng, C, dtype, 0.0)
    eps = 1e-3 if C < 3 else 1e-6              # (one channel has no variance: rstd = eps^-1/2)
    y, mean, rstd = dcn.dcnv4_layer_norm(gpu(x), gpu(gamma), gpu(beta), eps=eps, stats=True)
    wy, wm, wr = ref.layer_norm(x, gamma, beta, eps)
    x64 = x.astype(np.float64)
    close("y", y, wy, dtype, slack_of_norm(x64, gamma, beta, wm, wr))
    close("mean", mean, wm, "f32", 64 * E * np.abs(x64).mean(-1))
    # d rstd / rstd = half the error of the variance, whose terms are off by that of the mean
    close("rstd", rstd, wr, "f32", 64 * E * wr * (1 + np.abs(x64).max(-1) * wr))
    assert torch.equal(dcn.dcnv4_layer_norm(gpu(x), gpu(gamma), gpu(beta), eps=eps), y)
    got = dcn.dcnv4_layer_norm_backward(gpu(x), gpu(gamma), mean, rstd, gpu(gy))
    m, r = mean.cpu().numpy(), rstd.cpu().numpy()
    want, size = ref.layer_norm_backward(x, gamma, m, r, gy)
    xhat_off = 4 * E * (np.abs(x64).max() + np.abs(m).max()) * np.abs(r).max()      # of xhat, absolutely
    g_size = np.abs(gy.astype(np.float64) * gamma.astype(np.float64))
    close("grad_x", got[0], want[0], dtype,
          64 * E * size[0] + 2 * xhat_off * r[:, None] * (g_size.mean(-1, keepdims=True) + g_size) * (1 + np.abs(x64 - m[:, None]) * r[:, None]))
    close("grad_gamma", got[1], want[1], dtype, 256 * E * size[1] + xhat_off * size[2])
    close("grad_beta", got[2], want[2], dtype, 256 * E * size[2])
    again = dcn.dcnv4_layer_norm_backward(gpu(x), gpu(gamma), mean, rstd, gpu(gy))
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_layer_norm_without_parameters(dtype):
    rng = np.random.default_rng(5)
    x, gy = rows(rng, (4, 5, 72), dtype), rows(rng, (4, 5, 72), dtype)
    y, mean, rstd = dcn.dcnv4_layer_norm(gpu(x), stats=True)
    assert mean.shape == (4, 5)
    wy, wm, wr = ref.layer_norm(x, None, None, 1e-6)
    close("y", y, wy, dtype, slack_of_norm(x.astype(np.float64), None, None, wm, wr))
    gx, none, nothing = dcn.dcnv4_layer_norm_backward(gpu(x), None, mean, rstd, gpu(gy))
    assert none is None and nothing is None
    want, size = ref.layer_norm_backward(x, None, mean.cpu().numpy(), rstd.cpu().numpy(), gy)
    close("grad_x", gx, want[0], dtype, 128 * E * (size[0] + 1))
    gamma = rows(rng, 72, dtype)
    only = dcn.dcnv4_layer_norm(gpu(x), gpu(gamma))
    close("y of gamma alone", only, ref.layer_norm(x, gamma, None, 1e-6)[0], dtype, slack_of_norm(x.astype(np.float64), gamma, None, wm, wr))


def test_layer_norm_far_from_zero_and_constant_rows():
    """Rows whose mean is thousands of times their spread keep it; a constant row gives beta."""
    rng = np.random.default_rng(6)
    x = (4096 + rng.integers(-8, 9, (6, 200))).astype(np.float32)
    x[3] = 4096
    beta = np.arange(200, dtype=np.float32)
    y = host(dcn.dcnv4_layer_norm(gpu(x), None, gpu(beta)))
    want, _, rstd = ref.layer_norm(x, None, beta, 1e-6)
    assert np.array_equal(y[3], beta)
    keep = [0, 1, 2, 4, 5]
    # the mean is off by at most 46 roundings of 4096, 1e-2 of a spread of about 5
    assert np.abs(y[keep] - want[keep]).max() <= 46 * 4096 * E * rstd[keep].max() * 2 + 64 * E * 210


def test_layer_norm_infinities_and_nans_stay_in_their_rows():
    x = torch.randn((5, 130), device="cuda")
    clean = dcn.dcnv4_layer_norm(x)
    x[1, 7], x[3, 129] = float("inf"), float("nan")
    y = dcn.dcnv4_layer_norm(x)
    assert torch.isnan(y[1]).all() and torch.isnan(y[3]).all()
    assert all(torch.equal(y[r], clean[r]) for r in (0, 2, 4))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 100003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout_and_its_gradient(n, p, dtype):
    rng = np.random.default_rng(n)
    x, r = rows(rng, n, dtype), rows(rng, n, dtype)
    seed, offset = 2 ** 63 + 12345, 2 ** 40 + n
    # a product by the rounded scale, and a sum: three roundings
    y = dcn.dcnv4_dropout(gpu(x), p, seed, offset)
    want = ref.dropout(x, p, seed, offset)
    gone = ref.dropped(n, p, seed, offset)
    assert np.array_equal(host(y)[gone], np.zeros(gone.sum()))
    close("y", y, want, dtype, 3 * E * np.abs(want))
    z = dcn.dcnv4_dropout(gpu(x), p, seed, offset, residual=gpu(r))
    close("z", z, want + r.astype(np.float64), dtype, 3 * E * (np.abs(want) + np.abs(r.astype(np.float64))))
    g = dcn.dcnv4_dropout_backward(gpu(x), p, seed, offset)
    assert torch.equal(g, y)                                             # the same linear map
    if p == 0.0:
        assert torch.equal(y, gpu(x))


def test_dropout_rate_offsets_and_seeds():
    """The share of dropped elements, and that other seeds and offsets drop others."""
    x = torch.ones(1 << 20, device="cuda")
    kept = lambda seed, offset: dcn.dcnv4_dropout(x, 0.3, seed, offset) != 0
    a = kept(1, 0)
    # five standard deviations of 2^20 decisions
    assert abs(a.float().mean().item() - 0.7) < 5 * (0.21 / (1 << 20)) ** 0.5 + 2.0 ** -16
    for other in (kept(2, 0), kept(1, 1), kept(1 + (1 << 32), 0), kept(1, 1 << 32)):
        agree = (other == a).float().mean().item()                       # 0.7^2 + 0.3^2 = 0.58
        assert abs(agree - 0.58) < 0.005
    assert torch.equal(a, kept(1, 0)) and torch.equal(a, kept(1 + (1 << 64), 0))


def test_dropped_elements_give_zero_whatever_they_hold():
    n, p = 4096, 0.4
    gone = ref.dropped(n, p, 9, 3)
    x = np.ones(n, np.float32)
    x[gone] = np.nan
    y = host(dcn.dcnv4_dropout(gpu(x), p, 9, 3))
    assert np.isfinite(y).all() and not y[gone].any()
    x[gone] = np.inf
    z, ln, _, _ = dcn.dcnv4_dropout_add_layer_norm(gpu(x.reshape(16, 256)), torch.zeros((16, 256), device="cuda"), None, None, p, 9, 3)
    assert torch.isfinite(z).all() and torch.isfinite(ln).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("P,C", [(1, 1), (5, 7), (37, 64), (300, 65), (2, 127), (21, 321), (64, 512), (11, 515), (1500, 1024), (5, 2050), (3, 4096),
                                 (2, 8193), (2, 16384), (20000, 16)])
def test_branch_end_and_its_gradient(P, C, dtype):
    rng = np.random.default_rng(P + C)
    x, r = rows(rng, (P, C), dtype), rows(rng, (P, C), dtype)
    gamma, beta = rows(rng, C, dtype, 1.0), rows(rng, C, dtype, 0.0)
    p, seed, offset, eps = 0.25, -3, 77, 1e-3
    z, y, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(gpu(x), gpu(r), gpu(gamma), gpu(beta), p, seed, offset, eps=eps)
    # the sum is dropout's, and the norm is the layer norm of what was stored
    assert torch.equal(z, dcn.dcnv4_dropout(gpu(x), p, seed, offset, residual=gpu(r)))
    alone = dcn.dcnv4_layer_norm(z, gpu(gamma), gpu(beta), eps=eps, stats=True)
    assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd), alone))
    gone = ref.dropped(P * C, p, seed, offset).reshape(P, C)
    assert np.array_equal(host(z)[gone], r.astype(np.float64)[gone])
    gy, gz = rows(rng, (P, C), dtype, 0.0), rows(rng, (P, C), dtype, 0.0)
    args = (z, gpu(gamma), mean, rstd, gpu(gy), p, seed, offset)
    gx, gr, gg, gb = dcn.dcnv4_dropout_add_layer_norm_backward(*args, grad_z=gpu(gz))
    nx, ng, nb = dcn.dcnv4_layer_norm_backward(z, gpu(gamma), mean, rstd, gpu(gy))
    assert torch.equal(gg, ng) and torch.equal(gb, nb)
    want, size = ref.layer_norm_backward(z.cpu().numpy(), gamma, mean.cpu().numpy(), rstd.cpu().numpy(), gy)
    z64, m, rs = host(z), mean.cpu().numpy(), rstd.cpu().numpy()
    xhat_off = 4 * E * (np.abs(z64).max() + np.abs(m).max()) * rs.max()
    g_size = np.abs(gy.astype(np.float64) * gamma.astype(np.float64))
    slack = 64 * E * (size[0] + np.abs(gz.astype(np.float64))) + 2 * xhat_off * rs[:, None] * (g_size.mean(-1, keepdims=True) + g_size) * \
        (1 + np.abs(z64 - m[:, None]) * rs[:, None])
    total = want[0] + gz.astype(np.float64)
    close("grad_residual", gr, total, dtype, slack)
    close("grad_x", gx, np.where(gone, 0, total / 0.75), dtype, (slack + 3 * E * np.abs(total)) / 0.75)
    assert not host(gx)[gone].any()
    # without the other path's gradient: the norm's own
    gx0, gr0, _, _ = dcn.dcnv4_dropout_add_layer_norm_backward(*args)
    assert torch.equal(gr0, nx)


def test_gradient_of_the_branch_end_against_differences():
    """grad_x, grad_residual, grad_gamma, grad_beta as slopes of sum(y * gy + z * gz), in double precision on the host."""
    rng = np.random.default_rng(3)
    P, C, p, seed, offset, eps = 3, 11, 0.3, 4, 1, 1e-2
    x, r, gamma, beta, gy, gz = (rng.standard_normal(s) for s in ((P, C), (P, C), C, C, (P, C), (P, C)))

    def value(x, r, gamma, beta):
        z = ref.dropout(x, p, seed, offset, residual=r)
        return (ref.layer_norm(z, gamma, beta, eps)[0] * gy + z * gz).sum()

    f = lambda a: gpu(a.astype(np.float32))
    z, _, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(f(x), f(r), f(gamma), f(beta), p, seed, offset, eps=eps)
    got = dcn.dcnv4_dropout_add_layer_norm_backward(z, f(gamma), mean, rstd, f(gy), p, seed, offset, grad_z=f(gz))
    h = 1e-5
    for which, g in enumerate(got):
        g = host(g).reshape(-1)
        for i in range(g.size):
            args = [a.copy() for a in (x, r, gamma, beta)]
            args[which].reshape(-1)[i] += h
            up = value(*args)
            args[which].reshape(-1)[i] -= 2 * h
            slope = (up - value(*args)) / (2 * h)
            # differences: h^2 of third derivatives of order 10^3, 1e-7; fp32: inputs rounded (2^-24 of them), 1e-5 at most
            assert abs(slope - g[i]) <= 2e-5 * (1 + abs(slope)), (which, i, slope, g[i])


def test_rows_behind_the_last_stay_as_they_were():
    """Outputs that are views of longer buffers: what lies behind is not written, odd sizes among them."""
    for P, C in ((3, 7), (2, 64), (5, 321), (1, 2049)):
        for dt in (torch.float16, torch.float32):
            x = torch.randn((P, C), device="cuda", dtype=dt)
            buffers = [torch.full((P * C + 64,), 7.0, device="cuda", dtype=dt) for _ in range(4)]
            z, y, gx, gr = (b[:P * C].view(P, C) for b in buffers)
            mean, rstd = torch.empty(P, device="cuda"), torch.empty(P, device="cuda")
            gamma = torch.ones(C, device="cuda", dtype=dt)
            dcn.dcnv4_dropout_add_layer_norm(x, x, gamma, None, 0.1, 1, out=(z, y, mean, rstd))
            gg = torch.full((C + 8,), 7.0, device="cuda", dtype=dt)
            gb = torch.full((C + 8,), 7.0, device="cuda", dtype=dt)
            dcn.dcnv4_dropout_add_layer_norm_backward(z, gamma, mean, rstd, x, 0.1, 1, out=(gx, gr, gg[:C], gb[:C]))
            for b in buffers:
                assert bool((b[P * C:] == 7.0).all())
            assert bool((gg[C:] == 7.0).all()) and bool((gb[C:] == 7.0).all())
            d = torch.full((P * C + 64,), 7.0, device="cuda", dtype=dt)
            dcn.dcnv4_dropout(x, 0.1, 1, out=d[:P * C].view(P, C))
            assert bool((d[P * C:] == 7.0).all()) and torch.equal(d[:P * C].view(P, C), dcn.dcnv4_dropout(x, 0.1, 1))


def test_other_streams_and_graphs():
    """A captured step, its offset advanced on the device, replayed with eager work between: every replay equals the eager calls."""
    P, C = 333, 200
    x, r, gy = (torch.randn((P, C), device="cuda", dtype=torch.float16) for _ in range(3))
    gamma, beta = torch.randn(C, device="cuda", dtype=torch.float16), torch.randn(C, device="cuda", dtype=torch.float16)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    work = torch.empty(dcn.dcnv4_layer_norm_workspace_bytes(P, C), dtype=torch.uint8, device="cuda")

    def run(offset, on_device):
        z, y, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(x, r, gamma, beta, 0.2, 11, offset, offset_on_device=on_device)
        back = dcn.dcnv4_dropout_add_layer_norm_backward(z, gamma, mean, rstd, gy, 0.2, 11, offset, offset_on_device=on_device, grad_z=gy,
                                                         workspace=work)
        d = dcn.dcnv4_dropout(x, 0.5, 3, offset, offset_on_device=on_device)
        return (z, y, *back, d, dcn.dcnv4_dropout_backward(gy, 0.5, 3, offset, offset_on_device=on_device))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(100, step)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(100, step)
    torch.cuda.synchronize()
    seen = []
    for k in range(3):
        x.normal_()
        step.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        want = run(100 + k, None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        seen.append(got[-2] == 0)
    assert not torch.equal(seen[0], seen[1])


def test_refusals():
    x = torch.zeros((4, 40), device="cuda", dtype=torch.float16)
    for bad in (torch.zeros((4, 40), device="cuda"), torch.zeros((4, 40), dtype=torch.float16), torch.zeros((40, 4), device="cuda", dtype=torch.float16).t(),
                torch.zeros((4, 41), device="cuda", dtype=torch.float16)):
        with pytest.raises(ValueError):
            dcn.dcnv4_dropout(x, 0.1, 1, residual=bad)
        with pytest.raises(ValueError):
            dcn.dcnv4_dropout_add_layer_norm(x, bad, None, None, 0.1, 1)
    stat = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        dcn.dcnv4_layer_norm(x, torch.zeros(39, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        dcn.dcnv4_layer_norm_backward(x, None, stat.half(), stat, x)
    with pytest.raises(ValueError):
        dcn.dcnv4_dropout(x, 0.1, 1, offset_on_device=torch.zeros(1, device="cuda"))
    with pytest.raises(TypeError):
        dcn.dcnv4_layer_norm(torch.zeros((4, 40), device="cuda", dtype=torch.bfloat16))
    out = torch.full((4, 40), 7.0, device="cuda", dtype=torch.float16)
    cases = [(3, lambda: dcn.dcnv4_dropout(x, 1.5, 1, out=out)), (3, lambda: dcn.dcnv4_dropout(x, float("nan"), 1, out=out)),
             (3, lambda: dcn.dcnv4_layer_norm(x, eps=-1.0, out=out)), (1, lambda: dcn.dcnv4_layer_norm(x[:0])),          # (an empty tensor has no address)
             (4, lambda: dcn.dcnv4_dropout(x.view(-1)[1:33], 0.1, 1)),
             (2, lambda: dcn.dcnv4_layer_norm_backward(x, x[0], stat, stat, x, workspace=torch.empty(16, device="cuda")))]
    for status, call in cases:
        with pytest.raises(dcn.Dcnv4Error) as e:
            call()
        assert e.value.status == status
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_more_than_32_bits_of_elements():
    """2^32 elements and more: what lies behind them is what the definition says, and what a call on the end alone gives."""
    n, p, seed, offset = 2 ** 32 + 13, 0.5, 21, 4
    x = torch.ones(n, device="cuda", dtype=torch.float16)
    y = dcn.dcnv4_dropout(x, p, seed, offset)
    for first in (0, 2 ** 31 - 5, 2 ** 32 - 100):
        count = min(500, n - first)
        gone = ref.dropped(count, p, seed, offset, first=first)
        assert np.array_equal(y[first:first + count].cpu().numpy() == 0, gone)
    del x, y
    P, C = 2 ** 20 + 3, 2056
    x = torch.randn((64, C), device="cuda", dtype=torch.float16).repeat(P // 64 + 1, 1)[:P].contiguous()
    gamma = torch.randn(C, device="cuda", dtype=torch.float16)
    y, mean, rstd = dcn.dcnv4_layer_norm(x, gamma, stats=True)
    last = x[-70:].clone()
    alone = dcn.dcnv4_layer_norm(last, gamma, stats=True)
    assert all(torch.equal(a[-70:], b) for a, b in zip((y, mean, rstd), alone))
    gx, _, _ = dcn.dcnv4_layer_norm_backward(x, gamma, mean, rstd, y)
    only, _, _ = dcn.dcnv4_layer_norm_backward(last, gamma, alone[1], alone[2], alone[0])
    assert torch.equal(gx[-70:], only)


def test_explicit_streams():
    """A call on a stream that is handed over runs there, whatever stream is current."""
    x = torch.randn((64, 100), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = dcn.dcnv4_layer_norm(x, stream=s)
    d = dcn.dcnv4_dropout(x, 0.5, 1, residual=y, stream=s)
    s.synchronize()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, dcn.dcnv4_layer_norm(x)) and torch.equal(d, dcn.dcnv4_dropout(x, 0.5, 1, residual=y))


def test_one_parameter_gradient_alone():
    """grad_gamma or grad_beta may be left out, also where there is no gamma; numbers of numpy's types are numbers."""
    P, C = 40, 72
    x, gy = torch.randn((P, C), device="cuda"), torch.randn((P, C), device="cuda")
    gamma = torch.randn(C, device="cuda")
    _, mean, rstd = dcn.dcnv4_layer_norm(x, gamma, eps=np.float32(1e-5), stats=True)
    both = dcn.dcnv4_layer_norm_backward(x, gamma, mean, rstd, gy)
    work = torch.empty(dcn.dcnv4_layer_norm_workspace_bytes(P, C), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for keep in (1, 2):
        out = [torch.empty_like(x), torch.empty_like(gamma) if keep == 1 else None, torch.empty_like(gamma) if keep == 2 else None]
        ptr = [None if t is None else t.data_ptr() for t in (x, gamma, mean, rstd, gy, *out)]
        assert dcn.load_library().dcnv4_layer_norm_backward(*ptr, work.data_ptr(), work.numel(), P, C, 0, stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(out[0], both[0]) and torch.equal(out[keep], both[keep])
    # a norm with beta alone
    gx, gb = torch.empty_like(x), torch.empty_like(gamma)
    assert dcn.load_library().dcnv4_layer_norm_backward(x.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), gy.data_ptr(), gx.data_ptr(), None,
                                                        gb.data_ptr(), work.data_ptr(), work.numel(), P, C, 0, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(gb, both[2]) and torch.equal(gx, dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy)[0])
    a = dcn.dcnv4_dropout(x, np.float64(0.5), np.int64(-7), np.int32(3))
    assert torch.equal(a, dcn.dcnv4_dropout(x, 0.5, 2 ** 64 - 7, 3))


def test_workspaces_are_of_the_stream_of_the_call():
    """A call on a stream that is handed over, which has other work to do first: what the current stream allocates and writes after the
    call's return stays as it is."""
    P, C = 3000, 130
    x, gy = torch.randn((P, C), device="cuda"), torch.randn((P, C), device="cuda")
    gamma = torch.randn(C, device="cuda")
    _, mean, rstd = dcn.dcnv4_layer_norm(x, gamma, stats=True)
    norm = lambda **kw: dcn.dcnv4_layer_norm_backward(x, gamma, mean, rstd, gy, **kw)
    branch = lambda **kw: dcn.dcnv4_dropout_add_layer_norm_backward(x, gamma, mean, rstd, gy, 0.3, 5, **kw)
    m = torch.randn((4096, 4096), device="cuda")
    s = torch.cuda.Stream()
    for call in (norm, branch):
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(4):
                m @ m
        got = call(stream=s)
        after = torch.full((dcn.dcnv4_layer_norm_workspace_bytes(P, C),), 7, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert bool((after == 7).all()) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_prepared_arguments_need_their_tensors():
    x = torch.randn((8, 40), device="cuda")
    gamma, stat = torch.ones(40, device="cuda"), torch.ones(8, device="cuda")
    y = torch.empty_like(x)
    for call in (lambda **kw: dcn.dcnv4_layer_norm(x, **kw), lambda **kw: dcn.dcnv4_dropout(x, 0.5, 1, **kw),
                 lambda **kw: dcn.dcnv4_dropout_backward(x, 0.5, 1, **kw)):
        with pytest.raises(ValueError):
            call(prepare_only=True)
        assert call(prepare_only=True, out=y)
    with pytest.raises(ValueError):
        dcn.dcnv4_layer_norm_backward(x, gamma, stat, stat, x, out=(y, gamma.clone(), gamma.clone()), prepare_only=True)
    with pytest.raises(ValueError):
        dcn.dcnv4_dropout_add_layer_norm(x, x, None, None, 0.1, 1, prepare_only=True)
    args = dcn.dcnv4_layer_norm_backward(x, None, stat, stat, x, out=(y, None, None), prepare_only=True)
    assert dcn.load_library().dcnv4_layer_norm_backward(*args) == 0
    torch.cuda.synchronize()
    assert torch.equal(y, dcn.dcnv4_layer_norm_backward(x, None, stat, stat, x)[0])
