"""Softmax cross entropy out of the last linear layer, and its gradient, against the definition in double precision (torch, on the
GPU, from the same stored inputs).

Tolerances.  A logit is an fp32 sum of exact products, sixteen to an instruction that rounds twice at most: K / 8 + 8 roundings of
2^-23 (the matrix unit's addition) of the sum of magnitudes.  fp32 operands are held as three bf16 numbers, whose products leave out
2^-22 of a product at most.  The sum of exponentials: 64 terms in a lane's chain, 2 + 16 joins, an exponential and a logarithm, each
within 2^-22: 128 * 2^-23.  d is off by p times the error of logit - lse, and by its rounding, 2^-11 (fp16) or 2^-22 of it.  The gradients' sums
add (n / 8 + 80) * 2^-23 of the sum of magnitudes, n the length of the sum, and one rounding of the type."""
import numpy as np
import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11}
LEAST = {"f32": 0.0, "f16": 2.0 ** -25}
D_STEP = {"f32": 2.0 ** -22, "f16": 2.0 ** -11}
E = 2.0 ** -23
IGNORE = -100


def inputs(P, K, V, dtype, seed=0, ignored=0.2, bias=True):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000 + P + K + V)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    x, w = r(P, K).to(DT[dtype]), (r(V, K) * (2 / K ** 0.5)).to(DT[dtype])
    b = (0.3 * r(V)).to(DT[dtype]) if bias else None
    t = torch.randint(0, V, (P,), generator=gen, device="cuda")
    gone = torch.rand(P, generator=gen, device="cuda") < ignored
    t = torch.where(gone, torch.full_like(t, IGNORE), t)
    g = r(P) * (1024.0 if dtype == "f16" else 1.0)
    return x, w, b, t, g


def expected(x, w, b, t, g):
    """The definition, and what each result may be off by before its rounding."""
    f32 = x.dtype is torch.float32
    K, V = w.shape[1], w.shape[0]
    X, W = x.double(), w.double()
    B = torch.zeros(V, dtype=torch.float64, device="cuda") if b is None else b.double()
    logits, size = X @ W.T + B, X.abs() @ W.abs().T + torch.where(B.isfinite(), B, torch.zeros_like(B)).abs()
    off = ((K / 8 + 8) * E + (2.0 ** -22 if f32 else 0)) * size
    lse = torch.logsumexp(logits, -1)
    ok = t != IGNORE
    at = torch.where(ok, t, torch.zeros_like(t))[:, None]
    loss = torch.where(ok, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    lse_off = off.max(-1).values + 128 * E + 2 * E * lse.abs()
    loss_off = lse_off + off.max(-1).values + 2 * E * logits.gather(1, at)[:, 0].abs()
    p = (logits - lse[:, None]).exp()
    d = p.clone()
    d.scatter_add_(1, at, -torch.ones_like(lse)[:, None])
    d = d * ok[:, None]
    d_off = (p * (off + lse_off[:, None] + 4 * E * (1 + logits.abs().nan_to_num(posinf=0))) + D_STEP["f32" if f32 else "f16"] * d.abs() + 2.0 ** -39) * ok[:, None]
    G = g.double()[:, None] * ok[:, None]
    gd, gd_off = G * d, G.abs() * d_off
    top = G.abs().max() * 2
    gd_off_w = gd_off + D_STEP["f32" if f32 else "f16"] * gd.abs() + top * 2.0 ** -39
    P = x.shape[0]
    res = {"loss": (loss, loss_off), "lse": (lse, lse_off),
           "grad_x": (gd @ W, gd_off @ W.abs() + ((V / 8 + 80) * E + 2.0 ** -21) * (gd.abs() @ W.abs())),
           "grad_w": (gd.T @ X, gd_off_w.T @ X.abs() + ((P / 8 + 80) * E + 2.0 ** -21) * (gd.abs().T @ X.abs())),
           "grad_b": (gd.sum(0), gd_off_w.sum(0) + (P / 8 + 80) * E * gd.abs().sum(0))}
    return res


def close(name, got, want, dtype):
    ref, slack = want
    got = got.double()
    if dtype == "f16":                                                   # fp16 ends at 65504: from 65520 on it rounds to infinity
        ends = ref.abs() + slack >= 65520
        got = torch.where(ends & (got == ref.sign() * float("inf")), ref, got)
    err, lim = (got - ref).abs(), U[dtype] * (ref.abs() + slack) + LEAST[dtype] + slack
    bad = ~(err <= lim)
    if bad.any():
        i = int((err / lim).nan_to_num(nan=float("inf")).argmax())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off; at {np.unravel_index(i, ref.shape)} got {got.reshape(-1)[i].item()!r}, "
                             f"want {ref.reshape(-1)[i].item()!r}, limit {lim.reshape(-1)[i].item()!r}")


def check(P, K, V, dtype, seed=0, bias=True, ignored=0.2):
    x, w, b, t, g = inputs(P, K, V, dtype, seed, ignored, bias)
    want = expected(x, w, b, t, g)
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    close("loss", loss, want["loss"], "f32")
    close("lse", lse, want["lse"], "f32")
    assert not loss[t == IGNORE].any()
    got = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    for name, a in zip(("grad_x", "grad_w", "grad_b"), got):
        if a is not None:
            close(name, a, want[name], dtype)
    assert not got[0][t == IGNORE].any() and (got[2] is None) == (b is None)
    return (x, w, b, t, g), (loss, lse, *got)


SIZES = [(1, 16, 1), (1, 32, 2), (2, 16, 3), (3, 16, 5), (63, 64, 64), (64, 64, 63), (65, 48, 129), (130, 256, 150), (257, 96, 1000), (300, 128, 700),
         (100, 1040, 257), (1, 1024, 5000), (2000, 32, 2), (513, 512, 513)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("P,K,V", SIZES)
def test_loss_and_its_gradient(P, K, V, dtype):
    check(P, K, V, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("tile", [1, 2, 3])
@pytest.mark.parametrize("P,K,V", [(70, 80, 130), (301, 160, 515), (9, 96, 777)])
def test_every_tile(P, K, V, tile, dtype):
    dcn.dcnv4_set_option("loss_tile", tile)
    check(P, K, V, dtype, seed=tile)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("splits,piece", [(1, 256), (3, 0), (4, 256), (7, 512)])
def test_split_sums_and_pieces(splits, piece, dtype):
    dcn.dcnv4_set_option("loss_splits", splits)
    dcn.dcnv4_set_option("loss_piece", piece)
    check(700, 64, 1100, dtype, seed=splits)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_large(dtype):
    """Sizes that the library itself cuts into pieces, without a bias and with every row labelled."""
    P, V = (8192, 33001) if dtype == "f16" else (4096, 40009)
    check(P, 128, V, dtype, bias=False, ignored=0.0)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_results_do_not_change_from_run_to_run(dtype):
    (x, w, b, t, g), first = check(1000, 96, 1500, dtype, seed=3)
    for _ in range(2):
        loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
        again = (loss, lse, *dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b))
        assert all(torch.equal(a, c) for a, c in zip(first, again))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_masked_classes_rows_and_bad_targets(dtype):
    P, K, V = 90, 64, 200
    x, w, b, t, g = inputs(P, K, V, dtype, 5, ignored=0.3)
    # classes that a bias of -infinity takes out: probability 0, gradient 0
    b[7:150] = float("-inf")
    t = torch.where((t >= 7) & (t < 150), t * 0 + 3, t)
    want = expected(x, w, b, t, g)
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    gx, gw, gb = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    for name, a, ty in (("loss", loss, "f32"), ("lse", lse, "f32"), ("grad_x", gx, dtype), ("grad_w", gw, dtype), ("grad_b", gb, dtype)):
        close(name, a, want[name], ty)
    assert not gw[7:150].any() and not gb[7:150].any()
    # a masked target has infinite loss
    u = t.clone()
    u[0] = 20
    assert dcn.dcnv4_linear_cross_entropy(x, w, u, b)[0][0].item() == float("inf")
    # the type's lowest value in place of -infinity
    low = b.clone()
    low[7:150] = torch.finfo(DT[dtype]).min
    other = dcn.dcnv4_linear_cross_entropy(x, w, t, low)
    assert torch.equal(other[0], loss) and torch.equal(other[1], lse)
    # ignored rows, and rows without a gradient, count for nothing whatever they hold
    bad = x.clone()
    bad[t == IGNORE] = float("nan")
    quiet = g.clone()
    first = int((t != IGNORE).nonzero()[0])
    quiet[first] = 0
    base = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, quiet, b)
    bad[first] = float("inf")
    bad_lse = lse.clone()
    bad_lse[t == IGNORE] = float("nan")
    got = dcn.dcnv4_linear_cross_entropy_backward(bad, w, t, bad_lse, quiet, b)
    assert all(torch.equal(a, c) for a, c in zip(base, got))
    assert not dcn.dcnv4_linear_cross_entropy(bad, w, t, b)[0][t == IGNORE].any()
    # all rows ignored
    none = torch.full_like(t, IGNORE)
    got = dcn.dcnv4_linear_cross_entropy_backward(bad, w, none, bad_lse, g, b)
    assert not any(a.any() for a in got)
    # targets that are no class: NaN, here and in what they reach; the other rows as before
    for wrong in (V, -1, 2 ** 40, -2 ** 62):
        u = t.clone()
        u[first] = wrong
        loss2, lse2 = dcn.dcnv4_linear_cross_entropy(x, w, u, b)
        assert loss2[first].isnan() and torch.equal(loss2[first + 1:], loss[first + 1:]) and torch.equal(lse2, lse)
        gx2, gw2, _ = dcn.dcnv4_linear_cross_entropy_backward(x, w, u, lse2, g, b)
        assert gx2[first].isnan().all() and torch.equal(gx2[first + 1:], gx[first + 1:]) and gw2.isnan().any()
    # every class masked: there is no distribution
    assert dcn.dcnv4_linear_cross_entropy(x, w, t, torch.full_like(b, float("-inf")))[0][first].isnan()


def test_large_logits_and_small_gradients():
    """Logits of several hundred, and losses scaled by 2^-20 and 2^12: no overflow, no lost bits."""
    x, w, b, t, g = inputs(200, 64, 300, "f16", 8)
    x = x * 40
    want = expected(x, w, b, t, g)
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    close("loss", loss, want["loss"], "f32")
    close("lse", lse, want["lse"], "f32")
    x32, w32, b32 = x.float(), w.float(), b.float()
    for dtype, args in (("f16", (x, w, b)), ("f32", (x32, w32, b32))):
        for scale in (2.0 ** -20, 1.0, 2.0 ** 3):
            s = g * scale
            got = dcn.dcnv4_linear_cross_entropy_backward(args[0], args[1], t, lse, s, args[2])
            want = expected(*args, t, s)
            for name, a in zip(("grad_x", "grad_w", "grad_b"), got):
                close(f"{name} {dtype} {scale}", a, want[name], dtype)


def test_gradient_against_differences():
    rng = np.random.default_rng(0)
    P, K, V = 5, 8, 9
    x, w, b, g = (rng.standard_normal(s) for s in ((P, K), (V, K), V, P))
    t = np.array([0, 8, IGNORE, 3, 3])

    def value(x, w, b):
        z = x @ w.T + b
        lse = np.log(np.exp(z).sum(-1))
        return sum(g[i] * (lse[i] - z[i, t[i]]) for i in range(P) if t[i] != IGNORE)

    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    T = torch.from_numpy(t).cuda()
    loss, lse = dcn.dcnv4_linear_cross_entropy(f(x), f(w), T, f(b))
    assert abs((loss.double() * f(g).double()).sum().item() - value(x, w, b)) < 1e-5 * np.abs(g).sum() * 10
    got = dcn.dcnv4_linear_cross_entropy_backward(f(x), f(w), T, lse, f(g), f(b))
    h = 1e-5
    for which, grad in enumerate(got):
        grad = grad.double().cpu().numpy().reshape(-1)
        for i in range(grad.size):
            args = [a.copy() for a in (x, w, b)]
            args[which].reshape(-1)[i] += h
            up = value(*args)
            args[which].reshape(-1)[i] -= 2 * h
            # fp32 inputs (2^-24 of them) and sums, differences to h^2: 1e-5 covers them
            assert abs((up - value(*args)) / (2 * h) - grad[i]) < 1e-5 * (1 + abs(grad[i]))


def test_rows_behind_the_last_stay_as_they_were():
    for dtype in ("f16", "f32"):
        P, K, V = 37, 32, 71
        x, w, b, t, g = inputs(P, K, V, dtype)
        dt = DT[dtype]
        long = {n: torch.full((s + 128,), 7.0, device="cuda", dtype=ty) for n, s, ty in
                (("loss", P, torch.float32), ("lse", P, torch.float32), ("gx", P * K, dt), ("gw", V * K, dt), ("gb", V, dt))}
        loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b, out=(long["loss"][:P], long["lse"][:P]))
        dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b, out=(long["gx"][:P * K].view(P, K), long["gw"][:V * K].view(V, K), long["gb"][:V]))
        for n, s in (("loss", P), ("lse", P), ("gx", P * K), ("gw", V * K), ("gb", V)):
            assert bool((long[n][s:] == 7.0).all()), n


def test_streams_graphs_and_dirty_workspaces():
    """A captured pass replayed with new inputs, its workspace filled with NaNs before each replay."""
    x, w, b, t, g = inputs(400, 64, 600, "f16", 2)
    P, K, V = 400, 64, 600
    work = torch.empty(dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, True), dtype=torch.uint8, device="cuda")
    small = torch.empty(dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, False), dtype=torch.uint8, device="cuda")

    def run(own):
        loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b, workspace=small if own else None)
        return (loss, lse, *dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b, workspace=work if own else None))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(True)
    for k in range(3):
        torch.cuda.synchronize()
        x.normal_()
        t.random_(0, V)
        work.fill_(255)
        small.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = run(False)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), k


def test_refusals():
    x, w, b, t, g = inputs(4, 32, 40, "f16")
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    for call in (lambda: dcn.dcnv4_linear_cross_entropy(x, w.float(), t, b), lambda: dcn.dcnv4_linear_cross_entropy(x, w[:, :16], t, b),
                 lambda: dcn.dcnv4_linear_cross_entropy(x, w, t.int(), b), lambda: dcn.dcnv4_linear_cross_entropy(x, w, t[:3], b),
                 lambda: dcn.dcnv4_linear_cross_entropy(x, w, t, b[:39]), lambda: dcn.dcnv4_linear_cross_entropy(x.t(), w, t, b),
                 lambda: dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse.half(), g, b),
                 lambda: dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g.half(), b),
                 lambda: dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b, out=(x, w))):
        with pytest.raises(ValueError):
            call()
    out = torch.full((4,), 7.0, device="cuda")
    tiny = torch.empty(64, dtype=torch.uint8, device="cuda")
    with pytest.raises(dcn.Dcnv4Error) as e:
        dcn.dcnv4_linear_cross_entropy(x, w, t, b, workspace=tiny, out=(out, lse))
    assert e.value.status == 2
    odd = torch.zeros((4, 24), device="cuda", dtype=torch.float16)
    with pytest.raises(dcn.Dcnv4Error) as e:
        dcn.dcnv4_linear_cross_entropy(odd, torch.zeros((40, 24), device="cuda", dtype=torch.float16), t, out=(out, lse))
    assert e.value.status == 3
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_more_than_32_bits_of_bytes():
    """x of more than 4 GiB: the last rows are what a call on them alone gives, and gradients of zero weight stay out."""
    P, K, V = 2 ** 20 - 1, 2064, 40
    few, w, b, t0, _ = inputs(128, K, V, "f16", 4)
    x, t = few.repeat(P // 128 + 1, 1)[:P].contiguous(), t0.repeat(P // 128 + 1)[:P].contiguous()
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    g = torch.zeros(P, device="cuda")
    g[-100:] = 3.0
    got = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    tail = slice(P - 100, P)
    want = expected(x[tail], w, b, t[tail], g[tail])
    close("loss", loss[tail], want["loss"], "f32")
    close("grad_x", got[0][tail], want["grad_x"], "f16")
    assert not got[0][:P - 100].any()
    close("grad_w", got[1], want["grad_w"], "f16")
    close("grad_b", got[2], want["grad_b"], "f16")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_class_as_the_ignored_one(dtype):
    """ignore_index may be a class: its rows count for nothing, and it is a class for the others."""
    P, K, V = 200, 48, 6
    x, w, b, t, g = inputs(P, K, V, dtype, 6, ignored=0.0)
    other = torch.where(t == 3, torch.full_like(t, IGNORE), t)
    first = dcn.dcnv4_linear_cross_entropy(x, w, other, b)
    second = dcn.dcnv4_linear_cross_entropy(x, w, t, b, ignore_index=3)
    assert all(torch.equal(a, c) for a, c in zip(first, second))
    back = [dcn.dcnv4_linear_cross_entropy_backward(x, w, u, first[1], g, b, ignore_index=i) for u, i in ((other, IGNORE), (t, 3))]
    assert all(torch.equal(a, c) for a, c in zip(*back))


def test_one_vector_and_maps():
    """x of one vector, and of a map of pixels: targets, losses and gradients have its shape."""
    x, w, b, t, g = inputs(30, 32, 11, "f32", 7, ignored=0.0)
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    m = dcn.dcnv4_linear_cross_entropy(x.view(2, 3, 5, 32), w, t.view(2, 3, 5), b)
    assert m[0].shape == (2, 3, 5) and torch.equal(m[0].view(-1), loss)
    gx = dcn.dcnv4_linear_cross_entropy_backward(x.view(2, 3, 5, 32), w, t.view(2, 3, 5), m[1], g.view(2, 3, 5), b)[0]
    assert gx.shape == (2, 3, 5, 32) and torch.equal(gx.view(30, 32), dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)[0])
    one = dcn.dcnv4_linear_cross_entropy(x[0].clone(), w, t[0].clone(), b)
    assert one[0].shape == () and abs(one[0].item() - loss[0].item()) <= 1e-5


def test_more_logits_than_a_grid_has_lanes_for():
    """2^20 rows and 700001 classes: more than 2^39 logits, in several launches.  A row's sum has 2735 tiles, 171 of them one after the other and
    16 more joins, each within 3 * 2^-22 (two exponentials, a product, a sum): 2^-12.8 in all."""
    P, K, V = 2 ** 20, 16, 700001
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    x = torch.randn((P, K), generator=gen, device="cuda").half()
    w = torch.randn((V, K), generator=gen, device="cuda").half()
    t = torch.randint(0, V, (P,), generator=gen, device="cuda")
    t[-1] = V - 1
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t)
    rows = [0, 1, 255, 256, P // 2 - 1, P // 2, P - 257, P - 1]
    want = expected(x[rows], w, None, t[rows], torch.ones(len(rows), device="cuda"))
    for name, got in (("loss", loss), ("lse", lse)):
        ref, slack = want[name]
        close(name, got[rows], (ref, slack + 2.0 ** -12.8), "f32")


def test_workspaces_are_of_the_stream_of_the_call():
    """A call on a stream that is handed over, which has other work to do first: what the current stream allocates and writes after the
    call's return stays as it is."""
    x, w, b, t, g = inputs(700, 64, 500, "f16", 9)
    P, K, V = 700, 64, 500
    s = torch.cuda.Stream()
    want = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    back = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, want[1], g, b)
    m = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(4):
            m @ m
    got = dcn.dcnv4_linear_cross_entropy(x, w, t, b, stream=s)
    after = [torch.full((dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, False),), 7, dtype=torch.uint8, device="cuda")]
    got_back = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, want[1], g, b, stream=s)
    after.append(torch.full((dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, True),), 7, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert all(bool((a == 7).all()) for a in after)
    assert all(torch.equal(a, c) for a, c in zip((*got, *got_back), (*want, *back)))


def test_prepared_arguments_need_their_tensors():
    x, w, b, t, g = inputs(40, 32, 50, "f16", 10)
    loss, lse = out = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    work = torch.empty(dcn.dcnv4_linear_cross_entropy_workspace_bytes(40, 32, 50, dcn.DCNV4_F16, True), dtype=torch.uint8, device="cuda")
    for kw in ({}, {"out": out}, {"workspace": work}):
        with pytest.raises(ValueError):
            dcn.dcnv4_linear_cross_entropy(x, w, t, b, prepare_only=True, **kw)
    new = tuple(torch.zeros_like(o) for o in out)
    args = dcn.dcnv4_linear_cross_entropy(x, w, t, b, out=new, workspace=work, prepare_only=True)
    assert dcn.load_library().dcnv4_linear_cross_entropy(*args) == 0
    torch.cuda.synchronize()
    assert torch.equal(new[0], loss) and torch.equal(new[1], lse)
