"""AdamW over many tensors against a plain double-precision form, through the C ABI.

Tolerances.  Moments are made in 64 bits and rounded to fp32 once: half a step, 2^-24.  The move is a product of a rounded rate, m, and the reciprocal (one
step) of a fused product and sum of the rounded root: rate 1, rate * m 1, root 1/2 + the half of v's 1, unbias 1, sum 1, reciprocal 2, product 1, in
halves of fp32's steps: 8.  The parameter: decay, its fused product and the difference, 3.  Copies are rounded once more.  States of 8 bits have to be
the definition's, but where the rounded number is within two fp32 steps of a border between two of them."""
import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
BETAS, EPS = (0.9, 0.999), 1e-8
SIZES = [1, 7, 8, 9, 255, 256, 257, 511, 2047, 2048, 2049, 8191, 8192, 8193, 40001]


class Tensors:
    """Lists of tensors inside larger buffers whose rest has to stay as it is."""

    def __init__(self, sizes, dtype, bits, seed, copies=True):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits, self.dtype, self.guards = sizes, bits, dtype, []
        gt = torch.float16 if dtype == "f16" else torch.float32
        f = lambda a, t=torch.float32: torch.from_numpy(np.asarray(a, dtype=np.float32)).to(t)
        draw = lambda n, s: rng.standard_normal(n) * s
        self.p = [self.guarded(f(draw(n, 0.1))) for n in sizes]
        self.g = [self.guarded(f(draw(n, 0.02), gt)) for n in sizes]
        self.c = [self.guarded(f(np.zeros(n), torch.float16)) if copies and dtype == "f16" and i % 3 != 1 else None for i, n in enumerate(sizes)]
        self.s = None
        if bits == 8:
            f8 = torch.float8_e4m3fn
            self.m = [self.guarded(f(np.zeros(n), f8)) for n in sizes]
            self.v = [self.guarded(f(np.zeros(n), f8)) for n in sizes]
            self.s = [self.guarded(f(np.zeros((-(-n // 256), 2)))) for n in sizes]
        else:
            self.m = [self.guarded(f(draw(n, 0.01))) for n in sizes]
            self.v = [self.guarded(f(draw(n, 0.01) ** 2)) for n in sizes]

    def guarded(self, t):
        room = torch.full((t.numel() + 2 * 64,), 3.0, dtype=t.dtype if t.element_size() > 1 else torch.float32, device="cuda")
        if t.element_size() == 1:
            room = room.to(t.dtype)
        room[64:64 + t.numel()] = t.reshape(-1).cuda()
        self.guards.append((room, t.numel()))
        return room[64:64 + t.numel()].view(t.shape)

    def plan(self, lr=1e-2, wd=0.1):
        return dcn.dcnv4_adamw_plan(self.p, self.g, self.m, self.v, lr, wd, scales=self.s, copies=self.c if any(c is not None for c in self.c) else None)

    def check_guards(self):
        for room, n in self.guards:
            assert bool((room[:64].float() == 3.0).all()) and bool((room[64 + n:].float() == 3.0).all())

    def states(self, i):
        """m and v of tensor i as they stand, in 64 bits."""
        h = lambda t: t.float().double().cpu().numpy().reshape(-1)
        if self.bits == 32:
            return h(self.m[i]), h(self.v[i])
        s = np.repeat(self.s[i].double().cpu().numpy(), 256, axis=0)[:self.sizes[i]]
        return h(self.m[i]) * s[:, 0], (h(self.v[i]) * s[:, 1]) ** 2


def h(t):
    return t.float().double().cpu().numpy()


def step_and_check(ts, plan, t, lrs, wds, seed=0, factors=None, betas=BETAS, eps=EPS, on_device=0):
    count = len(ts.sizes)
    before = [(h(ts.p[i]), h(ts.g[i]), *ts.states(i)) for i in range(count)]
    f = None if factors is None else torch.tensor(factors, dtype=torch.float32, device="cuda")
    more = torch.tensor([on_device], device="cuda") if on_device else None
    dcn.dcnv4_adamw_step(plan, t - on_device, betas=betas, eps=eps, seed=seed, step_on_device=more, factors_on_device=f)
    torch.cuda.synchronize()
    used = (1.0, 1.0) if f is None else tuple(f.double().tolist())
    for i in range(count):
        p, g, m, v = before[i]
        wp, wm, wv, move = ref.adamw(p, g, m, v, lrs[i], wds[i], betas, eps, t, used)
        lim = 3 * E * (np.abs(p) + move) + 8 * E * move + 2.0 ** -126
        got = h(ts.p[i])
        assert np.all(np.abs(got - wp) <= lim), (i, np.max(np.abs(got - wp) / lim))
        if ts.c[i] is not None:
            assert torch.equal(ts.c[i], ts.p[i].half())
        if ts.bits == 32:
            assert np.all(np.abs(h(ts.m[i]) - wm) <= E * np.abs(wm) * 1.01 + 2.0 ** -149), i
            assert np.all(np.abs(h(ts.v[i]) - wv) <= E * np.abs(wv) * 1.01 + 2.0 ** -149), i
            continue
        m32, r32 = (a.astype(np.float32).astype(np.float64) for a in (wm, np.sqrt(wv.astype(np.float32).astype(np.float64))))
        (tm, sm), (tr, sr) = ref.scaled(m32), ref.scaled(r32)
        assert np.allclose(h(ts.s[i]), np.stack([sm, sr], -1), rtol=4 * E, atol=0)
        near = (1 - 2.0 ** -22, 1.0, 1 + 2.0 ** -22)
        bits = ref.halves(ts.sizes[i], i, t, seed)
        assert np.all(np.any([h(ts.m[i]) == ref.e4m3(np.clip(tm * k, -448, 448)) for k in near], axis=0)), i
        assert np.all(np.any([h(ts.v[i]) == ref.e4m3_by(np.minimum(tr * k, 448), bits) for k in near], axis=0)), i
        if ts.sizes[i] > 1000:                              # and nearly all of them are the definition's
            assert np.mean(h(ts.m[i]) == ref.e4m3(tm)) > 0.999 and np.mean(h(ts.v[i]) == ref.e4m3_by(tr, bits)) > 0.999
    ts.check_guards()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps(bits, dtype):
    ts = Tensors(SIZES, dtype, bits, 3)
    lrs, wds = [1e-2 / (1 + i) for i in range(len(SIZES))], [0.1 * (i % 2) for i in range(len(SIZES))]
    plan = ts.plan(lrs, wds)
    for t in (1, 2, 3):
        for k, g in enumerate(ts.g):
            g.copy_(torch.from_numpy(np.random.default_rng(100 * t + k).standard_normal(g.shape) * 0.02))
        step_and_check(ts, plan, t, lrs, wds, seed=-7 * t)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes(bits):
    """Three launches, the generator's numbers of a tensor being those of its place in the whole list."""
    sizes = [1 + (37 * i * i) % 700 for i in range(120)] + [20000]
    ts = Tensors(sizes, "f16", bits, 4)
    step_and_check(ts, ts.plan(1e-3, 0.05), 5, [1e-3] * len(sizes), [0.05] * len(sizes), seed=2 ** 63 + 5)


@pytest.mark.parametrize("bits", [32, 8])
def test_factors_and_step_on_the_device(bits):
    ts = Tensors([300, 5000], "f16", bits, 5)
    plan = ts.plan(1e-2, 0.1)
    for t in (1, 2, 1000):
        step_and_check(ts, plan, t, [1e-2] * 2, [0.1] * 2, seed=9, factors=(1 / 64, 0.3), on_device=t)
    step_and_check(ts, plan, 1001, [1e-2] * 2, [0.1] * 2, seed=9, factors=(2.0, 0.0), on_device=1000)
    plan.set(lr=[0.5, 0.25], weight_decay=0.0)
    step_and_check(ts, plan, 1002, [0.5, 0.25], [0.0] * 2, seed=9)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("factor", [float("inf"), float("nan"), float("-inf")])
def test_a_factor_that_is_not_finite_changes_nothing(bits, factor):
    ts = Tensors([300, 5000], "f16", bits, 6)
    step_and_check(ts, ts.plan(), 1, [1e-2] * 2, [0.1] * 2)
    every = [t for l in (ts.p, ts.m, ts.v, ts.s or [], [c for c in ts.c if c is not None]) for t in l]
    before = [t.clone() for t in every]
    ts.g[0].fill_(float("nan"))
    dcn.dcnv4_adamw_step(ts.plan(), 2, factors_on_device=torch.tensor([factor, 1.0], device="cuda"))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(every, before))


@pytest.mark.parametrize("bits", [32, 8])
def test_zeros_and_extremes(bits):
    """Blocks of zeros, of one element, of tiny and of large gradients; beta of zero."""
    ts = Tensors([256 * 5 + 3], "f32", bits, 7)
    g = ts.g[0]
    g[:256] = 0
    g[256:512] = 0
    g[300] = 1e-3
    g[512:768] *= 1e-25                                      # squares below fp32's least
    g[768:1024] *= 1e15
    if bits == 32:
        ts.m[0].zero_()
        ts.v[0].zero_()
    plan = ts.plan(1e-3, 0.0)
    for t in (1, 2):
        step_and_check(ts, plan, t, [1e-3], [0.0], seed=1)
    step_and_check(ts, plan, 3, [1e-3], [0.0], seed=1, betas=(0.0, 0.0))
    assert bool(torch.isfinite(ts.p[0]).all())


def test_second_state_of_8_bits_follows_its_mean():
    """Rounding to the nearest would leave the root where it was for ever; by the random bits it follows the squares of the gradients."""
    n, start, later = 256 * 64, 1.0, 0.25
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), later, device="cuda")
    g[::256] = start                                        # keeps each block's scale
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    s = torch.zeros((n // 256, 2), device="cuda")
    v.copy_(torch.full((n,), 448.0, device="cuda"))
    s[:, 1] = start / 448.0
    plan = dcn.dcnv4_adamw_plan([p], [g], [m], [v], 1e-3, scales=[s])
    steps, beta = 1000, 0.999
    for t in range(1, steps + 1):
        dcn.dcnv4_adamw_step(plan, t, betas=(0.9, beta), seed=3)
    root = (v.float().view(-1, 256) * s[:, 1:]).double()[:, 1:].cpu().numpy()
    # r^2 follows v's recursion but for the rounding's variance: a step of r of at most 2^-3 of it, taken with probability (1 - beta) / 2 / 2^-3 at
    # most, adds up to (1 - beta) / 2 * 2^-3 to r^2's relative growth of a step, where v loses (1 - beta) (1 - g^2 / v): 1/16 of v at most
    want = later ** 2 + (start ** 2 - later ** 2) * beta ** steps
    assert want * 0.95 < (root ** 2).mean() < want * 1.12
    # (rounded to nearest it would still be 1)
    assert (root ** 2).mean() < 0.6


def test_captured_step_replays():
    ts, eager = Tensors([300, 5000], "f16", 8, 8), Tensors([300, 5000], "f16", 8, 8)
    count, factors = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([0.5, 1.0], device="cuda")
    plan, plain = ts.plan(), eager.plan()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        dcn.dcnv4_adamw_step(plan, 0, seed=4, step_on_device=count, factors_on_device=factors)
    for t in (1, 2, 3):
        count.fill_(t)
        for a, b in zip(ts.g, eager.g):
            a.normal_()
            b.copy_(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        dcn.dcnv4_adamw_step(plain, t, seed=4, factors_on_device=factors)
        torch.cuda.synchronize()
        for a, b in ((ts.p, eager.p), (ts.m, eager.m), (ts.v, eager.v), (ts.s, eager.s)):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b)), t


def test_on_another_stream():
    ts, plain = Tensors([70000], "f32", 32, 9), Tensors([70000], "f32", 32, 9)
    plan, other = ts.plan(), plain.plan()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for t in (1, 2, 3):
        dcn.dcnv4_adamw_step(plan, t, stream=s)
        dcn.dcnv4_adamw_step(other, t)
    torch.cuda.synchronize()
    assert torch.equal(ts.p[0], plain.p[0]) and torch.equal(ts.v[0], plain.v[0])


def test_refusals_of_the_plan():
    r = lambda n, t=torch.float32: torch.zeros(n, device="cuda", dtype=t)
    p, g, m, v = r(300), r(300), r(300), r(300)
    for bad in (([p], [g], [m], [v, v]), ([p], [g], [m], [r(299)]), ([p], [r(300, torch.float16)], [m], [p]), ([p], [p], [m], [v]), ([p, p], [g, g], [m, r(300)], [v, r(300)]),
                ([], [], [], []), ([p.cpu()], [g], [m], [v]), ([p[::2]], [g[::2]], [m[::2]], [v[::2]])):
        with pytest.raises(ValueError):
            dcn.dcnv4_adamw_plan(*bad, 1e-3)
    with pytest.raises(TypeError):
        dcn.dcnv4_adamw_plan([p], [g], [m.half()], [v], 1e-3)
    with pytest.raises(TypeError):
        dcn.dcnv4_adamw_plan([p], [g.bfloat16()], [m], [v], 1e-3)
    with pytest.raises(ValueError):
        dcn.dcnv4_adamw_plan([p], [g], [m], [v], [1e-3, 1e-3])
    with pytest.raises(ValueError):
        dcn.dcnv4_adamw_plan([p], [g], [m], [v], 1e-3, copies=[r(300, torch.float16)])
    e = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        dcn.dcnv4_adamw_plan([p], [g], [r(300, e)], [r(300, e)], 1e-3)
    with pytest.raises(ValueError):
        dcn.dcnv4_adamw_plan([p], [g], [r(300, e)], [r(300, e)], 1e-3, scales=[r((1, 2))])
    plan = dcn.dcnv4_adamw_plan([p], [g], [m], [v], 1e-3)
    for kw in ({"step": 0}, {"step": 1, "eps": 0.0}, {"step": 1, "betas": (1.0, 0.9)}, {"step": -1, "step_on_device": torch.ones(1, dtype=torch.int64, device="cuda")}):
        with pytest.raises(dcn.Dcnv4Error):
            dcn.dcnv4_adamw_step(plan, **kw)
    with pytest.raises(ValueError):
        dcn.dcnv4_adamw_step(plan, 1, factors_on_device=torch.ones(1, device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_large_tensors_and_their_parts(bits):
    """A part of a large tensor by itself gets the same bits."""
    n, part = 2 ** 24 + 100003, 2 ** 20 + 256
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = lambda size: torch.randn(n, device="cuda", generator=gen) * size
    p, g, m, v = r(0.1), r(0.02).half(), r(0.01), r(0.01) ** 2
    scales = None
    if bits == 8:
        m, v = (t.clamp(-1, 1).to(torch.float8_e4m3fn) for t in (m, v))
        scales = [torch.rand((-(-n // 256), 2), device="cuda", generator=gen) * 0.1]
        scales.append(scales[0].clone())
    # of the beginning (whose elements have the same numbers in both), and without states of 8 bits of the end
    cuts = [slice(0, part)] + ([slice(n - part - 3, n)] if bits == 32 else [])
    alone = [[t[c].clone() for t in (p, g, m, v)] for c in cuts]
    few = part // 256
    small = dcn.dcnv4_adamw_plan(*map(list, zip(*alone)), 1e-2, 0.1, scales=None if bits == 32 else [scales[1][:few].clone()])
    large = dcn.dcnv4_adamw_plan([p], [g], [m], [v], 1e-2, 0.1, scales=None if bits == 32 else [scales[0]])
    for t in (1, 2):
        dcn.dcnv4_adamw_step(large, t, seed=5)
        dcn.dcnv4_adamw_step(small, t, seed=5)
    torch.cuda.synchronize()
    for c, (ap, _, am, av) in zip(cuts, alone):
        for a, b in ((ap, p[c]), (am, m[c]), (av, v[c])):
            assert torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8))
    if bits == 8:
        assert torch.equal(small.held[4][0], scales[0][:few])
    assert bool(torch.isfinite(p).all())
