"""A training step as it would be put together: norm, gated layer, projection down, the block's end, classifier and loss, back through all of them, and AdamW
over every parameter; against the same step by torch's autograd in double precision on the CPU, and captured as a graph.

In half precision the parameters are float32, and the step leaves float16 copies for the next forward pass; gradients come with a loss scale that the
step takes out again."""
import numpy as np
import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

N, H, W, C, F, V, EPS = 3, 6, 7, 64, 96, 37, 1e-5
SHAPES = {"norm_g": (C,), "norm_b": (C,), "w": (2, F, C), "b": (2, F), "down_w": (C, F), "down_b": (C,), "scale": (C,), "first_g": (C,), "first_b": (C,),
          "second_g": (C,), "second_b": (C,), "head_w": (V, C), "head_b": (V,)}
LR, DECAY, BETAS = 1e-2, {k: 0.1 if len(s) > 1 else 0.0 for k, s in SHAPES.items()}, (0.9, 0.999)


def start(seed=0):
    rng = np.random.default_rng(seed)
    p = {k: rng.standard_normal(s) * (0.2 if len(s) == 1 else 1.0 / np.sqrt(s[-1])) + (1.0 if k.endswith("_g") or k == "scale" else 0.0)
         for k, s in SHAPES.items()}
    x = rng.standard_normal((N, H, W, C))
    gate = np.array([1 / 0.9, 0.0, 1 / 0.9], dtype=np.float32)
    return p, x, gate, rng.integers(0, V, (N, H, W))


class Net:
    """Parameters, gradients and states on the GPU, and the step over them."""

    def __init__(self, dtype, bits, seed=0):
        p, x, gate, target = start(seed)
        self.dt = torch.float16 if dtype == "f16" else torch.float32
        cuda = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)
        self.x, self.gate, self.target = cuda(x, self.dt), cuda(gate, torch.float32), cuda(target, torch.int64)
        self.up = 256.0 if dtype == "f16" else 1.0
        self.master = {k: cuda(v, torch.float32) for k, v in p.items()}
        # (what the forward pass reads, and what the first step starts from, are the same numbers)
        self.p = {k: v.to(self.dt) for k, v in self.master.items()}
        if dtype == "f16":
            for k, v in self.p.items():
                self.master[k].copy_(v)
        else:
            self.p = self.master
        self.grads = {k: torch.zeros_like(v) for k, v in self.p.items()}
        state = torch.float32 if bits == 32 else torch.float8_e4m3fn
        self.m, self.v = ([torch.zeros(s, device="cuda").to(state) for s in SHAPES.values()] for _ in range(2))
        scales = None if bits == 32 else [torch.zeros((-(-int(np.prod(s)) // 256), 2), device="cuda") for s in SHAPES.values()]
        self.scales = scales or []
        self.plan = dcn.dcnv4_adamw_plan(list(self.master.values()), list(self.grads.values()), self.m, self.v, LR, [DECAY[k] for k in SHAPES],
                                         scales=scales, copies=list(self.p.values()) if dtype == "f16" else None)
        self.factors = torch.tensor([1 / self.up, 1.0], device="cuda")
        self.grad_loss = torch.full((N, H, W), self.up / (N * H * W), device="cuda")

    def step(self, t, on_device=None, work=None):
        """(loss, gradient of x); gradients go where the plan reads them."""
        p, g, w = self.p, self.grads, work or {}
        y0, mean, rstd = dcn.dcnv4_layer_norm(self.x, p["norm_g"], p["norm_b"], eps=EPS, stats=True)
        h = dcn.dcnv4_gated_linear(y0, p["w"], p["b"], workspace=w.get("gated"))
        branch = dcn.dcnv4_linear(h, p["down_w"], p["down_b"])
        first, second = (p["first_g"], p["first_b"]), (p["second_g"], p["second_b"])
        z, y, *stats = dcn.dcnv4_norm_scale_add_norm(branch, self.x, p["scale"], self.gate, first, second, eps=EPS)
        loss, lse = dcn.dcnv4_linear_cross_entropy(y, p["head_w"], self.target, p["head_b"], workspace=w.get("loss"))
        gy = torch.empty_like(y)
        dcn.dcnv4_linear_cross_entropy_backward(y, p["head_w"], self.target, lse, self.grad_loss, p["head_b"], workspace=w.get("loss_back"),
                                                out=[gy, g["head_w"], g["head_b"]])
        gbranch, gx = torch.empty_like(branch), torch.empty_like(branch)
        dcn.dcnv4_norm_scale_add_norm_backward(branch, z, p["scale"], self.gate, first, second, stats, gy, grad_gate=False, workspace=w.get("end"),
                                               out=[gbranch, gx, g["scale"], None, g["first_g"], g["first_b"], g["second_g"], g["second_b"]])
        gh = torch.empty_like(h)
        dcn.dcnv4_linear_backward(h, p["down_w"], gbranch, p["down_b"], workspace=w.get("down"), out=[gh, g["down_w"], g["down_b"]])
        gy0 = torch.empty_like(y0)
        dcn.dcnv4_gated_linear_backward(y0, p["w"], gh, p["b"], workspace=w.get("gated"), out=[gy0, g["w"], g["b"]])
        gin = torch.empty_like(y0)
        dcn.dcnv4_layer_norm_backward(self.x, p["norm_g"], mean, rstd, gy0, workspace=w.get("norm"), out=[gin, g["norm_g"], g["norm_b"]])
        dcn.dcnv4_adamw_step(self.plan, t, betas=BETAS, seed=7, step_on_device=on_device, factors_on_device=self.factors)
        return loss, gx.float() + gin.float()

    def workspaces(self):
        P, code = N * H * W, dcn._dtype_code(self.x)
        size = {"gated": dcn.dcnv4_gated_linear_workspace_bytes(P, C, F, code, True), "loss": dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, C, V, code, False),
                "loss_back": dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, C, V, code, True), "end": dcn.dcnv4_norm_scale_add_norm_workspace_bytes(P, C, N),
                "down": dcn.dcnv4_linear_backward_workspace_bytes(P, F, C, code), "norm": dcn.dcnv4_layer_norm_workspace_bytes(P, C)}
        return {k: torch.empty(v, dtype=torch.uint8, device="cuda") for k, v in size.items()}


class Plain:
    """The same by torch's autograd in double precision, from the numbers that the net starts from."""

    def __init__(self, net):
        self.net = net
        self.master = {k: v.double().cpu() for k, v in net.master.items()}
        self.m = {k: torch.zeros(s, dtype=torch.float64) for k, s in SHAPES.items()}
        self.v = {k: torch.zeros(s, dtype=torch.float64) for k, s in SHAPES.items()}

    def step(self, t):
        leaf = lambda a: a.detach().clone().requires_grad_(True)
        p = {k: leaf(v) for k, v in self.master.items()}
        x, gate = leaf(self.net.x.double().cpu()), self.net.gate.double().cpu()
        norm = lambda v, g, b: torch.nn.functional.layer_norm(v, (C,), g, b, EPS)
        y0 = norm(x, p["norm_g"], p["norm_b"])
        a, u = y0 @ p["w"][0].T + p["b"][0], y0 @ p["w"][1].T + p["b"][1]
        branch = (torch.nn.functional.silu(a) * u) @ p["down_w"].T + p["down_b"]
        z = x + gate.view(-1, 1, 1, 1) * p["scale"] * norm(branch, p["first_g"], p["first_b"])
        y = norm(z, p["second_g"], p["second_b"])
        loss = torch.nn.functional.cross_entropy((y @ p["head_w"].T + p["head_b"]).reshape(-1, V), self.net.target.cpu().reshape(-1), reduction="none")
        loss.mean().backward()
        with torch.no_grad():
            for k, v in self.master.items():
                g = p[k].grad
                self.m[k] = BETAS[0] * self.m[k] + (1 - BETAS[0]) * g
                self.v[k] = BETAS[1] * self.v[k] + (1 - BETAS[1]) * g * g
                v.mul_(1 - LR * DECAY[k]).sub_(LR / (1 - BETAS[0] ** t) * self.m[k] / ((self.v[k] / (1 - BETAS[1] ** t)).sqrt() + 1e-8))
        return loss.detach().reshape(N, H, W), x.grad, {k: v.grad for k, v in p.items()}


def off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_step_against_autograd(dtype):
    """Relative 2-norms.  fp16: up to eight tensors follow one another on the way to a gradient (y0, h, branch, z, y, d of the loss, and three gradients),
    each rounded to half a step, and norms whose slopes are about 1 pass that on, as do projections of unit rows: 12 half steps; fp32: as many, and sums of
    some hundred terms in between, 8 times that.  The first step of AdamW moves by lr * g / (|g| + eps) whatever the gradient's size is, so that where a gradient is
    near zero its sign is uncertain: parameters are held against AdamW of the framework's own gradients."""
    net = Net(dtype, 32)
    before = {k: v.double().cpu() for k, v in net.master.items()}
    plain = Plain(net)
    loss, gx = net.step(1)
    wloss, wgx, wgrads = plain.step(1)
    tol = 12 * (2.0 ** -11 if dtype == "f16" else 8 * 2.0 ** -24)
    assert off(loss.reshape(N, H, W), wloss) <= tol and off(gx / net.up, wgx) <= tol
    for k, want in wgrads.items():
        assert off(net.grads[k].float() / net.up, want) <= tol, (k, off(net.grads[k].float() / net.up, want))
    for k, b in before.items():
        g = net.grads[k].double().cpu() / net.up
        want = b * (1 - LR * DECAY[k]) - LR * g / (g.abs() + 1e-8)
        assert off(net.master[k], want) <= 4 * 2.0 ** -24, k
        if dtype == "f16":
            assert torch.equal(net.p[k], net.master[k].half())


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_follow_one_another_and_replay_from_a_graph(bits):
    """Several steps eagerly, and the same ones as replays of one graph whose step number is on the device: the same bits, parameters and states."""
    eager, caught = Net("f16", bits), Net("f16", bits)
    work, count = caught.workspaces(), torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        outs = caught.step(0, on_device=count, work=work)
    losses = []
    for t in (1, 2, 3, 4):
        count.fill_(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = eager.step(t)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), t
        for k in SHAPES:
            assert torch.equal(eager.master[k], caught.master[k]) and torch.equal(eager.grads[k], caught.grads[k]), (t, k)
        for a, b in zip(eager.m + eager.v + eager.scales, caught.m + caught.v + caught.scales):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), t
        losses.append(float(want[0].mean()))
    assert all(np.isfinite(losses))
