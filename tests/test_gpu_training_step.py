"""A training step as it would be put together: module, branch end, classifier and loss forward, and back through the loss, the branch end
and the operator; against the same step out of plain double-precision forms, and captured as a graph."""
import numpy as np
import pytest
import torch

import oracle
import training_ref as ref
from paper_2401_06197_amd import binding as dcn
from paper_2401_06197_amd.synth import Config, make_inputs, make_module_params

pytestmark = pytest.mark.gpu

CFG = Config("step", N=2, H=9, W=11, C=64, G=4)
V, P_DROP, SEED, EPS = 37, 0.2, 5, 1e-5


def parts(dtype):
    inp = make_inputs(CFG, dtype, seed=4)
    prm = make_module_params(CFG, dtype, seed=4)
    rng = np.random.default_rng(4)
    dt = inp["x"].dtype
    more = {"gamma": (1 + 0.2 * rng.standard_normal(CFG.C)).astype(dt), "beta": (0.2 * rng.standard_normal(CFG.C)).astype(dt),
            "w": (rng.standard_normal((V, CFG.C)) / 4).astype(dt), "b": (0.1 * rng.standard_normal(V)).astype(dt)}
    target = rng.integers(0, V, (CFG.N, CFG.H, CFG.W))
    target[0, :2] = -100
    return inp, prm, more, target


def step(d, module, offset, on_device=None, work=None):
    """(loss, gradients of the branch, the residual, the norm's and the classifier's parameters)."""
    work = work or {}
    branch = dcn.dcnv4_module_forward(d["x"], module["w_om_padded"], module["b_om_padded"], CFG.G, w_in=module["w_in"], b_in=module["b_in"],
                                      w_out=module["w_out"], b_out=module["b_out"], workspace=work.get("module"))
    z, y, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(branch, d["x"], d["gamma"], d["beta"], P_DROP, SEED, offset, offset_on_device=on_device,
                                                        eps=EPS)
    loss, lse = dcn.dcnv4_linear_cross_entropy(y, d["w"], d["target"], d["b"], workspace=work.get("loss"))
    gy, gw, gb = dcn.dcnv4_linear_cross_entropy_backward(y, d["w"], d["target"], lse, d["g"], d["b"], workspace=work.get("grad"))
    back = dcn.dcnv4_dropout_add_layer_norm_backward(z, d["gamma"], mean, rstd, gy, P_DROP, SEED, offset, offset_on_device=on_device,
                                                     workspace=work.get("norm"))
    gop = dcn.dcnv4_backward(d["x"], d["offset"], d["mask"], back[0])
    return (branch, loss, gw, gb, *back, *gop)


def on_gpu(dtype):
    inp, prm, more, target = parts(dtype)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    d = {k: cuda(v) for k, v in {**inp, **more, "target": target}.items()}
    d["g"] = torch.full(target.shape, (256.0 if dtype == "f16" else 1.0) / int((target >= 0).sum()), device="cuda")
    return d, {k: cuda(v) for k, v in prm.items()}, inp, more, target


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_step_against_plain_forms(dtype):
    d, module, inp, more, target = on_gpu(dtype)
    branch, loss, gw, gb, gx, gr, gg, gbeta, *gop = step(d, module, 3)
    f64 = lambda a: a.astype(np.float64)
    # from the module's output on (whose own tests hold it against the oracle)
    z = ref.dropout(branch.cpu().numpy(), P_DROP, SEED, 3, residual=inp["x"])
    y, mean, rstd = ref.layer_norm(z, more["gamma"], more["beta"], EPS)
    w, b, g = f64(more["w"]), f64(more["b"]), d["g"].double().cpu().numpy()
    logits = y @ w.T + b
    lse = np.log(np.exp(logits).sum(-1))
    ok = target >= 0
    hot = np.zeros(logits.shape)
    np.put_along_axis(hot, np.where(ok, target, 0)[..., None], 1.0, -1)
    hot *= ok[..., None]
    wloss = np.where(ok, lse - (logits * hot).sum(-1), 0)
    delta = (np.exp(logits - lse[..., None]) - hot) * (g * ok)[..., None]
    (gz, wgg, wgbeta), _ = ref.layer_norm_backward(z, more["gamma"], mean, rstd, delta @ w)
    gone = ref.dropped(z.size, P_DROP, SEED, 3).reshape(z.shape)
    wgx = np.where(gone, 0, gz / (1 - ref.limit(P_DROP) / 65536))
    want = {"loss": wloss, "grad_w": np.einsum("nhwv,nhwc->vc", delta, y), "grad_b": delta.sum((0, 1, 2)), "grad_x": wgx, "grad_residual": gz,
            "grad_gamma": wgg, "grad_beta": wgbeta}
    got = {"loss": loss, "grad_w": gw, "grad_b": gb, "grad_x": gx, "grad_residual": gr, "grad_gamma": gg, "grad_beta": gbeta}
    # relative 2-norms: a chain of four roundings of the type in turn (z, y, d, the gradient of y) and its last, each at most one
    # half step relative to the values, which the norm's slope of about 1 and the loss's Lipschitz constant of 1 pass on: ten half steps
    for name, t in want.items():
        err = np.linalg.norm(got[name].double().cpu().numpy() - t) / np.linalg.norm(t)
        assert err <= 10 * (2.0 ** -11 if dtype == "f16" else 2.0 ** -24 * 8), (name, err)
    # and the operator's gradients of what arrives there
    rg = oracle.backward(inp["x"], inp["offset"], inp["mask"], gx.cpu().numpy())
    for a, r in zip(gop, rg):
        tol = 2e-2 if dtype == "f16" else 1e-5
        assert np.all(np.abs(a.cpu().numpy() - r) <= tol + tol * np.abs(r))


def test_step_replays_from_a_graph():
    d, module, *_ = on_gpu("f16")
    n = CFG.N * CFG.H * CFG.W
    size = {"module": dcn.dcnv4_module_workspace_bytes(CFG.N, CFG.H, CFG.W, CFG.G, CFG.Cg, dcn.DCNV4_F16, False),
            "loss": dcn.dcnv4_linear_cross_entropy_workspace_bytes(n, CFG.C, V, dcn.DCNV4_F16, False),
            "grad": dcn.dcnv4_linear_cross_entropy_workspace_bytes(n, CFG.C, V, dcn.DCNV4_F16, True),
            "norm": dcn.dcnv4_layer_norm_workspace_bytes(n, CFG.C)}
    work = {k: torch.empty(v, dtype=torch.uint8, device="cuda") for k, v in size.items()}
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(d, module, 0, count, work)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step(d, module, 0, count, work)
    for k in range(3):
        torch.cuda.synchronize()
        d["x"].normal_()
        count.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        want = step(d, module, k)
        torch.cuda.synchronize()
        # (the last three are the operator's, whose grad_x is summed with atomics)
        assert all(torch.equal(a, b) for a, b in zip(got[:8], want[:8])), k
        assert torch.allclose(got[8].float(), want[8].float(), rtol=2e-2, atol=2e-2)
