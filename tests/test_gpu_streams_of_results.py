"""Calls on a stream that is handed over, whose results are new tensors: they take no memory that the current stream still reads, and give none
back to it that the call still writes."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn
from paper_2401_06197_amd.synth import Config, make_inputs, make_module_params

pytestmark = pytest.mark.gpu

P, C, V = 1500, 264, 120


def calls():
    r = lambda *s: torch.randn(s, device="cuda")
    x, res, gy, gamma, beta = r(P, C), r(P, C), r(P, C), r(C), r(C)
    _, mean, rstd = dcn.dcnv4_layer_norm(x, gamma, beta, stats=True)
    w, b, t, g = r(V, C) / 8, r(V), torch.randint(0, V, (P,), device="cuda"), r(P)
    lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)[1]
    return {
        "norm": lambda **kw: dcn.dcnv4_layer_norm(x, gamma, beta, **kw),
        "norm with statistics": lambda **kw: dcn.dcnv4_layer_norm(x, gamma, beta, stats=True, **kw),
        "norm's gradient": lambda **kw: dcn.dcnv4_layer_norm_backward(x, gamma, mean, rstd, gy, **kw),
        "dropout": lambda **kw: dcn.dcnv4_dropout(x, 0.3, 5, **kw),
        "dropout's gradient": lambda **kw: dcn.dcnv4_dropout_backward(gy, 0.3, 5, **kw),
        "branch end": lambda **kw: dcn.dcnv4_dropout_add_layer_norm(x, res, gamma, beta, 0.3, 5, **kw),
        "branch end's gradient": lambda **kw: dcn.dcnv4_dropout_add_layer_norm_backward(x, gamma, mean, rstd, gy, 0.3, 5, **kw),
        "cross entropy": lambda **kw: dcn.dcnv4_linear_cross_entropy(x, w, t, b, **kw),
        "cross entropy's gradient": lambda **kw: dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b, **kw),
    }


def tensors(r):
    return [r] if isinstance(r, torch.Tensor) else [t for t in r if t is not None]


def check(call, same=torch.equal):
    want = tensors(call())
    m = torch.randn((4096, 4096), device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    tensors(call(stream=s))                                   # (what a first call loads and allocates is there)
    old = [torch.full_like(o, 3.0) for o in want]
    torch.cuda.synchronize()
    # the current stream has other work first, and then reads tensors of the results' sizes that have been given back
    for _ in range(4):
        m @ m
    copies = [o.clone() for o in old]
    del old
    got = tensors(call(stream=s))
    torch.cuda.synchronize()
    assert all(bool((c == 3.0).all()) for c in copies)
    assert all(same(a, b) for a, b in zip(got, want))
    # the other stream has work first: what the current one makes where dropped results lay stays as it is
    with torch.cuda.stream(s):
        for _ in range(4):
            m @ m
    del got
    call(stream=s)
    new = [torch.full_like(o, 7.0) for o in want]
    torch.cuda.synchronize()
    assert all(bool((o == 7.0).all()) for o in new)


@pytest.mark.parametrize("name", ["norm", "norm with statistics", "norm's gradient", "dropout", "dropout's gradient", "branch end",
                                  "branch end's gradient", "cross entropy", "cross entropy's gradient"])
def test_results_are_of_the_stream_of_the_call(name):
    check(calls()[name])


OLDER = ("forward", "backward", "softmax", "softmax's backward", "merged", "merged backward", "linear", "depthwise", "module")


def older_calls():
    cfg = Config("streams", N=2, H=28, W=28, C=128, G=8)
    d = {k: torch.from_numpy(v).cuda() for k, v in make_inputs(cfg, "f32", seed=3).items()}
    m = {k: torch.from_numpy(v).cuda() for k, v in make_module_params(cfg, "f32", seed=3).items()}
    om = torch.zeros((cfg.N, cfg.H, cfg.W, cfg.G, 32), device="cuda")
    om[..., :18], om[..., 18:27] = d["offset"].flatten(-2), d["mask"]
    taps = torch.randn((3, 3, cfg.C), device="cuda")
    ops = (d["x"], d["offset"], d["mask"])
    return dict(zip(OLDER, (
        lambda **kw: dcn.dcnv4_forward(*ops, **kw), lambda **kw: dcn.dcnv4_backward(*ops, d["grad_y"], **kw),
        lambda **kw: dcn.dcnv4_forward_softmax(*ops, **kw), lambda **kw: dcn.dcnv4_backward_softmax(*ops, d["grad_y"], **kw),
        lambda **kw: dcn.dcnv4_forward_merged(d["x"], om, **kw), lambda **kw: dcn.dcnv4_backward_merged(d["x"], om, d["grad_y"], **kw),
        lambda **kw: dcn.dcnv4_linear(d["x"], m["w_in"], m["b_in"], **kw), lambda **kw: dcn.dcnv4_depthwise3x3(d["x"], taps, **kw),
        lambda **kw: dcn.dcnv4_module_forward(d["x"], m["w_om_padded"], m["b_om_padded"], cfg.G, w_in=m["w_in"], b_in=m["b_in"],
                                              w_out=m["w_out"], b_out=m["b_out"], **kw))))


@pytest.mark.parametrize("name", OLDER)
def test_results_of_the_operator_and_the_module(name):
    # (grad_x is summed with atomics, in an order that changes: fp32 sums of some tens of terms)
    check(older_calls()[name], lambda a, b: torch.allclose(a, b, rtol=1e-4, atol=1e-4))
