"""Norms of rows at the ends of the range."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [3, 8, 72, 128, 321, 520, 1030, 1100, 2056, 2100, 4104, 6000, 9000, 16376])
def test_gradient_of_large_constant_rows(C):
    """A constant row: xhat = 0, whatever its size, so grad_x = rstd * (g - avg(g)).  What a lane has beyond the row's end counts for nothing,
    also where mean * rstd is more than fp32 holds."""
    P = 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(C)
    x = torch.full((P, C), 2.0 ** 115, device="cuda")           # (exact sums of up to 2^14 of them; 2^115 / sqrt(eps) overflows)
    gamma = torch.rand(C, generator=gen, device="cuda") + 0.5
    gy = torch.randn((P, C), generator=gen, device="cuda")
    eps = 2.0 ** -40
    y, mean, rstd = dcn.dcnv4_layer_norm(x, gamma, None, eps=eps, stats=True)
    if C & (C - 1) == 0:
        assert not y.any()
    mean, rstd = x[:, 0].contiguous(), torch.full((P,), 2.0 ** 20, device="cuda")
    g = gy.double() * gamma.double()
    want = 2.0 ** 20 * (g - g.mean(-1, keepdim=True))
    # 64 roundings of fp32 of what the terms add up from
    lim = 64 * 2.0 ** -24 * 2.0 ** 20 * (g.abs() + g.abs().mean(-1, keepdim=True))
    got = dcn.dcnv4_layer_norm_backward(x, gamma, mean, rstd, gy)
    assert ((got[0].double() - want).abs() <= lim).all()
    assert not got[1].any() and got[2].isfinite().all()
    branch = dcn.dcnv4_dropout_add_layer_norm_backward(x, gamma, mean, rstd, gy, 0.0, 1)
    assert torch.equal(branch[0], got[0]) and torch.equal(branch[1], got[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("P,C", [(1, 5), (700, 72), (90, 1030)])
def test_gradient_of_a_norm_with_beta_alone(P, C, dtype):
    """beta has its gradient without gamma, which then is a gamma of ones: the same numbers, bit for bit."""
    x, res, gy, gz = (torch.randn((P, C), device="cuda").to(dtype) for _ in range(4))
    beta, ones = torch.randn(C, device="cuda").to(dtype), torch.ones(C, device="cuda", dtype=dtype)
    y, mean, rstd = dcn.dcnv4_layer_norm(x, None, beta, stats=True)
    got = dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy, beta=beta)
    want = dcn.dcnv4_layer_norm_backward(x, ones, mean, rstd, gy)
    assert torch.equal(got[0], want[0]) and got[1] is None and torch.equal(got[2], want[2])
    assert dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy)[1:] == (None, None)
    z, _, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(x, res, None, beta, 0.3, 7)
    got = dcn.dcnv4_dropout_add_layer_norm_backward(z, None, mean, rstd, gy, 0.3, 7, grad_z=gz, beta=beta)
    want = dcn.dcnv4_dropout_add_layer_norm_backward(z, ones, mean, rstd, gy, 0.3, 7, grad_z=gz)
    assert got[2] is None and all(torch.equal(got[i], want[i]) for i in (0, 1, 3))
    work = torch.empty(dcn.dcnv4_layer_norm_workspace_bytes(P, C), dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(x), None, torch.empty_like(beta))
    again = dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy, beta=beta, workspace=work, out=out)
    assert again[2] is out[2]
    with pytest.raises(ValueError):
        dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy, beta=beta, out=out, prepare_only=True)
    with pytest.raises(ValueError):
        dcn.dcnv4_layer_norm_backward(x, None, mean, rstd, gy, beta=beta[:-1])
