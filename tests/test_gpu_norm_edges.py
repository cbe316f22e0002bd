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
