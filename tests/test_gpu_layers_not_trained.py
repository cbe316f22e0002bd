"""Gradients of layers whose own parameters get none: grad_x alone, by the bits that it has beside the others."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("P,K,F", [(37, 48, 40), (700, 136, 264)])
def test_grad_x_alone(P, K, F, dtype):
    r = lambda *s: torch.randn(s, device="cuda").to(dtype)
    x, w, b, g = r(P, K), r(2, F, K), r(2, F), r(P, F)
    want = dcn.dcnv4_gated_linear_backward(x, w, g, b)
    for kw, there in (({"need_w": False}, (1, 0, 1)), ({"need_b": False}, (1, 1, 0)), ({"need_w": False, "need_b": False}, (1, 0, 0)), ({"need_x": False, "need_w": False}, (0, 0, 1))):
        got = dcn.dcnv4_gated_linear_backward(x, w, g, b, **kw)
        assert all((a is not None) == bool(t) and (a is None or torch.equal(a, c)) for a, c, t in zip(got, want, there)), kw
    out = [torch.empty_like(x), None, None]
    assert dcn.dcnv4_gated_linear_backward(x, w, g, b, need_w=False, need_b=False, out=out)[0] is out[0] and torch.equal(out[0], want[0])
    bias = b[0].contiguous()
    want = dcn.dcnv4_linear_backward(x, w[0], g, bias)
    for args, kw, there in (((bias,), {}, (1, 0, 1)), ((), {}, (1, 0, 0)), ((bias,), {"need_x": False}, (0, 0, 1))):
        got = dcn.dcnv4_linear_backward(x, w[0], g, *args, need_w=False, **kw)
        assert all((a is not None) == bool(t) and (a is None or torch.equal(a, c)) for a, c, t in zip(got, want, there)), kw


def test_no_gradient_at_all_is_refused():
    x, w, g = (torch.randn(s, device="cuda") for s in ((5, 16), (2, 8, 16), (5, 8)))
    with pytest.raises(dcn.Dcnv4Error):
        dcn.dcnv4_gated_linear_backward(x, w, g, need_x=False, need_w=False)
    with pytest.raises(dcn.Dcnv4Error):
        dcn.dcnv4_linear_backward(x, w[0], g, need_x=False, need_w=False)
    with pytest.raises(ValueError):
        dcn.dcnv4_linear_backward(x, w[0], g, need_w=False, out=[torch.empty_like(x), torch.empty_like(w[0]), None])
