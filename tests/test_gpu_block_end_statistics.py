"""The block's end without statistics, and its gradient, which takes them: a norm's missing ones are refused by name, before any launch."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["f", "s", "fs", ""])
def test_a_gradient_without_the_norms_statistics_is_refused(form):
    r = lambda *s: torch.randn(s, device="cuda")
    x, res, gz, gy, pair = r(2, 5, 24), r(2, 5, 24), r(2, 5, 24), r(2, 5, 24), (r(24), r(24))
    first, second = (pair if "f" in form else None), (pair if "s" in form else None)
    z, _, *none = dcn.dcnv4_norm_scale_add_norm(x, res, None, None, first, second, stats=False)
    assert none == [None] * 4
    stats = dcn.dcnv4_norm_scale_add_norm(x, res, None, None, first, second)[2:]
    back = lambda s: dcn.dcnv4_norm_scale_add_norm_backward(x, z, None, None, first, second, s, gy if second else None, gz)
    want = back(stats)
    if not form:
        assert torch.equal(back(none)[0], want[0])
        return
    for name in [n for n, there in (("mean1", "f"), ("rstd1", "f"), ("mean2", "s"), ("rstd2", "s")) if there in form]:
        at = ("mean1", "rstd1", "mean2", "rstd2").index(name)
        with pytest.raises(ValueError, match=name):
            back([None if i == at else t for i, t in enumerate(stats)])
    with pytest.raises(ValueError, match="mean"):
        back(none)
    with pytest.raises(ValueError, match="stats"):
        back(None)
    with pytest.raises(ValueError, match="stats"):
        back(stats[:2])
