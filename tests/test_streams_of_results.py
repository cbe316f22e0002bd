"""What a call makes by itself is made on the stream that it is handed (no GPU needed: the stream is a mark, the allocations are the host's)."""
import contextlib

import pytest
import torch

from paper_2401_06197_amd import binding as dcn


@pytest.fixture
def made(monkeypatch):
    """The stream that is current, as torch.cuda.stream sets it, at each new tensor."""
    now, at = [None], []

    @contextlib.contextmanager
    def stream(s):
        now[0], before = s, now[0]
        yield
        now[0] = before

    def noted(f):
        def g(*a, **kw):
            at.append(now[0])
            return f(*a, **kw)
        return g

    monkeypatch.setattr(torch.cuda, "stream", stream)
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "new_empty", noted(torch.Tensor.new_empty))
    return at


@pytest.mark.parametrize("stream", [None, "side"])
def test_results_and_workspaces(made, stream):
    x, f32 = torch.zeros((3, 8)), torch.float32
    y, none, stat, half = dcn._outputs(x, None, (("y", x.shape, f32), None, ("mean", (3,), f32), ("grad_w", (5, 8), torch.float16)), stream)
    assert y.shape == (3, 8) and none is None and stat.shape == (3,) and half.dtype is torch.float16
    dcn._new_like(x, stream)
    dcn._workspace(x, None, 100, stream)
    assert made == [stream] * 5
    # those that are handed over stay what they are
    out = [torch.zeros((3, 8))]
    del made[:]
    assert dcn._outputs(x, out, (("y", x.shape, f32),), stream)[0] is out[0] and not made


@pytest.mark.parametrize("stream", [None, "side"])
def test_results_of_the_operator_and_the_module(made, stream):
    x, offset = torch.zeros((1, 2, 2, 4)), torch.zeros((1, 2, 2, 1, 9, 2))
    assert dcn._uninitialised(x, (1, 3, 3, 4), stream).shape == (1, 3, 3, 4)
    assert dcn._uninitialised(torch.nn.Parameter(x), (2, 2), stream).shape == (2, 2)
    a, b = dcn._empty_like(stream, x, offset)
    assert a.shape == x.shape and b.shape == offset.shape
    assert made == [stream] * 4
