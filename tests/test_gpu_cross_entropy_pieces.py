"""The cross entropy's forward pass over pieces of the classes, whose maxima and sums are joined one after the other.  Tolerances are those of
test_gpu_cross_entropy.py; a piece adds one join, three roundings of 2^-22."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn
from test_gpu_cross_entropy import close, expected, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("P,V,piece", [(1, 700, 256), (100, 257, 256), (333, 2600, 512), (5000, 1100, 256)])
def test_pieces_that_hold_nothing_or_everything(P, V, piece, dtype):
    """The largest logit in the first piece, in the last one, in between; pieces whose classes a bias of -infinity takes out, at either end; targets
    everywhere."""
    K = 64
    dcn.dcnv4_set_option("loss_piece", piece)
    x, w, b, t, g = inputs(P, K, V, dtype, 11)
    last = (V - 1) // piece * piece                           # the last piece's first class (pieces may be shorter: then some of them)
    for gone in (slice(0, 0), slice(0, min(piece, V - 1)), slice(max(last, 1), V), slice(0, V - 1), slice(1, V)):
        for peak in (0, V // 2, V - 1):
            bias = b.clone()
            bias[peak] += 30
            bias[gone] = float("-inf")
            target = torch.where(bias[t.clamp(min=0)].isinf(), torch.full_like(t, int(bias.argmax())), t)
            want = expected(x, w, bias, target, g)
            loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, target, bias)
            pieces = V // 256 + 1
            for name, a in (("loss", loss), ("lse", lse)):
                ref, slack = want[name]
                close(name, a, (ref, slack + pieces * 3 * 2.0 ** -22), "f32")
    # every class gone: there is no distribution
    none = dcn.dcnv4_linear_cross_entropy(x, w, t.clamp(min=0), torch.full_like(b, float("-inf")))[0]
    assert none.isnan().all()


def test_pieces_the_library_makes_itself():
    """So many rows that the maxima and sums of all tiles of classes would not fit: the workspace is dirty, and a graph replays the pass."""
    P, K, V = 2 ** 17, 16, 70_001
    x, w, b, t, _ = inputs(P, K, V, "f16", 12)
    need = dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, False)
    assert need < P * V / 32 * 0.95
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    rows = list(range(0, P, 4999)) + [P - 1]

    def check(loss, lse):
        want = expected(x[rows], w, b, t[rows], torch.ones(len(rows), device="cuda"))
        for name, a in (("loss", loss), ("lse", lse)):
            ref, slack = want[name]
            close(name, a[rows], (ref, slack + (V // 64 // 16 + 16 + 4) * 3 * 2.0 ** -22), "f32")

    check(*dcn.dcnv4_linear_cross_entropy(x, w, t, b, workspace=work))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = dcn.dcnv4_linear_cross_entropy(x, w, t, b, workspace=work)
    for k in range(2):
        torch.cuda.synchronize()
        t.random_(0, V)
        work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(*outs)
        assert all(torch.equal(a, c) for a, c in zip(outs, dcn.dcnv4_linear_cross_entropy(x, w, t, b)))
