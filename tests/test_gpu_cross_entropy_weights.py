"""Gradients of the cross entropy where grad_loss differs from row to row by many powers of two (class weights, focal losses, an
outlier), in fp16: classes that only rows of small weight reach.

Two groups of rows and classes: a row's first feature and a class's first weight set the logits of the other group 80 lower, so that
its probabilities, e^-80, are far below anything that counts.  The rows of the second group have a weight `ratio` times as large.

Tolerances, before the rounding of the result.  d = softmax - onehot: p times the error of logit - lse, one rounding of fp16, 2^-11 of it,
and half of the least step, 2^-25, of 2^15 * d.  x in grad_w's product, times its row's part of the largest grad_loss and a power of two that
leaves this between 2^-8 and 1 (for rows of at least 2^-32 of the largest): one more rounding, 2^-11, and half of fp16's
least step, 2^-25, over 2^-8.  Sums: (n / 8 + 80) * 2^-23 of the sum of magnitudes and 2^-21 of it, n the length of the sum.  All of it per row, with that row's own grad_loss."""
import pytest
import torch

from paper_2401_06197_amd import binding as dcn
from test_gpu_cross_entropy import IGNORE, close

pytestmark = pytest.mark.gpu

E = 2.0 ** -23
X_OFF = 2.0 ** -17


def inputs(P, K, V, ratio, seed=0, features=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + P + K + V)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    second, other = torch.arange(P, device="cuda") % 2 == 1, torch.arange(V, device="cuda") % 2 == 1
    x, w = r(P, K) * features, r(V, K) * (0.5 / K ** 0.5 / features)
    x[:, 0] = torch.where(second, -1.0, 1.0)
    w[:, 0] = torch.where(other, -40.0, 40.0)
    t = torch.randint(0, V // 2, (P,), generator=gen, device="cuda") * 2 + second.long()
    t[4::9] = IGNORE
    g = (0.5 + torch.rand(P, generator=gen, device="cuda")) * 65536.0
    g = torch.where(second, g * ratio, g)
    return x.half(), w.half(), (0.3 * r(V)).half(), t, g


def expected(x, w, b, t, g):
    K, V, P = w.shape[1], w.shape[0], x.shape[0]
    X, W, B = x.double(), w.double(), b.double()
    logits, size = X @ W.T + B, X.abs() @ W.abs().T + B.abs()
    off = (K / 8 + 8) * E * size
    lse = torch.logsumexp(logits, -1)
    lse_off = off.max(-1).values + 128 * E + 2 * E * lse.abs()
    ok = t != IGNORE
    p = (logits - lse[:, None]).exp()
    d = p.clone()
    d.scatter_add_(1, torch.where(ok, t, 0)[:, None], -torch.ones_like(lse)[:, None])
    d = d * ok[:, None]
    d_off = (p * (off + lse_off[:, None] + 4 * E * (1 + logits.abs())) + 2.0 ** -11 * d.abs() + 2.0 ** -40) * ok[:, None]
    G = g.double()[:, None] * ok[:, None]
    gd, gd_off = G * d, G.abs() * d_off
    more = lambda n: (n / 8 + 80) * E + 2.0 ** -21
    return {"grad_x": (gd @ W, gd_off @ W.abs() + more(V) * (gd.abs() @ W.abs())),
            "grad_w": (gd.T @ X, gd_off.T @ X.abs() + gd.abs().T @ (2.0 ** -11 * X.abs() + X_OFF) + more(P) * (gd.abs().T @ X.abs())),
            "grad_b": (gd.sum(0), gd_off.sum(0) + more(P) * gd.abs().sum(0))}


def check(P, K, V, ratio, seed=0, features=1.0):
    x, w, b, t, g = inputs(P, K, V, ratio, seed, features)
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, t, b)
    got = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    for (name, want), a in zip(expected(x, w, b, t, g).items(), got):
        close(f"{name}, ratio {ratio}", a, want, "f16")
    again = dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    assert all(torch.equal(a, c) for a, c in zip(got, again))
    return (x, w, b, t, g), (lse, *got)


@pytest.mark.parametrize("ratio", [1.0, 2.0 ** -7, 2.0 ** -8, 1e-3, 1e-5, 1e-6, 1e-7, 1e-8])
@pytest.mark.parametrize("P,K,V", [(300, 64, 40), (1500, 96, 150)])
def test_rows_of_small_weight_keep_their_classes(P, K, V, ratio):
    check(P, K, V, ratio)


@pytest.mark.parametrize("ratio", [1e-3, 1e-6])
def test_small_features(ratio):
    """Features of 2^-6: what a weight takes from their bits is counted absolutely."""
    check(1200, 64, 60, ratio, features=2.0 ** -6)


@pytest.mark.parametrize("tile", [1, 2, 3])
@pytest.mark.parametrize("splits,piece", [(1, 0), (3, 256), (8, 0)])
def test_every_tile_split_and_piece(tile, splits, piece):
    dcn.dcnv4_set_option("loss_tile", tile)
    dcn.dcnv4_set_option("loss_splits", splits)
    dcn.dcnv4_set_option("loss_piece", piece)
    check(900, 80, 600, 1e-5, seed=tile)


def test_many_weights_in_one_call():
    """Rows over thirty powers of two, neighbours among them far apart: each class is reached by rows of one weight alone."""
    P, K, V, steps = 620, 64, 31, 31
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x, w = torch.randn((P, K), generator=gen, device="cuda"), torch.zeros((V, K), device="cuda")
    t = torch.arange(P, device="cuda") * 7 % V
    # logits of 64 for the row's own class, 0 for the others: d = -1 / (1 + e^64 / 30) where it is the target's, and as small elsewhere;
    # a target beside it (the next class) has d = -1 there and +1 at its own
    x[:, :V] = torch.nn.functional.one_hot(t, V).float()
    w[:, :V] = 64 * torch.eye(V, device="cuda")
    g = 2.0 ** (10 - (t % steps).float())
    x, w = x.half(), w.half()
    target = torch.where(torch.arange(P, device="cuda") < P // 2, t, (t + 1) % V)
    b = torch.zeros(V, device="cuda").half()
    loss, lse = dcn.dcnv4_linear_cross_entropy(x, w, target, b)
    got = dcn.dcnv4_linear_cross_entropy_backward(x, w, target, lse, g, b)
    for (name, want), a in zip(expected(x, w, b, target, g).items(), got):
        close(name, a, want, "f16")


def test_weights_that_are_zero_tiny_or_infinite():
    (x, w, b, t, g), (lse, *want) = check(700, 64, 50, 1.0, seed=5)
    back = lambda g: dcn.dcnv4_linear_cross_entropy_backward(x, w, t, lse, g, b)
    # a row without a finite weight: its own gradient, and those of what it reaches; the others' as where it has none
    row = int((t != IGNORE).nonzero()[3])
    none, inf = g.clone(), g.clone()
    none[row], inf[row] = 0.0, float("inf")
    a, c = back(none), back(inf)
    keep = torch.arange(700, device="cuda") != row
    assert torch.equal(a[0][keep], c[0][keep]) and not a[0][row].any()
    assert not c[0][row].isfinite().all() and not c[1].isfinite().all()
    # every weight below fp32's normal numbers: gradients that fp16 does not hold, and no NaN
    assert not any(o.any() for o in back(torch.full_like(g, 1e-40)))
    # signs: the gradient is odd in the weights, exactly where vector instructions add it up (the matrix unit cuts off sums of either sign
    # towards the same side)
    got = back(-g)
    assert torch.equal(got[2], -want[2])
    for (name, ref), a in zip(expected(x, w, b, t, -g).items(), got):
        close(name, a, ref, "f16")
