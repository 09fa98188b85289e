"""Sums of the output layer's losses on the tensor cores, which cut where they add: what is exact stays exact, and long sums lose no more
than the additions of one accumulator."""
import math

import pytest

from test_gpu_loss import DEV, DT, call, make, pkg, reference, verify  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def one_output(x, w, at, dtype="bf16"):
    """A call in which a bias of -inf leaves output `at` alone: log-sum-exp and maximum are its logit, bit by bit, and the loss is zero."""
    N, V = x.shape[0], w.shape[0]
    b = torch.full((V,), -math.inf, device=DEV)
    b[at] = 0.0
    return dict(x=x, w=w, b=b, t=torch.full((N,), at, dtype=torch.int32, device=DEV), dloss=None, tau=1.0)


SIZES = [(130, 640, 1), (257, 8, 5), (300, 64, 1), (300, 640, 257), (300, 1024, 1), (270, 1032, 33), (300, 2048, 300), (1000, 1536, 9), (300, 4104, 7),
         (700, 65536, 1), (2000, 2048, 4864), (300, 1032, 40000)]


@pytest.mark.parametrize("N,H,V", SIZES)
def test_sums_that_are_exact(pkg, N, H, V):  # noqa: F811
    """One value a row (a product, and zeros added to it), and small whole numbers (partial sums below 2^24): nothing is cut, and nothing
    may be added."""
    g = torch.Generator(device=DEV).manual_seed(N + H + V)
    w = torch.randn(V, H, generator=g, device=DEV).bfloat16()
    x = torch.zeros(N, H, dtype=torch.bfloat16, device=DEV)
    at = torch.randint(0, H, (N,), generator=g, device=DEV)
    x[torch.arange(N, device=DEV), at] = torch.randn(N, generator=g, device=DEV).bfloat16()
    for v in {0, V - 1}:
        got = call(pkg, one_output(x, w, v), grad=False)
        assert torch.equal(got["lse"].double(), (x.double() @ w[v].double()))
        assert bool((got["loss"] == 0).all())
    x = torch.randint(-5, 6, (N, H), generator=g, device=DEV).bfloat16()
    w = torch.randint(-7, 8, (V, H), generator=g, device=DEV).bfloat16()     # (|sums| <= 35 x 65536 < 2^24)
    got = call(pkg, one_output(x, w, V - 1), grad=False)
    assert torch.equal(got["lse"].double(), (x.double() @ w[V - 1].double()))


@pytest.mark.parametrize("N,H,V", [(300, 1024, 3), (300, 1032, 3), (300, 2048, 3), (1000, 4096, 2), (300, 16384, 2), (2000, 2048, 4864)])
@pytest.mark.parametrize("kind", ["normal", "relu", "positive"])
def test_long_sums_of_logits(pkg, N, H, V, kind):  # noqa: F811
    """A logit loses at most 2^-23 of the magnitudes in its accumulator with each of its additions, of which an accumulator takes 64 at most,
    and half of that in each joining of two accumulators, which rounds."""
    g = torch.Generator(device=DEV).manual_seed(N + H)
    x = torch.randn(N, H, generator=g, device=DEV)
    w = torch.randn(V, H, generator=g, device=DEV) / math.sqrt(H)
    x, w = (x.relu(), w) if kind == "relu" else (x.abs(), w.abs()) if kind == "positive" else (x, w)
    x, w = x.bfloat16(), w.bfloat16()
    got = call(pkg, one_output(x, w, V - 1), grad=False)["lse"].double()
    want, size = x.double() @ w[V - 1].double(), x.double().abs() @ w[V - 1].double().abs()
    additions = 64 + math.ceil(H / 1024) / 2
    assert bool(((got - want).abs() <= additions * 2.0 ** -23 * size).all())
    # One way: over many rows of normal operands a random walk of 64 additions loses a share of 64 x 2^-25 on the mean: half a step is cut,
    # a step is 0.72 x 2^-23 of the accumulator on the mean, the accumulator two thirds of its end.
    if kind == "normal" and H > 1024:
        share = float(((got - want) * want.sign()).sum() / want.abs().sum())
        assert abs(share) <= 64 * 2.0 ** -25, share


def test_long_sums_of_dw(pkg):  # noqa: F811
    """Two million rows of positive activations against equal probabilities: dW's sums are cut one way, but only within an accumulator."""
    N, H, V = 1 << 21, 1792, 2048
    g = torch.Generator(device=DEV).manual_seed(1)
    x = (0.5 + 0.5 * torch.rand(N, H, generator=g, device=DEV, dtype=torch.bfloat16)).clamp_(max=1.0)
    w = torch.zeros(V, H, dtype=torch.bfloat16, device=DEV)
    t = torch.zeros(N, dtype=torch.int32, device=DEV)
    lse = torch.full((N,), math.log(V), device=DEV)
    dw = torch.full((V, H), math.nan, dtype=torch.bfloat16, device=DEV)
    ws = pkg.alloc_loss_workspace(w, N, 0, True)
    pkg.wind_label_loss_grad(x, w, None, t, lse, None, None, dw, None, ws, check=True)
    # g is 2^-11 but for the target's output (of which lse's rounding, at most 2^-21 relative, is lost in g's rounding to bf16)
    want = torch.stack([x[:, h0: h0 + 128].sum(0, dtype=torch.float64) for h0 in range(0, H, 128)]).flatten() * 2.0 ** -11
    # The columns' sums are 767 with a sigma of 0.1, bf16's step there is 4: all round the same way, by up to half a step, so that neither a
    # column's nor the mean's distance says anything below 2^-8.  Rounding is monotone, though: the fp32 sum lies between the exact one less
    # 4096 cuts of at most 2^-23 of the accumulator (half its end on the mean, as it grows evenly) and the exact one plus 32 joinings' 2^-24.
    low, high = ((want * f).float().bfloat16() for f in (1.0 - 4096 * 2.0 ** -24, 1.0 + 32 * 2.0 ** -24))
    assert bool((dw[1:] >= low).all()) and bool((dw[1:] <= high).all()), (float(dw[1:].min()), float(dw[1:].max()), float(low.min()), float(high.max()))


@pytest.mark.parametrize("N,H,V,kinds", [(70000, 264, 1100, ("dx", "dw", "db")), (131100, 1544, 300, ("dw",)), (200, 136, 70001, ("dx", "dw", "db"))])
def test_sums_cut_for_their_length(pkg, N, H, V, kinds):  # noqa: F811
    """Rows and outputs from which on a sum of dW or dx has several parts for its length, ragged ones among them."""
    from test_gpu_loss import verify_in_slices
    c = make(N + H, "bf16", N, H, V, pad=0.1)
    got = call(pkg, c, want=kinds)
    if len(kinds) == 3:
        verify_in_slices(got, c, 20000)
        return
    keep = c["t"] >= 0
    z = torch.where(keep[:, None], c["x"].float(), 0.0).double() @ c["w"].double().T + c["b"].double()
    q = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    q[torch.arange(N, device=DEV)[keep], c["t"][keep].long()] -= 1.0
    q *= torch.where(keep, c["dloss"].double(), 0.0)[:, None]
    xd = torch.where(keep[:, None], c["x"].double(), 0.0)
    want, size = q.T @ xd, q.abs().T @ xd.abs()
    # a bf16 rounding of g and one of dW, the sums' cuts, and what p is off (a share of g of at most 2^-10: logits 2^-14 off)
    assert bool(((got["dw"].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -11) * size + 2.0 ** -8 * want.abs()).all())
