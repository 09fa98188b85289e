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
