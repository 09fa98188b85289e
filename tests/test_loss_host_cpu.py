"""Host side of the output layer's losses beside test_loss_cpu.py: hooks, sizes of the largest calls, refusals (no GPU needed)."""
import ctypes as C

import pytest

import paper_2505_13765_b200 as pkg
from paper_2505_13765_b200 import binding as bd
from test_loss_cpu import layer, lib, size  # noqa: F401


def test_stall_hook_round_trip(lib):  # noqa: F811
    assert pkg.wind_debug_stall_loss(9) == 0 and pkg.wind_debug_stall_loss(10) == 9 and pkg.wind_debug_stall_loss(0) == 0


def test_reported_sizes_are_enough_over_the_whole_range(lib):  # noqa: F811
    """A workspace of the reported size is taken by calls of as many rows and of fewer, up to the largest calls (they go on to the device,
    which is not there)."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the calls have addresses that must not reach a device")
    import random
    r = random.Random(5)
    p, ws, n_long = 1 << 20, 1 << 21, 0
    for i in range(6000):
        H, n_out = min(65536, int(2 ** r.uniform(0, 16))), min((1 << 24) - 1, int(2 ** r.uniform(0, 24)))
        N = min(1 << 24, (1 << 40) // n_out, int(2 ** r.uniform(0, 24)))
        K = r.choice([0, 0, 7, 256])
        o = layer(H=H, ldw=H, n_out=n_out, dtype=r.choice([bd.WIND_DT_BF16, bd.WIND_DT_BF16, bd.WIND_DT_F32]))
        n_long += N > 65536 and o.dtype == bd.WIND_DT_BF16
        ref, have = C.byref(o), size(lib, o, N, K, 1)
        assert have > 0
        for n in {N, max(1, int(N * r.random())), min(N, 256), min(N, int(2 ** r.uniform(0, 24)))}:
            rows = (p, p, n, K, 1.0) if K else (p, n)
            f = lib.wind_distill_loss_grad if K else lib.wind_label_loss_grad
            st = f(ref, p, H, *rows, p, p, p, H, p, H, p, ws, have, None)
            assert st == bd.WIND_ERR_CUDA, (st, H, n_out, o.dtype, N, n, K)
    assert n_long > 500


def test_temperatures_without_a_reciprocal_are_refused(lib):  # noqa: F811
    o, p, ws = C.byref(layer()), 1 << 20, 1 << 21
    for tau in (1e-45, 1e-39, 3e-39, 1.17e-38):
        assert lib.wind_distill_loss(o, p, 640, p, p, 4, 8, tau, p, p, ws, 1 << 40, None) == bd.WIND_ERR_INVALID_ARG
        assert lib.wind_distill_loss_grad(o, p, 640, p, p, 4, 8, tau, p, p, p, 640, p, 640, p, ws, 1 << 40, None) == bd.WIND_ERR_INVALID_ARG
    for tau in (2.0 ** -126, 3e38):      # (refused for the workspace alone)
        assert lib.wind_distill_loss(o, p, 640, p, p, 4, 8, tau, p, p, ws, 100, None) == bd.WIND_ERR_WORKSPACE
