"""Host side of the output layer's losses: refusals before any launch, and workspace sizes (no GPU needed)."""
import ctypes as C

import pytest

import __graft_entry__ as entry
import paper_2505_13765_b200 as pkg
from paper_2505_13765_b200 import binding as bd


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return pkg.load_library()


def layer(**kw):
    d = dict(n_out=1025, H=640, dtype=bd.WIND_DT_BF16, reserved=0, w=1 << 20, ldw=640, b=None)
    d.update(kw)
    return bd.wind_output_t(**d)


def size(lib, o, N, K=0, grad=0):
    n = C.c_size_t(0)
    st = lib.wind_loss_workspace_bytes(C.byref(o), N, K, grad, C.byref(n))
    return n.value if st == bd.WIND_OK else -st


def test_workspace_sizes(lib):
    n = C.c_size_t(0)
    assert lib.wind_loss_workspace_bytes(None, 1, 0, 0, C.byref(n)) == bd.WIND_ERR_INVALID_ARG
    assert lib.wind_loss_workspace_bytes(C.byref(layer()), 1, 0, 0, None) == bd.WIND_ERR_INVALID_ARG
    for bad in (dict(n_out=0), dict(H=0), dict(dtype=2), dict(ldw=-1)):
        assert size(lib, layer(**bad), 1) == -bd.WIND_ERR_INVALID_ARG, bad
    assert size(lib, layer(), -1) == -bd.WIND_ERR_INVALID_ARG
    assert size(lib, layer(), 1, -1) == -bd.WIND_ERR_INVALID_ARG
    for N, K, kw in ((1, 257, {}), ((1 << 24) + 1, 0, {}), (1, 0, dict(n_out=1 << 24)), (1 << 24, 0, dict(n_out=1 << 17)), (1, 0, dict(H=65537))):
        assert size(lib, layer(**kw), N, K) == -bd.WIND_ERR_UNSUPPORTED
    assert size(lib, layer(), 0) > 0
    # a loss keeps three numbers per row and 128 outputs, never a row's logits
    big = layer(n_out=65536, H=2048, ldw=2048)
    x = 4096 * 2048 * 2
    assert x < size(lib, big, 4096) < x + 4096 * (65536 // 128) * 12 + (1 << 20)
    # a gradient keeps at most 512 MB of its share of logits (or 2048 outputs' worth)
    g = size(lib, big, 4096, 0, 1)
    assert g < 2 * x + (512 << 20) + (512 << 20) // 64 + 2 * 814 * 128 * 256 * 4
    rows = 1 << 20
    many = layer(n_out=65536, H=64, ldw=64)
    assert size(lib, many, rows, 0, 1) < rows * (2048 * 2 + 64 * (2 + 4) + 2048 // 128 * 4 + 64)
    # rows that do not start on 16 bytes, and fp32: W in the kernels' own layout
    assert size(lib, layer(w=(1 << 20) + 2), 8) >= size(lib, layer(), 8) + 1025 * 640 * 2
    assert size(lib, layer(ldw=641), 8) >= size(lib, layer(), 8) + 1025 * 640 * 2
    assert size(lib, layer(dtype=bd.WIND_DT_F32), 8) >= size(lib, layer(), 8) + 1025 * 640 * 6
    # what N rows need serves fewer rows and entries
    rows_of = sorted(set([0, 1, 2, 127, 128, 129, 255, 256, 257, 384, 385, 512, 513, 8192, 8193, 20011, 32768, 32769, 100000, 1 << 20] +
                         list(range(130, 9000, 331))))
    for kw in (dict(), dict(n_out=33, H=64, ldw=64), dict(n_out=8193, H=1024, ldw=1024), dict(n_out=65536, H=2048, ldw=2048),
               dict(dtype=bd.WIND_DT_F32), dict(dtype=bd.WIND_DT_F32, n_out=8193, H=1024, ldw=1024), dict(H=1, ldw=1, n_out=1)):
        for K, grad in ((0, 0), (0, 1), (16, 0), (256, 1)):
            sizes = [size(lib, layer(**kw), N, K, grad) for N in rows_of]
            assert sizes == sorted(sizes), (kw, K, grad)
            assert size(lib, layer(**kw), 777, 0, grad) <= size(lib, layer(**kw), 777, 16, grad)


def test_calls_are_refused_before_any_launch(lib):
    # device addresses that are never followed: every call returns on the host
    p, ws, some = 1 << 20, 1 << 21, (1 << 40)
    o = C.byref(layer())
    lab = [o, p, 640, p, 4, p, p, ws, some, None]
    grad = [o, p, 640, p, 4, p, p, p, 640, p, 640, p, ws, some, None]
    dist = [o, p, 640, p, p, 4, 8, 1.0, p, p, ws, some, None]
    dgrad = [o, p, 640, p, p, 4, 8, 1.0, p, p, p, 640, p, 640, p, ws, some, None]

    def refused(f, args, at, value, status=bd.WIND_ERR_INVALID_ARG):
        a = list(args)
        a[at] = value
        assert f(*a) == status, (f, at, value)

    for f, args, n_at in ((lib.wind_label_loss, lab, 4), (lib.wind_label_loss_grad, grad, 4), (lib.wind_distill_loss, dist, 5),
                          (lib.wind_distill_loss_grad, dgrad, 5)):
        refused(f, args, 0, None)
        refused(f, args, 1, None)                                   # x
        refused(f, args, 2, -1)                                     # its row distance
        refused(f, args, 3, None)                                   # target, ids
        refused(f, args, n_at, -1)
        refused(f, args, n_at, (1 << 24) + 1, bd.WIND_ERR_UNSUPPORTED)
        refused(f, args, len(args) - 3, None)                       # workspace
        refused(f, args, len(args) - 3, ws + 16, bd.WIND_ERR_WORKSPACE)
        refused(f, args, len(args) - 2, 100, bd.WIND_ERR_WORKSPACE)
        for bad in (dict(w=None), dict(n_out=0), dict(H=-3), dict(dtype=7), dict(ldw=-640)):
            refused(f, args, 0, C.byref(layer(**bad)))
    # addresses that are none of an element's
    for f, args, vectors, matrices in ((lib.wind_label_loss, lab, (3, 5, 6), (1,)), (lib.wind_label_loss_grad, grad, (3, 5, 6, 11), (1, 7, 9)),
                                       (lib.wind_distill_loss, dist, (3, 4, 8, 9), (1,)),
                                       (lib.wind_distill_loss_grad, dgrad, (3, 4, 8, 9, 14), (1, 10, 12))):
        for at in vectors:
            refused(f, args, at, p + 2)
        for at in matrices:
            refused(f, args, at, p + 1)
            refused(f, [C.byref(layer(dtype=bd.WIND_DT_F32))] + args[1:], at, p + 2)
        refused(f, args, 0, C.byref(layer(w=(1 << 20) + 1)))
    refused(lib.wind_label_loss, lab, 5, None)
    refused(lib.wind_label_loss, lab, 6, None)
    refused(lib.wind_label_loss_grad, grad, 5, None)                # lse
    refused(lib.wind_label_loss_grad, grad, 8, 639)                 # rows of dx, dw shorter than H
    refused(lib.wind_label_loss_grad, grad, 10, 639)
    for f, args in ((lib.wind_distill_loss, dist), (lib.wind_distill_loss_grad, dgrad)):
        refused(f, args, 4, None)                                   # teacher
        refused(f, args, 6, 0)
        refused(f, args, 6, 257, bd.WIND_ERR_UNSUPPORTED)
        for tau in (0.0, -1.0, float("inf"), float("nan")):
            refused(f, args, 7, tau)
        refused(f, args, 8, None)                                   # loss, lse
    refused(lib.wind_distill_loss, dist, 9, None)
    assert lib.wind_loss_status(None, None) == bd.WIND_ERR_INVALID_ARG


def test_reported_sizes_are_enough(lib):
    """A workspace of the reported size is accepted by calls of as many rows and of fewer (they go on to the device, which is not there)."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the calls have addresses that must not reach a device")
    import random
    r = random.Random(3)
    p, ws = 1 << 20, 1 << 21
    for _ in range(3000):
        H, n_out = int(2 ** r.uniform(0, 12)), int(2 ** r.uniform(0, 17))
        o = layer(H=H, ldw=H, n_out=n_out, dtype=r.choice([0, 1]))
        N, K = int(2 ** r.uniform(0, 18)), r.choice([0, 1, 40])
        n = max(1, min(N, int(N * r.choice([1.0, 1.0, r.random()]))))
        ref, rows = C.byref(o), ((p, p, n, K, 1.0) if K else (p, n))
        for grad in (0, 1):
            have = size(lib, o, N, K, grad)
            assert have > 0
            if grad:
                f = lib.wind_distill_loss_grad if K else lib.wind_label_loss_grad
                st = f(ref, p, H, *rows, p, p, p, H, p, H, p, ws, have, None)
            else:
                f = lib.wind_distill_loss if K else lib.wind_label_loss
                st = f(ref, p, H, *rows, p, p, ws, have, None)
            assert st == bd.WIND_ERR_CUDA, (st, H, n_out, o.dtype, N, n, K, grad)


def test_no_cpu_path(lib):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is there")
    x, w = torch.zeros(2, 8), torch.zeros(3, 8)
    v, t = torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        pkg.wind_label_loss(x, w, None, t, v, v, torch.zeros(1 << 20, dtype=torch.uint8))
