"""Calls of the output layer's losses that their documentation allows, beside those of test_gpu_loss.py, and refusals of the binding."""
import ctypes as C
import math

import pytest

from test_gpu_loss import DEV, DT, call, make, pkg, reference, verify, verify_in_slices  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 3, 200, 300])
def test_a_single_row_may_be_any_distance_from_the_next(pkg, dtype, N):  # noqa: F811
    """One output: the distance between W's rows says nothing.  (Through the C interface: torch gives such a matrix its own distance.)"""
    bd, lib = pkg.binding, pkg.load_library()
    c = make(13 + N, dtype, N, 64, 1, pad=0.0)
    ref = reference(c)
    stream = torch.cuda.current_stream().cuda_stream
    for ld in (0, 7, 8, 64, 1 << 41, 1 << 50):
        o = bd.wind_output_t(n_out=1, H=64, dtype=bd.WIND_DT_F32 if dtype == "f32" else bd.WIND_DT_BF16, reserved=0, w=c["w"].data_ptr(), ldw=ld,
                             b=c["b"].data_ptr())
        sizes = [C.c_size_t(0), C.c_size_t(0)]
        for grad in (0, 1):
            assert lib.wind_loss_workspace_bytes(C.byref(o), N, 0, grad, C.byref(sizes[grad])) == 0
        size = max(s.value for s in sizes)
        ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
        loss, lse = (torch.full((N,), math.nan, device=DEV) for _ in range(2))
        dx, dw, db = torch.full_like(c["x"], math.nan), torch.full_like(c["w"], math.nan), torch.full((1,), math.nan, device=DEV)
        x, t = c["x"].data_ptr(), c["t"].data_ptr()
        ldx = ld if N == 1 else 64
        assert lib.wind_label_loss(C.byref(o), x, ldx, t, N, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), size, stream) == 0
        assert lib.wind_label_loss_grad(C.byref(o), x, ldx, t, N, lse.data_ptr(), c["dloss"].data_ptr(), dx.data_ptr(), 64, dw.data_ptr(), 64,
                                        db.data_ptr(), ws.data_ptr(), size, stream) == 0
        assert lib.wind_loss_status(ws.data_ptr(), stream) == 0
        verify(dict(loss=loss, lse=lse, dx=dx, dw=dw, db=db), ref, ld)


def test_what_is_no_tensor_is_refused_by_name(pkg):  # noqa: F811
    c, d = make(1, "bf16", 6, 16, 9), make(2, "bf16", 6, 16, 9, 2)
    ws = pkg.alloc_loss_workspace(c["w"], 6, 2, True)
    v = [torch.empty(6, device=DEV) for _ in range(2)]
    label = dict(x=c["x"], weight=c["w"], bias=c["b"], target=c["t"], loss=v[0], lse=v[1], workspace=ws)
    distill = dict(x=d["x"], weight=d["w"], bias=d["b"], ids=d["ids"], teacher=d["y"], tau=1.0, loss=v[0], lse=v[1], workspace=ws)
    grads = dict(dloss=None, dx=torch.empty_like(c["x"]), dw=torch.empty_like(c["w"]), db=torch.empty(9, device=DEV))
    label_grad = {**{k: v for k, v in label.items() if k != "loss"}, **grads}
    distill_grad = {**{k: v for k, v in distill.items() if k != "loss"}, **grads}
    optional = ("bias", "dloss", "dx", "dw", "db", "tau")
    for f, good in ((pkg.wind_label_loss, label), (pkg.wind_distill_loss, distill), (pkg.wind_label_loss_grad, label_grad),
                    (pkg.wind_distill_loss_grad, distill_grad)):
        f(**good, check=True)
        for k in good:
            for bad in ([1.0, 2.0], 3) + ((None,) if k not in optional else ()):
                if k != "tau":
                    with pytest.raises(ValueError, match=k if k not in ("loss", "lse") or bad is not None else "loss"):
                        f(**{**good, k: bad})
    with pytest.raises(ValueError, match="weight"):
        pkg.alloc_loss_workspace(None, 6)
