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


WANTS = [("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db"), ("dx", "dw")]


@pytest.mark.parametrize("dtype,N,H,V,K,slices", [
    ("bf16", 3000, 1024, 9001, 0, 0),         # a CTA to a tile of logits, two to one of dx and dW
    ("bf16", 3000, 1208, 9001, 5, 0),         # the same with logits from several accumulators
    ("bf16", 8192, 1544, 40000, 0, 2048),     # two pieces of the outputs, tiles by two CTAs throughout
    ("bf16", 9000, 2048, 31000, 3, 1500),     # the last piece a fraction of the first, rows that end inside a tile
    ("f32", 333, 136, 1100, 3, 0), ("bf16", 100, 64, 300, 0, 0), ("bf16", 7, 640, 1025, 8, 0), ("f32", 44001, 16, 2300, 0, 20000),
    ("bf16", 140001, 24, 4200, 0, 20000),
])
def test_some_of_the_gradients_in_every_form(pkg, dtype, N, H, V, K, slices):  # noqa: F811
    """All gradients against the definition, then any of them alone: the same bits, whatever else is asked for."""
    c = make(N + H + V + K, dtype, N, H, V, K, pad=0.1 if N > 10 else 0.0)
    got = call(pkg, c)
    if slices:
        verify_in_slices(got, c, slices)
    else:
        verify(got, reference(c))
    for want in WANTS:
        some = call(pkg, c, want=want)
        for k in want:
            assert torch.equal(some[k], got[k]), (want, k)


@pytest.mark.parametrize("dtype,N,H,V,K", [("bf16", 900, 2048, 12289, 5), ("bf16", 3000, 1208, 9001, 0), ("f32", 500, 72, 700, 3), ("bf16", 70, 64, 300, 0)])
def test_every_form_captured_and_replayed(pkg, dtype, N, H, V, K):  # noqa: F811
    first, second = (make(s, dtype, N, H, V, K, pad=0.1) for s in (5, 6))
    c = {k: (v.clone() if torch.is_tensor(v) else v) for k, v in first.items()}
    ws = pkg.alloc_loss_workspace(c["w"], N, K, True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(pkg, c, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call(pkg, c, ws=ws, check=False)
    for d in (second, first):
        for k, v in d.items():
            if torch.is_tensor(v):
                c[k].copy_(v)
        for v in out.values():
            v.fill_(math.nan)
        g.replay()
        assert pkg.wind_loss_status(ws) == 0
        verify(out, reference(d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_teacher_by_its_own_window_and_a_students_loss(pkg, dtype):  # noqa: F811
    """The chain as a user runs it: the teacher's K best labels of single frames by wind_window_first_output go into the distillation of
    another model's output layer as they are; an utterance without a frame there is a row of padding."""
    import numpy as np
    from naive_model import random_weights
    r = np.random.default_rng(9)
    B, T, V, K, H = 40, 12, 60, 7, 48
    teacher = random_weights(r, 32, 64, 64, 2, 96, V, act=0, bias_scale=0.1)
    enc = r.standard_normal((B, T, 32)).astype(np.float32)
    lens = r.integers(1, T + 1, B).astype(np.int32)
    lens[[3, 17]] = 0
    t0 = np.where(lens > 0, r.integers(0, 100, B) % np.maximum(lens, 1), 0).astype(np.int32)
    m = pkg.WindModel(teacher)
    up = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    logp = torch.full((B, 1, V + 1), math.nan, device=DEV)
    ids, jump = (torch.full((B, K), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    best = torch.full((B, K), math.nan, device=DEV)
    pkg.wind_window_first_output(m, pkg.to_device_enc(m, enc), up(lens), 1, up(r.integers(0, V, (B, 3)).astype(np.int32)),
                                 up(r.integers(0, 4, B).astype(np.int32)), up(t0), logp, pkg.alloc_workspace(m, B, T, 1), K=K, top_label=ids,
                                 top_jump=jump, top_logp=best)
    c = make(4, dtype, B, H, V + 1, pad=0.0)
    del c["t"]
    c.update(ids=ids, y=best, tau=2.0)
    ref = reference(c)
    assert ref["keep"].tolist() == [bool(n) for n in lens]
    got = call(pkg, c)
    verify(got, ref)
    # and from the whole distribution that the teacher gave, with the same labels kept: log-probabilities, renormalised at tau
    kept = torch.full((B, V + 1), -math.inf, dtype=torch.float64, device=DEV)
    rows = ref["keep"]
    kept[rows] = kept[rows].scatter(1, ids[rows].long(), logp[rows, 0].double().gather(1, ids[rows].long()))
    q = torch.softmax(kept[rows] / 2, 1)
    z = (c["x"].double() @ c["w"].double().T + c["b"].double())[rows] / 2
    want = 4 * (torch.special.xlogy(q, q) - q * torch.log_softmax(z, 1)).sum(1)
    assert bool(((got["loss"][rows].double() - want).abs() <= ref["tol_loss"]).all())


def test_two_calls_at_once_in_every_form(pkg):  # noqa: F811
    """Calls on streams of their own from threads of their own, each with its own workspace: pairs of CTAs, long rows, few rows, fp32."""
    import threading
    made = [make(30 + i, dtype, N, H, V, K, pad=0.1) for i, (dtype, N, H, V, K) in enumerate(
        [("bf16", 900, 2048, 12289, 3), ("bf16", 1700, 1640, 5377, 0), ("bf16", 600, 1100, 1000, 0), ("f32", 500, 200, 3000, 0), ("bf16", 1, 1024, 8193, 0)])]
    refs = [reference(c) for c in made]
    torch.cuda.synchronize()
    out = [None] * len(made)

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            ws = pkg.alloc_loss_workspace(made[i]["w"], made[i]["x"].shape[0], made[i]["ids"].shape[1] if "ids" in made[i] else 0, True)
            for _ in range(6):
                out[i] = call(pkg, made[i], ws=ws, check=False)
            assert pkg.wind_loss_status(ws, check=False) == 0
        s.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(made))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i, c in enumerate(made):
        assert out[i] is not None
        verify(out[i], refs[i], i)
