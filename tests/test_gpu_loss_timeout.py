"""Failure path of the losses' kernels: a wait that can never end (test hook) runs out after about two seconds and the CTAs leave by
themselves.  The workspace says so when it is asked, whatever calls came in between, and the next call on it is right."""
import pytest

from test_gpu_loss import call, make, pkg, reference, verify  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FORMS = {  # dtype, N, H, V, K
    "direct": ("bf16", 5, 64, 300, 0),            # reads x where it is, nothing runs ahead of the products
    "few": ("bf16", 200, 64, 300, 3),
    "f32": ("f32", 300, 72, 500, 0),
    "bf16": ("bf16", 700, 136, 2000, 0),
    "one_part": ("bf16", 700, 136, 100, 0),       # the products' kernel writes the results itself
    "long": ("bf16", 600, 1100, 1000, 0),
    "pairs": ("bf16", 900, 2048, 12289, 0),
}
CASES = [("direct", 0, 1), ("direct", 0, 2), ("direct", 0, 3), ("few", 0, 1), ("few", 1, 2), ("f32", 0, 3), ("f32", 1, 1), ("f32", 2, 2),
         ("bf16", 0, 1), ("bf16", 0, 2), ("bf16", 1, 1), ("bf16", 1, 3), ("bf16", 2, 1), ("bf16", 2, 2), ("one_part", 0, 2), ("long", 0, 2),
         ("long", 1, 1), ("pairs", 0, 1), ("pairs", 0, 2), ("pairs", 0, 3), ("pairs", 1, 2), ("pairs", 1, 3), ("pairs", 2, 1), ("pairs", 2, 3)]


@pytest.mark.parametrize("form,kernel,wait", CASES)
def test_wait_that_never_ends(pkg, form, kernel, wait):  # noqa: F811
    dtype, N, H, V, K = FORMS[form]
    c = make(7 + N, dtype, N, H, V, K, pad=0.1)
    ws = pkg.alloc_loss_workspace(c["w"], N, K, True)
    ws.zero_()
    call(pkg, c, ws=ws)
    prev = pkg.wind_debug_stall_loss(3 * kernel + wait)
    try:
        call(pkg, c, ws=ws, grad=kernel > 0, check=False)
        torch.cuda.synchronize()
    finally:
        pkg.wind_debug_stall_loss(prev)
    call(pkg, c, ws=ws, grad=kernel == 0, check=False)     # calls that come after do not cover it up
    with pytest.raises(pkg.WindError) as e:
        pkg.wind_loss_status(ws)
    assert e.value.status == pkg.binding.WIND_ERR_TIMEOUT
    assert pkg.wind_loss_status(ws) == 0                   # said once
    verify(call(pkg, c, ws=ws), reference(c))


def test_it_is_not_forgotten_where_there_are_no_rows(pkg):  # noqa: F811
    c = make(3, "bf16", 5, 64, 300)
    ws = pkg.alloc_loss_workspace(c["w"], 5, 0, True)
    ws.zero_()
    call(pkg, c, ws=ws)
    prev = pkg.wind_debug_stall_loss(1)
    try:
        call(pkg, c, ws=ws, grad=False, check=False)
        torch.cuda.synchronize()
    finally:
        pkg.wind_debug_stall_loss(prev)
    none = {k: (v[:0] if k in ("x", "t", "dloss") else v) for k, v in c.items()}
    call(pkg, none, ws=ws, check=False)
    assert pkg.wind_loss_status(ws, check=False) == pkg.binding.WIND_ERR_TIMEOUT
    assert pkg.wind_loss_status(ws) == 0
