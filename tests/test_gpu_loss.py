"""The output layer's losses and gradients against their definitions in 64 bits.

Bounds, element by element, from the arithmetic:
  logits   bf16 operands multiply exactly; a sum of H products in fp32 (tensor cores may cut instead of rounding: 2^-23 a step of 16)
           is off by at most (H / 16 + 8) 2^-23 times the sum of the magnitudes, A.  fp32 operands: six part products a product, those
           left out are below 2^-22 of it.
  loss     two logits or sums over them, and fp32 exponentials (2^-21) and logarithms: 2 e_z + 2^-20 (1 + the largest logit) (times tau^2)
  g        s (p - q): p is off by p (2 e_z + the loss's) and then g is rounded to bf16 (half a step: 2^-8; fp32: three parts, 2^-22)
  dx, dW   |g| |W| times that, plus fp32 sums of n products (n / 16 + 8 steps, 8 more for the joined parts), then bf16's half step
  db       |g| times g's bound without the rounding, plus an fp32 sum
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_13765_b200 as p
    p.load_library()
    return p


def strided(t, ld, offset=0, fill=float("nan")):
    """A copy of matrix t whose rows stand ld elements apart, `offset` elements behind the start of a buffer of `fill`."""
    buf = torch.full((offset + t.shape[0] * ld + 8,), fill, dtype=t.dtype, device=t.device)
    v = buf[offset: offset + t.shape[0] * ld].view(t.shape[0], ld)[:, : t.shape[1]]
    v.copy_(t)
    return v, buf


def make(seed, dtype, N, H, V, K=0, pad=0.2, bias=True, gain=2.0, full=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    u = lambda *s: torch.rand(*s, generator=g, device=DEV)  # noqa: E731
    c = dict(x=r(N, H).to(DT[dtype]), w=(r(V, H) * gain / math.sqrt(H)).to(DT[dtype]), b=r(V) if bias else None,
             dloss=u(N) + 0.5, tau=1.0)
    padding = u(N) < pad
    if K:
        ids = torch.randint(0, V, (N, K), generator=g, device=DEV)      # the same label may stand there twice
        gone = (u(N, K) < (0.0 if full else 0.3)) | padding[:, None]
        c["ids"] = torch.where(gone, -1, ids).int()
        y = 2.0 * r(N, K)
        y = torch.where(u(N, K) < 0.1, -math.inf, y)
        c["y"] = torch.where(gone, math.nan, y)                         # not read where there is no entry
        c["tau"] = 1.7
    else:
        c["t"] = torch.where(padding, -1, torch.randint(0, V, (N,), generator=g, device=DEV)).int()
    c["x"][padding] = math.nan                                          # not read either
    return c


def targets(c):
    """(rows that count, their target distribution [N, V] and its entropy) in 64 bits."""
    N, V = c["x"].shape[0], c["w"].shape[0]
    q = torch.zeros(N, V, dtype=torch.float64, device=DEV)
    ent = torch.zeros(N, dtype=torch.float64, device=DEV)
    if "t" in c:
        keep = c["t"] >= 0
        q[torch.arange(N, device=DEV)[keep], c["t"][keep].long()] = 1.0
        return keep, q, ent
    there = c["ids"] >= 0
    y = torch.where(there, c["y"].double(), -math.inf) / c["tau"]
    keep = (y > -math.inf).any(1)
    p = torch.softmax(torch.where(keep[:, None], y, torch.zeros_like(y)), 1) * keep[:, None] * there
    q.scatter_add_(1, c["ids"].clamp(min=0).long(), p)
    # every entry against the student's probability of its label: sum_k q_k ln q_k over entries, twice-named labels included
    ent = torch.special.xlogy(p, p).sum(1)
    return keep, q, ent


def reference(c, grad=True):
    keep, q, ent = targets(c)
    tau = c["tau"]
    x = torch.where(keep[:, None], c["x"].double(), 0.0)
    w = c["w"].double()
    b = torch.zeros(w.shape[0], dtype=torch.float64, device=DEV) if c["b"] is None else c["b"].double()
    z = (x @ w.T + b) / tau
    lse = torch.logsumexp(z, 1)
    qz = torch.where(q > 0, q * z, torch.zeros_like(z)).sum(1)
    loss = tau ** 2 * (ent + lse - qz)
    out = dict(keep=keep, loss=torch.where(keep, loss, 0.0), lse=torch.where(keep, lse, 0.0))
    H, V, N = w.shape[1], w.shape[0], x.shape[0]
    f32 = c["w"].dtype == torch.float32
    A = ((x.abs() @ w.abs().T).max() + torch.where(b > -1e30, b.abs(), torch.zeros_like(b)).max()) / tau   # (largest row of magnitudes)
    steps = (6 if f32 else 1) * H / 16 + 8
    e_z = float(A) * (steps * 2.0 ** -23 + (2.0 ** -22 if f32 else 0.0))
    top = float(torch.where(z > -1e30, z.abs(), torch.zeros_like(z)).max())
    out["tol_loss"] = tau ** 2 * (2 * e_z + 2.0 ** -20 * (1 + top))
    out["tol_lse"] = e_z + 2.0 ** -20 * (1 + top)
    if not grad:
        return out
    dl = torch.ones(N, dtype=torch.float64, device=DEV) if c["dloss"] is None else c["dloss"].double()
    s = torch.where(keep, dl * tau, 0.0)[:, None]
    p = torch.exp(z - lse[:, None])
    g = s * (p - q)
    off = s * (p * (2 * e_z + 2.0 ** -20 * (1 + top)) + 2.0 ** -22 * (p + q))     # before g is rounded
    g_off = off + g.abs() * (2.0 ** -22 if f32 else 2.0 ** -8)
    parts = 6 if f32 else 1
    last = 2.0 ** -24 if f32 else 2.0 ** -8
    sum_x, sum_w = (parts * V / 16 + 16) * 2.0 ** -23, (parts * N / 16 + 16) * 2.0 ** -23
    out["dx"], out["dw"], out["db"] = g @ w, g.T @ x, g.sum(0)
    cut = 2.0 ** -22 if f32 else 0.0
    out["tol_dx"] = (g_off + (sum_x + cut) * g.abs()) @ w.abs() * (1 + 2.0 ** -7) + last * out["dx"].abs()
    out["tol_dw"] = (g_off + (sum_w + cut) * g.abs()).T @ x.abs() * (1 + 2.0 ** -7) + last * out["dw"].abs()
    out["tol_db"] = (off + (N / 32 + 16) * 2.0 ** -23 * g.abs()).sum(0)
    out["abs_dw"], out["abs_db"] = g.abs().T @ x.abs(), g.abs().sum(0)
    return out


def verify_in_slices(got, c, slice_rows):
    """verify() for more rows than a reference of 64 bits has room for; sums over all rows have that many more fp32 steps than a slice's."""
    N, total = c["x"].shape[0], {}
    for r0 in range(0, N, slice_rows):
        rows = slice(r0, min(N, r0 + slice_rows))
        want = reference({k: (v[rows] if k in ("x", "t", "ids", "y", "dloss") else v) for k, v in c.items()})
        verify({k: got[k][rows] for k in ("loss", "lse", "dx")}, want, r0)
        for k in ("dw", "db", "tol_dw", "tol_db", "abs_dw", "abs_db"):
            total[k] = total.get(k, 0) + want[k]
    steps = N / 16 * (6 if c["w"].dtype == torch.float32 else 1) * 2.0 ** -23
    for k in ("dw", "db"):
        assert bool(((got[k].double() - total[k]).abs() <= total["tol_" + k] + steps * total["abs_" + k]).all()), k


def call(pkg, c, ws=None, grad=True, dx=None, dw=None, want=("dx", "dw", "db"), stream=None, check=True):
    N, V = c["x"].shape[0], c["w"].shape[0]
    K = c["ids"].shape[1] if "ids" in c else 0
    if ws is None:
        ws = pkg.alloc_loss_workspace(c["w"], N, K, grad)
        ws.fill_(255)                                      # NaN in every type: nothing may be read that was not written
    loss, lse = (torch.full((N,), math.nan, device=DEV) for _ in range(2))
    rows = (c["ids"], c["y"], c["tau"]) if K else (c["t"],)
    fwd, bwd = (pkg.wind_distill_loss, pkg.wind_distill_loss_grad) if K else (pkg.wind_label_loss, pkg.wind_label_loss_grad)
    fwd(c["x"], c["w"], c["b"], *rows, loss, lse, ws, stream=stream, check=check)
    out = dict(loss=loss, lse=lse)
    if grad:
        dx = torch.full((N, c["x"].shape[1]), math.nan, dtype=c["x"].dtype, device=DEV) if dx is None else dx
        dw = torch.full(tuple(c["w"].shape), math.nan, dtype=c["w"].dtype, device=DEV) if dw is None else dw
        db = torch.full((V,), math.nan, device=DEV)
        given = dict(dx=dx, dw=dw, db=db)
        bwd(c["x"], c["w"], c["b"], *rows, lse, c["dloss"], *(given[k] if k in want else None for k in ("dx", "dw", "db")), ws,
            stream=stream, check=check)
        out.update({k: given[k] for k in want})
    return out


def verify(got, ref, what=""):
    for k in got:
        tol = ref["tol_" + k]
        d = (got[k].double() - ref[k]).abs()
        same = got[k].double() == ref[k]                   # (infinities)
        bad = ~(same | (d <= tol))
        assert not bool(bad.any()), (what, k, int(bad.sum()), float(torch.nan_to_num(d, nan=math.inf).max()), float(torch.as_tensor(tol).max()))
    keep = ref["keep"]
    for k in ("loss", "lse", "dx"):
        if k in got:
            assert bool((got[k][~keep] == 0).all()), (what, k)


SHAPES = [  # N, H, V: around the sizes of tiles, bands and pieces
    (1, 8, 1), (1, 64, 33), (1, 1024, 8193), (2, 16, 2), (5, 40, 7), (63, 33, 129), (64, 1, 31), (65, 72, 128), (127, 96, 255),
    (128, 64, 256), (129, 64, 257), (130, 250, 300), (200, 640, 1025), (257, 264, 511), (1000, 136, 1500), (2300, 320, 700), (77, 1024, 8193),
    (4099, 64, 33),
]
LARGE = [  # enough tiles that two CTAs make one; odd numbers of row tiles, last tiles of a column or of a few columns of H
    (1700, 1640, 5377), (9100, 1544, 1025), (900, 2048, 12289), (20000, 8, 500), (2990, 640, 4097),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,H,V", SHAPES)
def test_label_loss_and_gradient(pkg, dtype, N, H, V):
    c = make(N + H + V, dtype, N, H, V, bias=(N + V) % 3 != 0, pad=0.25 if N > 2 else 0.0)
    verify(call(pkg, c), reference(c))


@pytest.mark.parametrize("N,H,V", LARGE)
@pytest.mark.parametrize("K", [0, 9])
def test_large_calls(pkg, N, H, V, K):
    c = make(N + H + V + K, "bf16", N, H, V, K, bias=N % 3 != 0, pad=0.1)
    verify(call(pkg, c), reference(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,H,V,K", [(1, 64, 33, 1), (3, 24, 5, 7), (7, 640, 1025, 8), (130, 72, 300, 33), (200, 640, 1025, 16), (257, 64, 8193, 64),
                                     (300, 48, 129, 256), (1500, 128, 513, 31), (90, 1000, 2000, 100)])
def test_distill_loss_and_gradient(pkg, dtype, N, H, V, K):
    c = make(N + H + V + K, dtype, N, H, V, K, pad=0.25 if N > 3 else 0.0, full=N <= 3)
    verify(call(pkg, c), reference(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("N", [100, 300])
@pytest.mark.parametrize("rows", ["none", "all", "last", "first", "every_other"])
def test_padding(pkg, dtype, K, N, rows):
    c = make(3, dtype, N, 72, 140, K, pad=0.0, full=True)
    r = torch.arange(N, device=DEV)
    out = {"none": r < 0, "all": r >= 0, "last": r >= 2 * N // 3, "first": r < 2 * N // 3, "every_other": r % 2 == 0}[rows]
    c["x"][out] = math.nan
    c["dloss"][out] = math.nan
    if K:
        c["ids"][out] = -1
    else:
        c["t"][out] = -1
    c["dloss"] = c["dloss"].contiguous()
    ref = reference({**c, "dloss": torch.where(out, torch.zeros_like(c["dloss"]), c["dloss"])})
    got = call(pkg, c)
    verify(got, ref, rows)
    if rows == "all":
        assert all(bool((got[k] == 0).all()) for k in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_teacher_lists_without_probability(pkg, dtype):
    c = make(11, dtype, 60, 40, 100, 6, pad=0.0, full=True)
    c["y"][3] = -math.inf                      # no probability anywhere: a row of padding
    c["y"][4, 1:] = -math.inf                  # one entry
    c["ids"][5] = 17                           # one label six times
    c["y"][6] = -3.0e38                        # the type's lowest values: equal probabilities
    c["ids"][7, 2:] = -1
    c["y"] = torch.where(c["ids"] < 0, math.nan, c["y"])
    ref = reference(c)
    assert not bool(ref["keep"][3]) and int(ref["keep"].sum()) == 59
    verify(call(pkg, c), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 4])
@pytest.mark.parametrize("ldx,ox,ldw,ow,lddx,odx,lddw,odw", [
    (72, 0, 80, 0, 72, 0, 72, 0), (73, 1, 79, 3, 75, 1, 77, 1), (100, 3, 72, 1, 99, 0, 88, 8), (64, 0, 64, 0, 66, 2, 65, 0)])
def test_row_distances_and_alignment(pkg, dtype, K, ldx, ox, ldw, ow, lddx, odx, lddw, odw):
    N, H, V = 150, 64, 200
    c = make(5, dtype, N, H, V, K, pad=0.1)
    ref = reference(c)
    c["x"], _ = strided(c["x"], ldx, ox)
    c["w"], _ = strided(c["w"], ldw, ow)
    dx, bx = strided(torch.zeros_like(c["x"]).contiguous(), lddx, odx, fill=7.0)
    dw, bw = strided(torch.zeros_like(c["w"]).contiguous(), lddw, odw, fill=7.0)
    verify(call(pkg, c, dx=dx, dw=dw), ref)
    for buf, v, ld, o in ((bx, dx, lddx, odx), (bw, dw, lddw, odw)):      # what lies between and behind the rows is left as it was
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[o: o + v.shape[0] * ld].view(v.shape[0], ld)[:, : v.shape[1]] = False
        assert bool((buf[rest] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_for_all(pkg, dtype):
    """Row distance 0: the same activations against many labels, and the same weights for every output."""
    c = make(9, dtype, 40, 64, 90, pad=0.1)
    one = torch.randn(1, 64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(DT[dtype])
    c["x"] = one.expand(40, 64)
    verify(call(pkg, c), reference(c))
    c["w"] = one.expand(90, 64)
    dw = torch.empty(90, 64, dtype=DT[dtype], device=DEV)
    verify(call(pkg, c, dw=dw), reference(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_outputs(pkg, dtype):
    """-inf, and the type's lowest value, in the bias: such outputs have probability zero."""
    c = make(21, dtype, 140, 64, 700, pad=0.1)
    c["b"][::3] = -math.inf
    c["b"][300:600] = -math.inf                # a whole tile of 128 columns and more
    c["b"][1::3] = torch.finfo(torch.float32).min
    c["t"] = torch.where(c["t"] < 0, c["t"], (c["t"] % 33) * 3 + 2)
    verify(call(pkg, c), reference(c))
    c["t"][5] = 0                              # a target that is masked
    got = call(pkg, c, grad=False)
    assert math.isinf(float(got["loss"][5])) and float(got["loss"][5]) > 0
    assert bool(torch.isfinite(got["loss"][6:]).all())


@pytest.mark.parametrize("N", [70, 400])
def test_full_lists_of_low_labels(pkg, N):
    """256 entries that all lie in the first few outputs (and some lists that end at an output's group of 32), no entry behind."""
    c = make(23, "bf16", N, 64, 700, 256, pad=0.0, full=True)
    c["ids"] = (c["ids"] % 20).contiguous()
    c["ids"][3] = 31
    c["ids"][4] = 32
    c["ids"][5] = 699
    c["ids"][6, :128], c["ids"][6, 128:] = 255, 256
    verify(call(pkg, c), reference(c))


@pytest.mark.parametrize("K", [2, 31, 32, 34, 63, 64, 65, 127, 128, 129, 255])
def test_lengths_of_lists(pkg, K):
    """Lists around the lengths at which a lane takes more entries, few labels (many entries of one label) and many."""
    for V in (17, 9000):
        for full in (False, True):
            c = make(40 + K, "f32", 37, 24, V, K, pad=0.1, full=full)
            verify(call(pkg, c), reference(c), (V, full))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 5])
def test_vectors_that_start_anywhere(pkg, dtype, K):
    """Everything but the matrices at addresses that are multiples of 4 bytes alone."""
    for N in (60, 700):
        c = make(24, dtype, N, 72, 333, K, pad=0.2)
        ref = reference(c)

        def shifted(t):
            buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
            v = buf[1:].view(t.shape)
            v.copy_(t)
            return v

        for k in ("t", "ids", "y", "dloss", "b"):
            if k in c:
                c[k] = shifted(c[k])
        ws = pkg.alloc_loss_workspace(c["w"], N, K, True)
        loss, lse, db = (shifted(torch.full((n,), math.nan, device=DEV)) for n in (N, N, 333))
        dx, dw = torch.empty(N, 72, dtype=DT[dtype], device=DEV), torch.empty(333, 72, dtype=DT[dtype], device=DEV)
        rows = (c["ids"], c["y"], c["tau"]) if K else (c["t"],)
        fwd, bwd = (pkg.wind_distill_loss, pkg.wind_distill_loss_grad) if K else (pkg.wind_label_loss, pkg.wind_label_loss_grad)
        fwd(c["x"], c["w"], c["b"], *rows, loss, lse, ws, check=True)
        bwd(c["x"], c["w"], c["b"], *rows, lse, c["dloss"], dx, dw, db, ws, check=True)
        verify(dict(loss=loss, lse=lse, dx=dx, dw=dw, db=db), ref)


def test_rows_far_apart(pkg):
    """Offsets that pass 32 bits: rows of x, W, dx and dW more than 2^31 bytes, then more than 2^31 elements, from the first."""
    ld = 1_100_000_000
    c = make(25, "bf16", 3, 64, 3, pad=0.0)
    ref = reference(c)
    out = {}
    for k in ("x", "w", "dx", "dw"):
        buf = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device=DEV)
        out[k] = buf.as_strided((3, 64), (ld, 1))
    for k in ("x", "w"):
        out[k].copy_(c[k])
        c[k] = out[k]
    verify(call(pkg, c, dx=out["dx"], dw=out["dw"]), ref)


def test_many_rows(pkg):
    """More than 2^31 values of g in one piece, and lists of more rows than a block counts."""
    for N, H, V, K in ((1_060_000, 8, 2100, 0), (70_001, 16, 70, 3)):
        c = make(26, "bf16", N, H, V, K, pad=0.1)
        verify_in_slices(call(pkg, c), c, 50_000)


def test_a_workspace_of_more_rows_serves_fewer(pkg):
    for dtype, K in (("bf16", 0), ("bf16", 6), ("f32", 0)):
        c = make(27, dtype, 3000, 136, 700, K)
        ws = pkg.alloc_loss_workspace(c["w"], 3000, K, True)
        for n in (3000, 1, 129, 2049, 300):
            d = {k: (v[:n] if k in ("x", "t", "ids", "y", "dloss") else v) for k, v in c.items()}
            verify(call(pkg, d, ws=ws), reference(d), n)


def test_without_bias_and_without_weights(pkg):
    c = make(31, "bf16", 100, 64, 300, bias=False)
    c["dloss"] = None
    verify(call(pkg, c), reference(c))


@pytest.mark.parametrize("want", [("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db"), ("dx", "dw")])
def test_some_of_the_gradients(pkg, want):
    for K in (0, 3):
        c = make(32, "bf16", 333, 136, 1100, K)
        ref = reference(c)
        verify(call(pkg, c, want=want), ref, want)


@pytest.mark.parametrize("dtype,N,H,V", [("bf16", 140001, 24, 4200), ("f32", 44001, 16, 2300)])
def test_several_pieces_of_the_outputs(pkg, dtype, N, H, V):
    c = make(41, dtype, N, H, V, pad=0.05)
    full = pkg.wind_loss_workspace_bytes(c["w"], N, 0, True)
    assert full < N * V * (6 if dtype == "f32" else 2)          # the gradient's share of logits is not kept whole
    verify_in_slices(call(pkg, c), c, 20000)


def test_gradient_against_differences(pkg):
    """Central differences of the loss itself: fp32, a direction per input."""
    for K in (0, 6):
        c = make(51, "f32", 20, 24, 50, K, pad=0.2)
        keep = reference(c)["keep"]
        c["x"] = torch.where(keep[:, None], c["x"], torch.zeros_like(c["x"]))
        got = call(pkg, c)
        g = torch.Generator(device=DEV).manual_seed(2)
        for k, dk in (("x", "dx"), ("w", "dw"), ("b", "db")):
            v = torch.randn(c[k].shape, generator=g, device=DEV)
            h = 2.0 ** -7
            f = [call(pkg, {**c, k: c[k] + sgn * h * v}, grad=False)["loss"].double() @ c["dloss"].double() for sgn in (1, -1)]
            slope, want = float(f[0] - f[1]) / (2 * h), float((got[dk].double() * v.double()).sum())
            # third derivatives are at most about |v|^3 ~ (sqrt(24) 2)^3 a row: h^2 / 6 of it; rounding of the losses: 20 rows x 2^-20 / h
            assert abs(slope - want) <= 20 * (h * h / 6 * 1000 + 2.0 ** -18 / h), (K, k, slope, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 9])
def test_same_bits_every_time(pkg, dtype, K):
    c = make(61, dtype, 700, 200, 1500, K)
    a, b = call(pkg, c), call(pkg, c)
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("K", [0, 4])
def test_labels_that_are_none(pkg, K):
    """An index outside the outputs: NaN in its row, an error status, nothing in the other rows."""
    for bad in (-2, 100, 2 ** 31 - 1, -2 ** 31):
        N = 200 if bad % 2 == 0 else 90
        c = make(71, "bf16", N, 64, 100, K, pad=0.1, full=True)
        ok = {k: (v.clone() if torch.is_tensor(v) else v) for k, v in c.items()}
        (c["ids"][13, 2:3] if K else c["t"][13:14]).fill_(bad)
        (ok["ids"][13] if K else ok["t"][13:14]).fill_(-1)          # as if the row were padding
        ref = reference(ok)
        ws = pkg.alloc_loss_workspace(c["w"], N, K, True)
        got = call(pkg, c, ws=ws, check=False)
        with pytest.raises(pkg.WindError) as e:
            pkg.wind_loss_status(ws)
        assert e.value.status == pkg.binding.WIND_ERR_INVALID_ARG
        for k in ("loss", "lse", "dx"):
            assert bool(torch.isnan(got[k][13]).all()), k
            got[k][13] = 0
        verify(got, ref)
        call(pkg, ok, ws=ws)                                        # the next call starts afresh (and checks its status)


def test_no_rows(pkg):
    c = make(81, "bf16", 4, 64, 50, 3)
    for d in (dict(c), {**make(81, "f32", 4, 64, 50)}):
        for k in ("x", "t", "ids", "y", "dloss"):
            if k in d:
                d[k] = d[k][:0]
        got = call(pkg, d)
        assert bool((got["dw"] == 0).all()) and bool((got["db"] == 0).all())


def test_captured_and_replayed(pkg):
    """Forward and gradient of both losses in one graph, replayed on new inputs; two graphs share a workspace."""
    made = {K: [make(90 + i, "bf16", 333, 128, 600, K) for i in range(2)] for K in (0, 5)}
    ws = pkg.alloc_loss_workspace(made[0][0]["w"], 333, 5, True)
    graphs = []
    for K in (0, 5):
        c = {k: (v.clone() if torch.is_tensor(v) else v) for k, v in made[K][0].items()}
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call(pkg, c, ws=ws)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call(pkg, c, ws=ws, check=False)
        graphs.append((K, c, g, out))
    for i in (1, 0):
        for K, c, g, out in graphs:
            for k, v in made[K][i].items():
                if torch.is_tensor(v):
                    c[k].copy_(v)
            for v in out.values():
                v.fill_(math.nan)
            g.replay()
        torch.cuda.synchronize()
        for K, c, g, out in graphs:
            verify(out, reference(made[K][i]), (K, i))


def test_streams_and_threads(pkg):
    """Two streams at once, each call with its own workspace, from two host threads."""
    import threading
    cases = [make(100 + i, "bf16" if i % 2 else "f32", 500, 128, 900, 7 * (i % 2)) for i in range(4)]
    refs = [reference(c) for c in cases]
    torch.cuda.synchronize()
    out = [None] * 4

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(3):
                out[i] = call(pkg, cases[i], check=True)
        s.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(4):
        verify(out[i], refs[i], i)


def test_arguments_are_checked(pkg):
    c = make(111, "bf16", 20, 64, 50)
    ws = pkg.alloc_loss_workspace(c["w"], 20, 3, True)
    v = torch.empty(20, device=DEV)
    ok = dict(x=c["x"], weight=c["w"], bias=c["b"], target=c["t"], loss=v, lse=v.clone(), workspace=ws)
    pkg.wind_label_loss(**ok, check=True)
    for k, bad in (("x", c["x"].float()), ("x", c["x"][:, :32]), ("x", c["x"].t().contiguous().t()), ("x", c["x"].cpu()), ("target", c["t"].long()),
                   ("target", c["t"][:5]), ("loss", v.double()), ("loss", v[:3]), ("lse", v.cpu()), ("bias", c["b"].bfloat16()), ("bias", c["b"][:7]),
                   ("weight", c["w"].half()), ("weight", c["w"][0]), ("workspace", ws.cpu()), ("workspace", ws.int()), ("target", None), ("loss", None)):
        with pytest.raises(ValueError):
            pkg.wind_label_loss(**{**ok, k: bad})
    with pytest.raises(pkg.WindError) as e:
        pkg.wind_label_loss(**{**ok, "workspace": ws[:4096]})
    assert e.value.status == pkg.binding.WIND_ERR_WORKSPACE
    d = make(112, "bf16", 20, 64, 50, 3)
    good = dict(x=d["x"], weight=d["w"], bias=None, ids=d["ids"], teacher=d["y"], tau=1.0, loss=v, lse=v.clone(), workspace=ws)
    pkg.wind_distill_loss(**good, check=True)
    for k, bad in (("ids", d["ids"].long()), ("ids", d["ids"][:, 0]), ("teacher", d["y"][:, :2]), ("teacher", d["y"].double()), ("ids", d["ids"].t())):
        with pytest.raises(ValueError):
            pkg.wind_distill_loss(**{**good, k: bad})
    for tau in (0.0, -2.0, math.inf, math.nan):
        with pytest.raises(pkg.WindError):
            pkg.wind_distill_loss(**{**good, "tau": tau})
    with pytest.raises(pkg.WindError):
        many = torch.zeros(20, 300, dtype=torch.int32, device=DEV)
        pkg.wind_distill_loss(**{**good, "ids": many, "teacher": many.float()})


def test_beside_the_decoder(pkg):
    """The losses of a model's own joint: its logits by wind_eval_joint_window, a teacher's best labels from another model's."""
    from naive_model import NaiveModel, random_weights
    r = np.random.default_rng(4)
    student = random_weights(r, 32, 24, 40, 1, 48, 60, act=1, bias_scale=0.1)
    teacher = random_weights(r, 32, 64, 64, 2, 96, 60, act=0, bias_scale=0.1)
    B, T, W = 6, 20, 5
    enc = r.standard_normal((B, T, 32)).astype(np.float32)
    lens = torch.full((B,), T, dtype=torch.int32, device=DEV)
    t0 = torch.from_numpy(r.integers(0, T - W, B).astype(np.int32)).to(DEV)
    prefix = torch.from_numpy(r.integers(0, 60, (B, 3)).astype(np.int32)).to(DEV)
    plen = torch.from_numpy(r.integers(0, 4, B).astype(np.int32)).to(DEV)
    logits = {}
    for name, weights in (("student", student), ("teacher", teacher)):
        m = pkg.WindModel(weights)
        logits[name] = torch.empty(B, W, 61, device=DEV)
        pkg.wind_eval_joint_window(m, pkg.to_device_enc(m, enc), lens, W, prefix, plen, t0, logits[name], pkg.alloc_workspace(m, B, T, W))
    nm = NaiveModel(student)
    x = np.zeros((B, W, 48))
    for b in range(B):
        h = nm.decoder(prefix[b, : int(plen[b])].tolist())[0]
        for i in range(W):
            e = nm.w_enc @ torch.tensor(enc[b, int(t0[b]) + i], dtype=torch.float64) + nm.b_enc
            x[b, i] = torch.tanh(e + nm.w_pred @ h + nm.b_pred).numpy()
    top = torch.topk(logits["teacher"].reshape(B * W, 61), 8)
    c = dict(x=torch.from_numpy(x.reshape(B * W, 48)).float().to(DEV), w=torch.from_numpy(student["w_out"]).to(DEV),
             b=torch.from_numpy(student["b_out"]).to(DEV), dloss=None, tau=2.0, ids=top.indices.int().contiguous(), y=top.values.contiguous())
    logp = torch.log_softmax(logits["student"].reshape(B * W, 61).double(), 1)
    labels = {**c, "t": top.indices[:, 0].int().contiguous(), "tau": 1.0}
    del labels["ids"], labels["y"]
    got = call(pkg, labels)
    want = -logp.gather(1, top.indices[:, :1])[:, 0]
    assert float((got["loss"].double() - want).abs().max()) <= 2e-4          # twice the bound of a logit on the fp32 path
    verify(got, reference(labels))
    got = call(pkg, c)
    logp2 = torch.log_softmax(logits["student"].reshape(B * W, 61).double() / 2, 1)
    q = torch.softmax(top.values.double() / 2, 1)
    want = 4 * (q * (q.log() - logp2.gather(1, top.indices))).sum(1)
    assert float((got["loss"].double() - want).abs().max()) <= 4 * 2e-4
    verify(got, reference(c))
