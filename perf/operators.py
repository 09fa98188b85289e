"""Cases of the operators that train and score the joint network's output layer.

Decoding evaluates the output layer z = W x + b (W [n_out, H], n_out labels with the blank among them) for its argmax;
scoring a transcript, training the layer or distilling a small model from a large one asks for a softmax over the same
logits, at every node of a lattice or every frame of an alignment.  A case is one pass through one of two operators:

  op    "label"    loss_r = logsumexp_v z_rv - z_r,t(r), for a row's label t(r); -1 marks padding (loss and gradient zero)
        "distill"  loss_r = tau^2 sum_k q_rk (ln q_rk - ln p_r,i(r,k)), q_r = softmax_k(y_rk / tau) over the teacher's best
                   labels i(r, k), p_r = softmax_v(z_rv / tau); label -1 marks an entry that the teacher does not have, a
                   row without any has no loss and no gradient
  grad  False: the losses and log-sum-exps; True: these, and then the gradients of sum_r s_r loss_r with regard to x, W and b
        (a training step's share of this layer), s_r being given

N rows, H activations, V outputs, K teacher's entries (0 for "label"), pad: share of the rows that are padding.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def case(name, op, grad, dtype, N, H, V, K=0, tau=1.0, pad=0.0, bias=True):
    c = dict(op=op, grad=grad, dtype=dtype, N=N, H=H, V=V, K=K, tau=tau, pad=pad, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the score of one label of a hypothesis, large vocabulary: latency, and one pass over W
        case("label_one_row", "label", False, "bf16", 1, 1024, 8193),
        # a training step of the smallest model, fp32: launches
        case("label_tiny_f32_step", "label", True, "f32", 100, 64, 33, pad=0.1),
        # the score of an alignment of a 100 s recording (1250 frames)
        case("label_score_1250", "label", False, "bf16", 1250, 640, 1025),
        # a step over the lattice nodes of a padded batch; the blank and 1024 labels
        case("label_lattice_step", "label", True, "bf16", 20011, 640, 1025, pad=0.35),
        # the same layer of an fp32 checkpoint
        case("label_f32_step", "label", True, "f32", 1999, 640, 1025, pad=0.1),
        # a step of the large-vocabulary model
        case("label_bigvocab_step", "label", True, "bf16", 8003, 1024, 8193, pad=0.1),
        # a step of a text model's output layer, 65 thousand labels
        case("label_text_step", "label", True, "bf16", 4096, 2048, 65536, bias=False),
        # one short utterance's distillation loss, the teacher's eight best
        case("distill_short", "distill", False, "bf16", 7, 640, 1025, K=8, tau=2.0),
        # a distillation step of the large model from one like it, sixteen labels
        case("distill_lattice_step", "distill", True, "bf16", 6007, 640, 1025, K=16, tau=2.0, pad=0.25),
        # held-out distillation loss of an fp32 checkpoint with the large vocabulary
        case("distill_f32_bigvocab", "distill", False, "f32", 777, 1024, 8193, K=32, tau=1.0, pad=0.1),
        # a distillation step with the large vocabulary, 64 labels
        case("distill_bigvocab_step", "distill", True, "bf16", 4001, 1024, 8193, K=64, tau=4.0, pad=0.1),
        # distilling a text model's output layer
        case("distill_text_step", "distill", True, "bf16", 2048, 2048, 32000, K=64, tau=1.0, bias=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["label", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    grad = rng.random() < 0.6
    H = log_int(32, 2048)
    if rng.random() < 0.6:
        H = -(-H // 32) * 32
    V = log_int(33, 65536)
    most = 4096 * 2048 * 65536
    N = log_int(1, max(1, min(20000, most // (H * V))))
    K = min(V, log_int(1, 128)) if op == "distill" else 0
    tau = rng.choice([1.0, 2.0, 4.0]) if op == "distill" else 1.0
    return case("", op, grad, dtype, N, H, V, K, tau, round(rng.choice([0.0, 0.1, rng.uniform(0.0, 0.6)]), 3), rng.random() < 0.7)


def prepare(c, seed):
    """Inputs like a partly trained model's: unit activations, logits of standard deviation two, the right label ahead."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    N, H, V, K, dt = c["N"], c["H"], c["V"], c["K"], DTYPES[c["dtype"]]
    w = (torch.randn(V, H, generator=g, device="cuda") * (2.0 / math.sqrt(H))).to(dt)
    b = torch.randn(V, generator=g, device="cuda") if c["bias"] else None
    label = torch.randint(0, V, (N,), generator=g, device="cuda")
    x = torch.randn(N, H, generator=g, device="cuda")
    x = (x + w[label].float() * (1.5 * torch.rand(N, 1, generator=g, device="cuda") + 0.25)).to(dt)
    padding = torch.rand(N, generator=g, device="cuda") < c["pad"]
    scale = (0.5 + torch.rand(N, generator=g, device="cuda")) / max(1, int((~padding).sum()))
    s = dict(op=c["op"], grad=c["grad"], tau=c["tau"], x=x, w=w, b=b, scale=scale)
    if K:
        ids = torch.randint(0, V, (N, K), generator=g, device="cuda")
        first = torch.randint(0, V, (N, 1), generator=g, device="cuda")
        stride = max(1, V // K)
        # distinct labels: one in each of K stretches of the vocabulary, in an order of its own
        order = torch.rand(N, K, generator=g, device="cuda").argsort(1)
        ids = (order * stride + ids % stride + first) % V
        ids[:, 0] = torch.where((ids == label[:, None]).any(1), ids[:, 0], label)
        y = torch.randn(N, K, generator=g, device="cuda").mul_(2.0).sort(1, descending=True).values
        y[:, 0] += 3.0
        short = torch.randint(1, 2 * K + 1, (N, 1), generator=g, device="cuda")   # half the lists are not full
        gone = (torch.arange(K, device="cuda")[None] >= short) | padding[:, None]
        s["ids"] = torch.where(gone, -1, ids).int().contiguous()
        s["y"] = torch.where(gone, -math.inf, y).contiguous()
    else:
        s["label"] = torch.where(padding, -1, label).int()
    # the buffers that a training program keeps
    s["loss"], s["lse"] = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    if c["grad"]:
        s["dx"], s["dw"] = torch.empty_like(x), torch.empty_like(w)
        s["db"] = torch.empty(V, device="cuda") if c["bias"] else None
    if own:
        import paper_2505_13765_b200 as wind
        s["ws"] = wind.alloc_loss_workspace(w, N, K, c["grad"])
    return s


def run_own(s):
    import paper_2505_13765_b200 as wind
    layer = (s["x"], s["w"], s["b"])
    if s["op"] == "label":
        wind.wind_label_loss(*layer, s["label"], s["loss"], s["lse"], s["ws"])
        if s["grad"]:
            wind.wind_label_loss_grad(*layer, s["label"], s["lse"], s["scale"], s["dx"], s["dw"], s["db"], s["ws"])
    else:
        wind.wind_distill_loss(*layer, s["ids"], s["y"], s["tau"], s["loss"], s["lse"], s["ws"])
        if s["grad"]:
            wind.wind_distill_loss_grad(*layer, s["ids"], s["y"], s["tau"], s["lse"], s["scale"], s["dx"], s["dw"], s["db"], s["ws"])
    out = dict(loss=s["loss"], lse=s["lse"])
    return dict(out, dx=s["dx"], dw=s["dw"], db=s["db"]) if s["grad"] else out


def run_plain(s):
    x, w, tau = s["x"].float(), s["w"].float(), s["tau"]
    z = x @ w.t()
    if s["b"] is not None:
        z += s["b"]
    z /= tau
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + torch.exp(z - top).sum(1).log()
    if s["op"] == "label":
        valid = s["label"] >= 0
        at = s["label"].clamp(min=0).long()[:, None]
        q = valid.float()[:, None]
        loss = lse - z.gather(1, at)[:, 0]
    else:
        there = s["ids"] >= 0
        valid = there.any(1)
        at = s["ids"].clamp(min=0).long()
        y = torch.where(there, s["y"], -math.inf) / tau
        y = torch.where(valid[:, None], y, torch.zeros_like(y))
        e = torch.exp(y - y.amax(1, keepdim=True))
        q = torch.where(there, e / e.sum(1, keepdim=True), torch.zeros_like(e))
        lnq = torch.where(q > 0, q, torch.ones_like(q)).log()
        loss = tau * tau * (q * (lnq - z.gather(1, at) + lse[:, None])).sum(1)
    zero = torch.zeros_like(loss)
    out = dict(loss=torch.where(valid, loss, zero), lse=torch.where(valid, lse, zero))
    if not s["grad"]:
        return out
    scale = torch.where(valid, s["scale"] * tau, zero)[:, None]
    d = torch.exp(z.sub_(lse[:, None])).mul_(scale)
    d.scatter_add_(1, at, -scale * q)
    return dict(out, dx=(d @ w).to(s["x"].dtype), dw=(d.t() @ x).to(s["w"].dtype), db=d.sum(0) if s["b"] is not None else None)


def run(s):
    return run_own(s) if own else run_plain(s)


def work(c):
    n = c["N"] * (1.0 - c["pad"])                  # rows of padding cost nothing but their mark
    N, H, V, K = c["N"], c["H"], c["V"], c["K"]
    e = 4 if c["dtype"] == "f32" else 2
    bytes_ = n * H * e + V * H * e + (4 * V if c["bias"] else 0) + (8.0 * N * K if K else 4.0 * N) + 8.0 * N
    flops = 2.0 * n * H * V
    if c["grad"]:                                  # the logits again, and two products of the same size
        bytes_ += 4.0 * N + N * H * e + V * H * e + (4 * V if c["bias"] else 0)
        flops *= 4.0
    return {"bytes": bytes_, "flops": flops}


def exact(c, seed):
    """The same from the definitions in 64 bits, 1024 rows at a time."""
    s = prepare(c, seed)
    N, V, tau = c["N"], c["V"], c["tau"]
    w = s["w"].double()
    b = torch.zeros(V, dtype=torch.float64, device="cuda") if s["b"] is None else s["b"].double()
    loss, lse = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
    dx, dw, db = torch.zeros_like(s["x"], dtype=torch.float64), torch.zeros_like(w), torch.zeros_like(b)
    for r0 in range(0, N, 1024):
        rows = slice(r0, min(N, r0 + 1024))
        x = s["x"][rows].double()
        target = torch.zeros(x.shape[0], V, dtype=torch.float64, device="cuda")   # the distribution aimed at
        r = torch.arange(x.shape[0], device="cuda")
        if c["op"] == "label":
            t = s["label"][rows].long()
            keep = t != -1
            target[r[keep], t[keep]] = 1.0
        else:
            i, y = s["ids"][rows].long(), s["y"][rows].double() / tau
            keep = (i != -1).any(1)
            n_of = (i != -1).nonzero()
            logq = y - torch.logsumexp(y.masked_fill(i == -1, -math.inf), 1, keepdim=True)
            target.index_put_((n_of[:, 0], i[i != -1]), logq[i != -1].exp(), accumulate=True)
        logp = torch.log_softmax(torch.addmm(b, x, w.T) / tau, 1)
        entropy = torch.special.xlogy(target, target).sum(1)
        loss[rows] = tau ** 2 * (entropy - (target * logp).sum(1)) * keep
        lse[rows] = (((x * w[0]).sum(1) + b[0]) / tau - logp[:, 0]) * keep
        if c["grad"]:
            e = (logp.exp() - target) * (s["scale"][rows].double() * tau * keep)[:, None]
            dx[rows] = e.mm(w)
            dw.addmm_(e.T, x)
            db += e.sum(0)
        del target, logp
    out = dict(loss=loss, lse=lse)
    return dict(out, dx=dx, dw=dw, db=db if c["bias"] else None) if c["grad"] else out
