"""Cases of the vocabulary losses: softmax cross-entropy and distillation from a teacher's top logits over a large
output layer, their losses alone (evaluation) and with the gradients of hidden states and weights (training).

A case: op "xent" or "distill"; grad; type "bf16" or "f32"; n rows of d inputs, V classes; `empty` rows without a
target (padding of a batch); for distillation k entries per row, temperature T, whether the teacher's own log-sum-exp
is given (tail kept out of the sum); `weighted`: a weight per row instead of the mean over the rows with a target.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, grad, type_, n, d, V, empty=0, k=0, T=1.0, tail=False, weighted=False):
    c = dict(op=op, grad=grad, type=type_, n=n, d=d, V=V, empty=empty, k=k, T=T, tail=tail, weighted=weighted)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the output layer of the small image network: a worker's minibatch of 20 rows, 100 hidden units, 10 classes
        _case("xent_grad_f32_20x100x10", "xent", True, "f32", 20, 100, 10),
        # one new token scored against a vocabulary (evaluation of a prompt token by token)
        _case("xent_loss_bf16_1x2048x50001", "xent", False, "bf16", 1, 2048, 50001),
        # a short sequence, single-precision training, odd sizes, a few padded rows
        _case("xent_grad_f32_1001x768x16001", "xent", True, "f32", 1001, 768, 16001, empty=13),
        # a worker's small minibatch: the weights' reading and their gradient's writing are the work
        _case("xent_grad_bf16_64x2048x65536", "xent", True, "bf16", 64, 2048, 65536),
        # an ordinary training step
        _case("xent_grad_bf16_4096x2048x32000", "xent", True, "bf16", 4096, 2048, 32000, weighted=True),
        # a padded batch of documents: 40 % of the rows carry no target, rows and classes ragged
        _case("xent_grad_bf16_5000x1024x50001", "xent", True, "bf16", 5000, 1024, 50001, empty=2000),
        # perplexity of a long document
        _case("xent_loss_bf16_8192x4096x65536", "xent", False, "bf16", 8192, 4096, 65536),
        # the largest step
        _case("xent_grad_bf16_8192x4096x131072", "xent", True, "bf16", 8192, 4096, 131072),
        # a handful of rows of a small student
        _case("distill_grad_bf16_8x256x1000", "distill", True, "bf16", 8, 256, 1000, k=8, T=2.0),
        # single-precision student, teacher's own normaliser given
        _case("distill_grad_f32_500x512x8191", "distill", True, "f32", 500, 512, 8191, empty=7, k=20, T=1.5, tail=True),
        # an ordinary distillation step
        _case("distill_grad_bf16_4096x2048x65536", "distill", True, "bf16", 4096, 2048, 65536, empty=96, k=64, T=2.0),
        # how far a student is from its teacher on held-out text
        _case("distill_loss_bf16_2047x4096x100003", "distill", False, "bf16", 2047, 4096, 100003, k=100, T=1.0, tail=True, weighted=False),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op, grad = rng.choice(["xent", "distill"]), rng.random() < 0.7
        type_ = "f32" if rng.random() < 0.3 else "bf16"
        n, d, V = _log_uniform(rng, 1, 8192), _log_uniform(rng, 32, 4096), _log_uniform(rng, 10, 131072)
        if rng.random() < 0.7:                         # widths of hidden layers are mostly round
            d = max(32, d // 64 * 64)
        c = _case(None, op, grad, type_, n, d, V, empty=int(n * rng.choice([0, 0, 0.1, 0.5])),
                  weighted=grad and rng.random() < 0.3)
        if op == "distill":
            c.update(k=_log_uniform(rng, 1, min(V, 128)), T=rng.choice([1.0, 1.5, 2.0, 4.0]), tail=rng.random() < 0.4)
        if _cost(c) <= most * (0.02 if type_ == "f32" else 1.0):
            return c


def _cost(c):
    return (3 if c["grad"] else 1) * 2.0 * c["n"] * c["V"] * c["d"] + 1e3 * c["V"] * c["d"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, d, V, k = case["n"], case["d"], case["V"], case["k"]
    dt = _TYPES[case["type"]]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    w = (randn(V, d) * (2.0 / math.sqrt(d))).to(dt)
    labels = (V * rand(n) ** 3).long().clamp_(max=V - 1)                  # frequent words have low indices
    h = (randn(n, d) + 2.0 * w[labels].float()).to(dt)                    # a model that has learnt something: z_label is near 8
    gone = torch.randperm(n, generator=g, device="cuda")[:case["empty"]]  # the rows without a target
    s = dict(case=case, h=h, w=w, weight=None)
    if case["weighted"]:
        s["weight"] = (rand(n) + 0.5) / n
    if case["op"] == "xent":
        labels[gone] = -1
        s["labels"] = labels.int()
    else:
        # the teacher's k largest logits, first the word that the student leans to; some rows of the list are shorter
        step = (rand(n, 1) * (V // k)).long().clamp_(min=1)
        at = torch.arange(k, device="cuda")
        idx = (labels[:, None] + at * step) % V
        t = 10.0 - 1.5 * torch.log(1.0 + at) + 0.3 * randn(n, k)
        idx = torch.where((rand(n, 1) < 0.2) & (at >= (1 + k) // 2), -1, idx)
        idx[gone] = -1
        s["top_idx"], s["top_logits"] = idx.int(), t
        T = case["T"]
        s["teacher_lse"] = torch.logsumexp(t / T, 1) + 0.25 * rand(n) if case["tail"] else None
    if own:
        import paper_1805_10111_b200 as dq
        s["layer"] = dq.Vocab(h, w, k=k, grad=case["grad"])
        s["loss"], s["lse"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        if case["grad"]:
            s["grad_h"], s["grad_w"] = torch.empty_like(h), torch.empty_like(w)
    return s


def _run_own(s):
    import paper_1805_10111_b200 as dq
    c = s["case"]
    if c["op"] == "xent":
        if not c["grad"]:
            dq.ok(dq.dq_xent_loss(s["layer"], s["labels"], s["loss"], s["lse"]))
            return s["loss"], s["lse"]
        dq.ok(dq.dq_xent_grad(s["layer"], s["labels"], s["weight"], s["loss"], s["lse"], s["grad_h"], s["grad_w"]))
        return s["loss"], s["lse"], s["grad_h"], s["grad_w"]
    if not c["grad"]:
        dq.ok(dq.dq_distill_loss(s["layer"], s["top_idx"], s["top_logits"], s["teacher_lse"], c["T"], s["loss"], s["lse"]))
        return s["loss"], s["lse"]
    dq.ok(dq.dq_distill_grad(s["layer"], s["top_idx"], s["top_logits"], s["teacher_lse"], c["T"], s["weight"], s["loss"], s["lse"],
                             s["grad_h"], s["grad_w"]))
    return s["loss"], s["lse"], s["grad_h"], s["grad_w"]


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    T, V, dt = c["T"], c["V"], _TYPES[c["type"]]
    h, w = state["h"].float(), state["w"].float()
    z = h @ w.t()
    if T != 1.0:
        z /= T
    m = z.max(1, keepdim=True).values
    if c["op"] == "xent":
        idx = state["labels"].long()[:, None]
        there = (idx >= 0) & (idx < V)
        q = there.float()
        at = torch.where(there, idx, 0)
        row = there[:, 0]
        zt = z.gather(1, at)
        z.sub_(m).exp_()
        total = z.sum(1, keepdim=True)
        lse = (m + total.log())[:, 0]
        loss = lse - zt[:, 0]
    else:
        idx, t = state["top_idx"].long(), state["top_logits"] / T
        there = (idx >= 0) & (idx < V) & (t != -math.inf)
        at = torch.where(there, idx, 0)
        row = there.any(1)
        t = torch.where(there, t, -math.inf)
        if state["teacher_lse"] is None:
            top = torch.where(row, t.max(1).values, 0.0)[:, None]
            tl = top + (t - top).exp().sum(1, keepdim=True).log()
        else:
            tl = state["teacher_lse"][:, None]
        logq = torch.where(there, t - tl, 0.0)
        q = torch.where(there, logq.exp(), 0.0)
        zt = z.gather(1, at)
        z.sub_(m).exp_()
        total = z.sum(1, keepdim=True)
        lse = (m + total.log())[:, 0]
        loss = T * T * (q * (logq - (zt - lse[:, None]))).sum(1)
    loss, lse = torch.where(row, loss, 0.0), torch.where(row, lse, 0.0)
    if not c["grad"]:
        return loss, lse
    weight = state["weight"] if state["weight"] is not None else 1.0 / row.sum().clamp(min=1).float()
    weight = torch.where(row, weight * T, 0.0)[:, None]
    z *= q.sum(1, keepdim=True) / total                       # the softmax, times the mass that the targets carry
    z.scatter_add_(1, at, -q)
    z *= weight
    return loss, lse, (z @ w).to(dt), (z.t() @ h).to(dt)


def exact(case, seed):
    """The definition in 64 bits, a block of rows at a time."""
    s = prepare(case, seed)
    n, V, T = case["n"], case["V"], case["T"]
    W = s["w"].double()
    H = s["h"].double()
    loss, lse = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    gh, gw = torch.zeros_like(H), torch.zeros_like(W) if case["grad"] else None
    if case["op"] == "xent":
        idx = s["labels"].long().view(n, 1)
        logq = torch.zeros(n, 1, dtype=torch.float64, device="cuda")
    else:
        idx, t = s["top_idx"].long(), s["top_logits"].double() / T
        t = t.masked_fill((idx < 0) | (idx >= V), -math.inf)
        logq = t - (torch.logsumexp(t, 1) if s["teacher_lse"] is None else s["teacher_lse"].double())[:, None]
    idx = idx.masked_fill(idx >= V, -1)
    has = (idx >= 0).any(1)
    weight = s["weight"].double() if s["weight"] is not None else torch.full_like(loss, 1.0 / max(1, int(has.sum())))
    for r in has.nonzero()[:, 0].split(1024):
        logp = torch.log_softmax(H[r] @ W.t() / T, 1)
        i, lq = idx[r], logq[r]
        ok = i >= 0
        i = i.clamp(min=0)
        q = lq.exp().masked_fill(~ok, 0.0)
        loss[r] = T * T * torch.where(ok, q * (lq - logp.gather(1, i)), torch.zeros_like(q)).sum(1)
        lse[r] = (H[r] * W[i[:, 0]]).sum(1) / T - logp.gather(1, i[:, :1])[:, 0]
        if case["grad"]:
            g = logp.exp_().mul_(q.sum(1, keepdim=True)).scatter_add_(1, i, -q).mul_((weight[r] * T)[:, None])
            gh[r] = g @ W
            gw += g.t() @ H[r]
    return (loss, lse, gh, gw) if case["grad"] else (loss, lse)


def work(case):
    size = 4 if case["type"] == "f32" else 2
    n, d, V, rows = case["n"], case["d"], case["V"], case["n"] - case["empty"]
    moved = size * d * (rows + V) + (8 * n * case["k"] if case["op"] == "distill" else 4 * n) + 8 * n
    if case["grad"]:
        moved += size * d * (n + V)
    return {"bytes": moved, "flops": (6 if case["grad"] else 2) * rows * V * d}
