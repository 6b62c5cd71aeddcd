"""Timed cases of the way out of a model: losses on the output head that keep no logits, and learning from a teacher.

A case is one pass through one of them:

  distill       divergence of logits from a teacher of whom the top logits of every token are known, with its gradient
  head_loss     cross-entropy of the logits X W^T against labels, with the gradients of tokens and head; the logits are not kept
  head_distill  the divergence of `distill` on the logits X W^T, with the gradients of tokens and head

Plain forms: elementary torch operations in fp32, rounded once.  With `own` the calls of the package.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # A unit-sized student: launches and latency.
        dict(name="distill_f32_small", op="distill", dtype="f32", T=256, V=1024, k=8, tau=1.0, rest=False, pad=0.0, cut=False),
        # A student of the paper's vocabulary on the benchmark's batch of 8192 tokens, 64 logits a token kept from the teacher, softened.
        dict(name="distill_bf16_32K", op="distill", dtype="bf16", T=8192, V=32000, k=64, tau=2.0, rest=False, pad=0.0, cut=False),
        # An odd vocabulary, a quarter of the tokens without a teacher (prompts, padding), as many logits a token as made up most of the
        # teacher's mass, the rest known by its log-sum.
        dict(name="distill_bf16_ragged", op="distill", dtype="bf16", T=1000, V=50001, k=20, tau=1.0, rest=True, pad=0.25, cut=True),
        # A unit-sized model's head.
        dict(name="head_loss_f32_small", op="head_loss", dtype="f32", T=256, V=1024, d=256, pad=0.0, dx=True, dw=True),
        # A full-precision run of odd sizes, as a bf16 one is compared with.
        dict(name="head_loss_f32_ragged", op="head_loss", dtype="f32", T=1023, V=5003, d=511, pad=0.0, dx=True, dw=True),
        # The last few labelled tokens of a sequence, a batch of one: the head is read and its gradient written, little else.
        dict(name="head_loss_bf16_few", op="head_loss", dtype="bf16", T=16, V=32000, d=2048, pad=0.0, dx=True, dw=True),
        # Evaluation at the paper's 500M width, four sequences of its length: the loss alone.
        dict(name="head_loss_bf16_eval", op="head_loss", dtype="bf16", T=4096, V=32000, d=1200, pad=0.0, dx=False, dw=False),
        # The head of the benchmark's 1B-like model on one worker's batch.
        dict(name="head_loss_bf16_1B", op="head_loss", dtype="bf16", T=16384, V=32000, d=2048, pad=0.0, dx=True, dw=True),
        # The paper's 1B width on a padded batch over an odd, larger vocabulary: a third of the tokens have no label.
        dict(name="head_loss_bf16_padded", op="head_loss", dtype="bf16", T=5000, V=50001, d=1600, pad=0.33, dx=True, dw=True),
        # A unit-sized student's head.
        dict(name="head_distill_f32_small", op="head_distill", dtype="f32", T=256, V=1024, d=256, k=8, tau=1.0, rest=False, pad=0.0, cut=False,
             dx=True, dw=True),
        # The 1B-like student's head on 8192 tokens, 64 logits a token from the teacher.
        dict(name="head_distill_bf16_1B", op="head_distill", dtype="bf16", T=8192, V=32000, d=2048, k=64, tau=2.0, rest=False, pad=0.0, cut=False,
             dx=True, dw=True),
        # A student whose head stays as it is (tied to a frozen embedding), on a padded batch at the paper's 500M width.
        dict(name="head_distill_bf16_frozen", op="head_distill", dtype="bf16", T=3000, V=50001, d=1200, k=20, tau=1.0, rest=True, pad=0.25, cut=True,
             dx=True, dw=False),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over the logarithm of the range."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["distill", "head_loss", "head_distill"])
    f32 = rng.random() < 0.25
    c = dict(op=op, dtype="f32" if f32 else "bf16")
    V = _log_int(rng, 256, 8192 if f32 and op != "distill" else 64000)
    T = _log_int(rng, 1, (2048 if op != "distill" else 4096) if f32 else 16384 if op != "distill" else 8192)
    pad = rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.9), 2)])
    if op == "distill":
        T = max(1, min(T, 8192 * 32000 // (V * (2 if f32 else 1))))
    else:
        d = _log_int(rng, 33, 512) if f32 else _log_int(rng, 64, 2048) // 8 * 8
        T = max(1, min(T, 16384 * 32000 * 2048 // (V * d)))
        c.update(d=d, **rng.choice([dict(dx=True, dw=True), dict(dx=True, dw=True), dict(dx=True, dw=False), dict(dx=False, dw=False)]))
    c.update(T=T, V=V, pad=pad)
    if op != "head_loss":
        c.update(k=_log_int(rng, 1, 128), tau=rng.choice([1.0, 1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)]), rest=rng.random() < 0.5, cut=rng.random() < 0.3)
    return c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, T, V, op = _DT[case["dtype"]], case["T"], case["V"], case["op"]

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = dict(case=case)
    perm = torch.randperm(V, generator=g, device="cuda")
    none = uniform(T) < case["pad"]
    if op == "head_loss":
        # frequencies fall about as 1 / rank, ranks lie anywhere in the vocabulary
        tops = perm[(V ** uniform(T)).long().clamp_(1, V) - 1][:, None]
        s["labels"] = torch.where(none, -100, tops[:, 0])
        live = ~none
    else:
        k = case["k"]
        # a teacher's top logits, the highest first, of different tokens of the vocabulary (k <= 128 < V)
        place = torch.arange(k, device="cuda")
        tops = perm[((V ** uniform(T)).long()[:, None] - 1 + place) % V]
        v = 14.0 + normal(T, 1) - 1.5 * torch.log1p(place.float()) - 0.05 * uniform(T, 1).float() * place
        kept = place < (torch.floor(uniform(T, 1) * k) + 1 if case["cut"] else k)
        s["ids"] = torch.where(kept & ~none[:, None], tops, -1).to(torch.int32)
        s["top"] = v.to(dt)
        z = torch.where(kept, s["top"].double() / case["tau"], -math.inf)
        s["top_lse"] = (torch.logsumexp(z, 1) + 0.02 + 0.3 * uniform(T)).float() if case["rest"] else None
        live = ~none
    s["scale"] = 1.0 / max(1, int(live.sum()))
    f32 = dict(dtype=torch.float32)
    if op == "distill":
        Z = normal(T, V, std=2.0)
        Z.scatter_add_(1, tops, 0.8 * v)  # a student that has learned some
        s["Z"] = Z.to(dt)
        s["out"] = (empty(T, **f32), empty(T, **f32), empty(T, V), empty(1, **f32))
    else:
        d = case["d"]
        s["W"] = normal(V, d, std=2.0 / math.sqrt(d)).to(dt)
        s["X"] = (normal(T, d) + 2.5 * s["W"][tops[:, 0]].float()).to(dt)  # hidden states that point to their token
        s["out"] = (empty(T, **f32), empty(T, **f32), empty(T, d) if case["dx"] else None, empty(V, d) if case["dw"] else None, empty(1, **f32))
    return s


def _run_own(s):
    import paper_2507_09029_amd as sdp

    c = s["case"]
    if c["op"] == "distill":
        return sdp.distill_loss(s["Z"], s["ids"], s["top"], temperature=c["tau"], top_lse=s["top_lse"], scale=s["scale"], out=s["out"])
    want = dict(want_dx=c["dx"], want_dw=c["dw"])
    if c["op"] == "head_loss":
        if "ws" not in s:  # kept by the program from its first step on
            s["ws"] = torch.empty(sdp.head_loss_workspace_bytes(s["X"].dtype, c["T"], c["V"], c["d"], **want), dtype=torch.uint8, device="cuda")
        return sdp.head_loss(s["X"], s["W"], s["labels"], scale=s["scale"], out=s["out"], ws=s["ws"], **want)
    if "ws" not in s:
        s["ws"] = torch.empty(sdp.head_distill_workspace_bytes(s["X"].dtype, c["T"], c["V"], c["d"], c["k"], **want), dtype=torch.uint8, device="cuda")
    return sdp.head_distill(s["X"], s["W"], s["ids"], s["top"], temperature=c["tau"], top_lse=s["top_lse"], scale=s["scale"], out=s["out"],
                            ws=s["ws"], **want)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    z = s["Z"].float() if c["op"] == "distill" else s["X"].float() @ s["W"].float().T
    if c["op"] == "head_loss":
        at, tau = s["labels"][:, None], 1.0
        q = ((at >= 0) & (at < c["V"])).float()
        at, log_q = torch.where(q > 0, at, 0), torch.zeros_like(q)
    else:
        tau, at = c["tau"], s["ids"].long()
        there = (at >= 0) & (at < c["V"])
        at = torch.where(there, at, 0)
        v = torch.where(there, s["top"].float() / tau, -math.inf)
        some = there.any(1, keepdim=True)
        if s["top_lse"] is None:
            top = torch.where(some, v.max(1, keepdim=True).values, 0.0)
            total = torch.where(some, top + (v - top).exp().sum(1, keepdim=True).log(), 0.0)
        else:
            total = s["top_lse"][:, None]
        log_q = torch.where(there, v - total, 0.0)
        q = torch.where(there, log_q.exp(), 0.0)
    mass = q.sum(1, keepdim=True)
    some = mass > 0
    z = z / tau
    m = z.max(1, keepdim=True).values
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lse = torch.where(some, m + total.log(), 0.0)[:, 0]
    per_token = (q * (log_q + (m - z.gather(1, at)) + total.log())).sum(1)
    dz = e * (mass / total)
    dz.scatter_add_(1, at, -q)
    dz *= s["scale"] / tau
    loss = (per_token.double().sum() * s["scale"]).float()[None]
    if c["op"] == "distill":
        return per_token, lse, dz.to(s["Z"].dtype), loss
    dx = (dz @ s["W"].float()).to(s["X"].dtype) if c["dx"] else None
    dw = (dz.T @ s["X"].float()).to(s["X"].dtype) if c["dw"] else None
    return per_token, lse, dx, dw, loss


def exact(case, seed):
    s = prepare(case, seed)
    T, V, op = case["T"], case["V"], case["op"]
    ids = s["labels"].unsqueeze(1) if op == "head_loss" else s["ids"].long()
    rows = torch.nonzero((ids >= 0).any(1)).squeeze(1)  # the tokens that have something to learn from
    ids, n = ids[rows], len(rows)
    there = ids >= 0
    tau = case.get("tau", 1.0)
    target = torch.zeros((n, V + 1), dtype=torch.float64, device="cuda")  # column V takes what is no entry
    column = torch.where(there, ids, V)
    if op == "head_loss":
        target.scatter_(1, column, 1.0)
        entropy = torch.zeros(n, dtype=torch.float64, device="cuda")
    else:
        a = (s["top"][rows].double() / tau).masked_fill(~there, -math.inf)
        log_q = torch.log_softmax(a, 1) if s["top_lse"] is None else a - s["top_lse"][rows].double().unsqueeze(1)
        entropy = torch.special.entr(log_q.exp()).sum(1)
        target.scatter_(1, column, log_q.exp())
    target = target[:, :V]
    if op == "distill":
        logits = s["Z"][rows].double().div_(tau)
    else:
        X, W = s["X"][rows].double(), s["W"].double()
        logits = torch.mm(X, W.t()).div_(tau)
    log_p = torch.log_softmax(logits, 1)
    kl, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    lse[rows] = torch.logsumexp(logits, 1)
    kl[rows] = torch.linalg.vecdot(target, -log_p) - entropy
    mass = target.sum(1, keepdim=True)
    d_logits = log_p.exp_().mul_(mass).sub_(target).mul_(s["scale"] / tau)
    loss = kl.sum().reshape(1) * s["scale"]
    if op == "distill":
        dZ = torch.zeros((T, V), dtype=torch.float64, device="cuda")
        dZ[rows] = d_logits
        return kl, lse, dZ, loss
    dX = dW = None
    if case["dx"]:
        dX = torch.zeros((T, case["d"]), dtype=torch.float64, device="cuda")
        dX[rows] = torch.mm(d_logits, W)
    if case["dw"]:
        dW = torch.mm(d_logits.t(), X)
    return kl, lse, dX, dW, loss


def work(case):
    T, V, e = case["T"], case["V"], 4 if case["dtype"] == "f32" else 2
    live = T * (1.0 - case["pad"])
    if case["op"] == "head_loss":
        small = 8 * T + 8 * T
    else:
        small = T * case["k"] * 4 + live * case["k"] * (0.5 if case["cut"] else 1.0) * e + (4 * T if case["rest"] else 0) + 8 * T
    if case["op"] == "distill":
        return {"bytes": live * V * e + T * V * e + small, "flops": 8 * live * V}
    d, products = case["d"], 1 + case["dx"] + case["dw"]
    return {"bytes": live * d * e + V * d * e + (T * d * e if case["dx"] else 0) + (V * d * e if case["dw"] else 0) + small,
            "flops": 2 * live * V * d * products + 8 * live * V}
