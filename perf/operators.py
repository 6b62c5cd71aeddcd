"""Timed cases of the operators around a stack of blocks: norms, the token embedding and the token loss.

A case is one pass through one of them:

  norm_fwd    layer or root-mean-square norm of tokens, alone or of the sum of a block half's output and its skip connection
  norm_bwd    its gradients: tokens (with the gradient that arrives over the skip connection), weight and bias
  embed_fwd   embedding rows of token ids, scaled
  embed_bwd   the embedding's gradient, all rows of it
  loss        cross-entropy of logits, mean over the tokens that have a label, with its gradient

Plain forms: elementary torch operations in fp32, rounded once.  With `own` the calls of the package.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


def listed():
    return [
        # The small fp32 workload of the benchmark (256 tokens of width 256): launches and latency.
        dict(name="norm_fwd_f32_small", op="norm_fwd", dtype="f32", form="layer", skip=False, T=256, d=256),
        # The benchmark's 1B-like width: the norm between a block's halves, with the skip connection's sum.
        dict(name="norm_fwd_bf16_1B", op="norm_fwd", dtype="bf16", form="layer", skip=True, T=16384, d=2048),
        # Its backward pass, with the skip connection's gradient.
        dict(name="norm_bwd_bf16_1B", op="norm_bwd", dtype="bf16", form="layer", skip=True, T=16384, d=2048),
        # The paper's 500M width, four sequences of its length, in the form of LLaMA-style blocks.
        dict(name="norm_bwd_bf16_paper_width", op="norm_bwd", dtype="bf16", form="rms", skip=True, T=4096, d=1200),
        # fp32 rows that fit no vector and no tile, as a ragged full-precision run gives them.
        dict(name="norm_bwd_f32_ragged", op="norm_bwd", dtype="f32", form="layer", skip=False, T=1023, d=511),
        # The way into the 1B-like model: one worker's batch, the paper's vocabulary of 32 K.
        dict(name="embed_fwd_bf16_1B", op="embed_fwd", dtype="bf16", T=16384, V=32000, d=2048, pad=0.0, scale=1.0),
        # A unit-sized model's embedding gradient: latency.
        dict(name="embed_bwd_f32_small", op="embed_bwd", dtype="f32", T=256, V=1024, d=256, pad=0.0, scale=16.0),
        # The embedding gradient of the 1B-like model.
        dict(name="embed_bwd_bf16_1B", op="embed_bwd", dtype="bf16", T=16384, V=32000, d=2048, pad=0.0, scale=1.0),
        # The paper's 1B width on a padded batch (a third of the ids name no row) over an odd, larger vocabulary.
        dict(name="embed_bwd_bf16_padded", op="embed_bwd", dtype="bf16", T=5000, V=50001, d=1600, pad=0.33, scale=40.0),
        # A unit-sized model's loss.
        dict(name="loss_f32_small", op="loss", dtype="f32", T=256, V=1024, pad=0.0),
        # The paper's vocabulary on the benchmark's batch of 8192 tokens: the largest tensor of the step.
        dict(name="loss_bf16_32K", op="loss", dtype="bf16", T=8192, V=32000, pad=0.0),
        # Rows of an odd vocabulary, which start at any alignment, a quarter of the tokens without a label (prompts, padding).
        dict(name="loss_bf16_ragged", op="loss", dtype="bf16", T=1000, V=50001, pad=0.25),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over the logarithm of the range."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "embed_fwd", "embed_bwd", "loss"])
    f32 = rng.random() < 0.25
    dtype = "f32" if f32 else "bf16"
    T = _log_int(rng, 1, 4096 if f32 else 16384)
    d = _log_int(rng, 64, 2048)
    if rng.random() < 0.6:
        d = max(64, d // 8 * 8)  # most models' widths
    V = _log_int(rng, 256, 64000)
    pad = rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.9), 2)])
    if op.startswith("norm"):
        return dict(op=op, dtype=dtype, form=rng.choice(["layer", "rms"]), skip=rng.random() < 0.5, T=T, d=d)
    if op.startswith("embed"):
        return dict(op=op, dtype=dtype, T=T, V=V, d=d, pad=pad, scale=rng.choice([1.0, round(math.sqrt(d), 3)]))
    return dict(op=op, dtype=dtype, T=min(T, 4096 if f32 else 8192, 8192 * 32000 // (V * (2 if f32 else 1))), V=V, pad=pad)


def _tokens(T, V, pad, g):
    """Token ids as text has them: frequencies fall about as 1 / rank, ranks lie anywhere in the vocabulary; `pad` of them are -1."""
    rank = (V ** torch.rand(T, generator=g, device="cuda", dtype=torch.float64)).long().clamp_(1, V) - 1
    ids = torch.randperm(V, generator=g, device="cuda")[rank]
    if pad:
        ids = torch.where(torch.rand(T, generator=g, device="cuda") < pad, -1, ids)
    return ids.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, T, op = _DT[case["dtype"]], case["T"], case["op"]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dt)

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = dict(case=case)
    if op.startswith("norm"):
        d, layer = case["d"], case["form"] == "layer"
        s.update(gamma=normal(d, std=0.2, mean=1.0), beta=normal(d, std=0.1) if layer else None)
        X = normal(T, d) + normal(1, d, std=0.5)  # columns with an offset of their own, as a residual stream has them
        if op == "norm_fwd":
            s.update(X=X, R=normal(T, d, std=0.3) if case["skip"] else None)
            s["out"] = (empty(T, d), empty(T, d) if case["skip"] else None,
                        empty(T, dtype=torch.float32) if layer else None, empty(T, dtype=torch.float32))
        else:
            x = X.double()  # the forward call's saved statistics
            mean = x.mean(1) if layer else torch.zeros_like(x[:, 0])
            rstd = ((x - mean[:, None]).square().mean(1) + _EPS).rsqrt()
            s.update(H=X, dY=normal(T, d), dH=normal(T, d) if case["skip"] else None,
                     mean=mean.float() if layer else None, rstd=rstd.float())
            s["out"] = (empty(T, d), empty(d), empty(d) if layer else None)
    elif op.startswith("embed"):
        V, d = case["V"], case["d"]
        s["ids"] = _tokens(T, V, case["pad"], g)
        if op == "embed_fwd":
            s.update(E=normal(V, d, std=0.02), out=empty(T, d))
        else:
            s.update(dY=normal(T, d, std=1e-2), out=empty(V, d))
    else:
        V = case["V"]
        s.update(Z=normal(T, V, std=2.0), labels=_tokens(T, V, case["pad"], g))
        s["out"] = (empty(T, dtype=torch.float32), empty(T, dtype=torch.float32), empty(T, V), empty(1, dtype=torch.float32))
        s["scale"] = empty(1, dtype=torch.float32)
    return s


def _run_own(s):
    import paper_2507_09029_amd as sdp

    c = s["case"]
    op = c["op"]
    if op == "norm_fwd":
        return sdp.norm_fwd(c["form"], s["X"], s["gamma"], s["beta"], residual=s["R"], eps=_EPS, out=s["out"])
    if op == "norm_bwd":
        if "ws" not in s:  # kept by the program from its first step on
            s["ws"] = torch.empty(sdp.norm_bwd_workspace_bytes(s["H"].dtype, c["T"], c["d"]), dtype=torch.uint8, device="cuda")
        return sdp.norm_bwd(c["form"], s["H"], s["dY"], s["gamma"], s["mean"], s["rstd"], dH=s["dH"], out=s["out"], ws=s["ws"])
    if op == "embed_fwd":
        return sdp.embed_fwd(s["E"], s["ids"], c["scale"], out=s["out"])
    if op == "embed_bwd":
        if "ws" not in s:
            s["ws"] = torch.empty(sdp.embed_bwd_workspace_bytes(s["dY"].dtype, c["T"], c["V"], c["d"]), dtype=torch.uint8, device="cuda")
        return sdp.embed_bwd(s["dY"], s["ids"], c["V"], c["scale"], out=s["out"], ws=s["ws"])
    sdp.label_scale(s["labels"], c["V"], out=s["scale"])
    return sdp.token_loss(s["Z"], s["labels"], scale_dev=s["scale"], out=s["out"])


def run(s):
    if own:
        got = _run_own(s)
        if s["case"]["op"] == "norm_fwd" and s["R"] is None:
            return got[0], None, got[2], got[3]
        return got
    c = s["case"]
    op = c["op"]
    if op == "norm_fwd":
        H = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(s["X"].dtype)
        h = H.float()
        mean = h.mean(1) if s["beta"] is not None else None
        h = h if mean is None else h - mean[:, None]
        rstd = (h.square().mean(1) + _EPS).rsqrt()
        y = h * rstd[:, None] * s["gamma"].float()
        y = y if mean is None else y + s["beta"].float()
        return y.to(H.dtype), None if s["R"] is None else H, mean, rstd
    if op == "norm_bwd":
        dy, dt, rstd = s["dY"].float(), s["H"].dtype, s["rstd"][:, None]
        x = s["H"].float()
        x = x * rstd if s["mean"] is None else (x - s["mean"][:, None]) * rstd
        gr = dy * s["gamma"].float()
        dx = gr - x * (gr * x).mean(1, keepdim=True)
        dx = dx if s["mean"] is None else dx - gr.mean(1, keepdim=True)
        dx = dx * rstd
        dx = dx if s["dH"] is None else dx + s["dH"].float()
        return dx.to(dt), (dy * x).sum(0).to(dt), None if s["mean"] is None else dy.sum(0).to(dt)
    if op == "embed_fwd":
        ids = s["ids"].long()
        live = (ids >= 0) & (ids < c["V"])
        return (s["E"][torch.where(live, ids, 0)].float() * c["scale"] * live[:, None]).to(s["E"].dtype)
    if op == "embed_bwd":
        ids = s["ids"].long()
        live = (ids >= 0) & (ids < c["V"])
        dE = torch.zeros((c["V"], c["d"]), dtype=torch.float32, device="cuda")
        dE.index_add_(0, torch.where(live, ids, 0), s["dY"].float() * live[:, None])
        return (dE * c["scale"]).to(s["dY"].dtype)
    labels = s["labels"].long()
    live = (labels >= 0) & (labels < c["V"])
    at = torch.where(live, labels, 0)[:, None]
    z = s["Z"].float()
    m = z.max(1, keepdim=True).values
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lse = torch.where(live, (m + total.log())[:, 0], 0.0)
    nll = torch.where(live, ((m - z.gather(1, at)) + total.log())[:, 0], 0.0)
    p = e / total
    p.scatter_add_(1, at, torch.full_like(total, -1.0))
    count = live.sum()
    scale = live.float() / count.clamp(min=1)
    dZ = (p * scale[:, None]).to(s["Z"].dtype)
    return nll, lse, dZ, (nll.double().sum() / count.clamp(min=1)).float()[None]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm_fwd":
        total = s["X"].to(torch.float64)
        if s["R"] is not None:
            total = total + s["R"].to(torch.float64)
        h = total.to(s["X"].dtype).to(torch.float64)  # the norm is that of the sum as it is stored
        mu = h.sum(1) / case["d"] * (1.0 if case["form"] == "layer" else 0.0)
        var = torch.linalg.vector_norm(h - mu.unsqueeze(1), dim=1) ** 2 / case["d"]
        sigma = torch.sqrt(var + _EPS)
        y = torch.addcmul(s["beta"].double() if s["beta"] is not None else torch.zeros((), dtype=torch.float64, device="cuda"),
                          (h - mu.unsqueeze(1)) / sigma.unsqueeze(1), s["gamma"].double())
        return y, total if s["R"] is not None else None, mu if case["form"] == "layer" else None, 1.0 / sigma
    if op == "norm_bwd":
        h, dy, gamma = s["H"].double(), s["dY"].double(), s["gamma"].double()
        if case["form"] == "layer":
            h = h - h.sum(1, keepdim=True) / case["d"]
        sigma = torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + _EPS)
        up = dy @ torch.diag(gamma)
        # derivative of h / sigma(h): the upstream gradient less its part along h, over sigma
        dx = up / sigma - h * ((up * h).sum(1, keepdim=True) / (case["d"] * sigma ** 3))
        if case["form"] == "layer":
            dx = dx - dx.sum(1, keepdim=True) / case["d"]  # through the mean: h sums to zero
        if s["dH"] is not None:
            dx = dx + s["dH"].double()
        return dx, torch.einsum("td,td->d", dy, h / sigma), dy.T @ torch.ones_like(dy[:, 0]) if case["form"] == "layer" else None
    if op == "embed_fwd":
        rows = torch.cat([s["E"].double() * case["scale"], torch.zeros((1, case["d"]), dtype=torch.float64, device="cuda")])
        return rows[s["ids"].long()]  # -1: the row of zeros behind the last
    if op == "embed_bwd":
        order = torch.argsort(s["ids"], stable=True)
        ids = s["ids"][order].long()
        rows, counts = torch.unique_consecutive(ids, return_counts=True)
        sums = torch.segment_reduce(s["dY"].double()[order], "sum", lengths=counts, axis=0)
        dE = torch.zeros((case["V"], case["d"]), dtype=torch.float64, device="cuda")
        dE[rows[rows >= 0]] = sums[rows >= 0] * case["scale"]
        return dE
    kept = torch.nonzero(s["labels"] >= 0)[:, 0]
    T, V, n = case["T"], case["V"], max(1, len(kept))
    nll, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    dZ = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    z, at = s["Z"][kept].double(), s["labels"][kept].long()
    lse[kept] = torch.logsumexp(z, 1)
    nll[kept] = lse[kept] - z[torch.arange(len(kept), device="cuda"), at]
    dZ[kept] = (z - lse[kept].unsqueeze(1)).exp_() / n
    dZ[kept, at] -= 1.0 / n
    return nll, lse, dZ, nll.sum().reshape(1) / n


def work(case):
    T, e = case["T"], 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "norm_fwd":
        layer = case["form"] == "layer"
        return {"bytes": (4 if case["skip"] else 2) * T * case["d"] * e + (2 if layer else 1) * (case["d"] * e + T * 4), "flops": 8 * T * case["d"]}
    if op == "norm_bwd":
        layer = case["form"] == "layer"
        return {"bytes": (4 if case["skip"] else 3) * T * case["d"] * e + (3 if layer else 2) * case["d"] * e + (2 if layer else 1) * T * 4,
                "flops": 14 * T * case["d"]}
    if op.startswith("embed"):
        V, d = case["V"], case["d"]
        live = T * (1.0 - case["pad"])
        # distinct ids of `live` draws whose rank's logarithm is uniform: for rank r the chance to be seen is 1 - exp(-live p_r)
        rows, r = 0.0, 1
        while r <= V:
            step = max(1, r // 16)
            rows += min(step, V + 1 - r) * (1.0 - math.exp(-live * math.log1p(1.0 / (r + step / 2)) / math.log(V)))
            r += step
        if op == "embed_fwd":
            return {"bytes": rows * d * e + T * d * e + 4 * T, "flops": T * d}
        return {"bytes": live * d * e + V * d * e + 4 * T, "flops": 2 * live * d}
    live = T * (1.0 - case["pad"])
    return {"bytes": live * case["V"] * e + T * case["V"] * e + 12 * T, "flops": 8 * live * case["V"]}
