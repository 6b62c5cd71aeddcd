"""Shared by the tests of the losses on logits and on the output head: 64-bit forms, entries of a teacher, and bounds on errors.

Bounds, elementwise (u = 2^-24; half = half a step of the stored type, 2^-8 relative for bf16):
  z      a logit X W^T in fp32 from exact products of bf16 (the matrix instruction adds 32 of them at a time, counted as four roundings): at most
         (d / 8 + 8) u sum |x w|; from fp32 operands (split into three bf16 terms or as they are), (d / 2 + 16) u sum |x w|: `z_err`
  exps   the exponents (z - max) log2(e) / tau are rounded three times, at most 64 each: 4 x 64 u ln 2 = 1.1e-5 relative, 2e-5 with the sum's own
         roundings and the hardware's 2^x: lse within 2e-5 + z_err / tau, p within 2e-5 + 2 z_err / tau relative
  q      the same exponents: 2e-5 relative; log q within 2e-5
  kl     sum q (log q - z / tau + lse): mass x (4e-5 + 2 z_err / tau) + 2e-5 sum q |log q - log p| + the sum's own roundings, 2e-6 of the same sum
  dz     c / tau (mass p - q): c / tau (mass p (2e-5 + 2 z_err / tau) + q 2e-5), and its rounding to the stored type; in the head with bf16 beside it
         5.2e-4 c / tau mass p from the 16-bit distance to the block's largest logit (elements of entries do without), and mass 2^-95 c / tau
         for what is below that distance's range
         Of 128 tokens with a target or fewer the head holds dz in two terms: 2^-17 of it instead of 2^-8 (`two`)
  dX, dW sums over dz's bound times |W|, |X|; the product's roundings, (depth / 8 + 8) u (fp32: depth / 2 + 16) times the sum of
         magnitudes; the result's rounding
"""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def entries(T, V, k, seed=0, pad=0.0, cut=False, wide=False, dtype=torch.float32, twice=False):
    """ids [T][k], top [T][k] of a teacher: different tokens of the vocabulary where k <= V and not `twice`; some rows and ends of rows are none."""
    g = torch.Generator().manual_seed(1000 + seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] if k <= V and not twice else torch.randint(0, V, (k,), generator=g) for _ in range(T)])
    top = 6.0 + torch.randn((T, k), generator=g) - 1.5 * torch.log1p(torch.arange(k).float())
    if cut:
        n = torch.randint(1, k + 1, (T, 1), generator=g)
        gone = torch.arange(k)[None] >= n
        low = torch.rand((T, k), generator=g) < 0.5  # one way to say that there is none, or the other
        ids = torch.where(gone & ~low, torch.where(torch.rand((T, k), generator=g) < 0.5, -1, V), ids)
        top = torch.where(gone & low, float("-inf"), top)
    if pad:
        ids[torch.rand(T, generator=g) < pad] = -1
    return ids.to(torch.int64 if wide else torch.int32), top.to(dtype)


def rest_of(top, ids, V, tau, seed=0):
    """A teacher's log-sum-exp over its whole vocabulary: that of the entries and some more."""
    g = torch.Generator().manual_seed(77 + seed)
    a = torch.where((ids >= 0) & (ids < V), top.double() / tau, float("-inf"))
    return (torch.logsumexp(a, 1).nan_to_num(0.0, 0.0, 0.0) + 0.02 + torch.rand(a.shape[0], generator=g, dtype=torch.float64)).float()


def targets64(ids, top, top_lse, V, tau):
    """-> dense q [T][V], sum q log q and sum q |log q| helpers: (q, entries' q, their log q, their ids or 0, live)."""
    there = (ids >= 0) & (ids < V)
    if top is not None:
        there = there & (top != float("-inf"))
    at = torch.where(there, ids.long(), 0)
    if top is None:
        q, log_q = there.double(), torch.zeros(ids.shape, dtype=torch.float64, device=ids.device)
    else:
        a = torch.where(there, top.double() / tau, float("-inf"))
        L = torch.logsumexp(a, 1, keepdim=True) if top_lse is None else top_lse.double()[:, None]
        log_q = torch.where(there, a - L, 0.0)
        q = torch.where(there, log_q.exp(), 0.0)
    dense = torch.zeros((ids.shape[0], V), dtype=torch.float64, device=ids.device).scatter_add_(1, at, q)
    return dense, q, log_q, at, there.any(1)


class Want:
    """The loss of logits z (64 bits) against targets, its gradient, and the bounds above; rows without a target are zeros whatever z holds."""

    def __init__(self, z, ids, top, top_lse, tau, c, z_err=0.0, stored=torch.float32, codes=False, half=None):
        T, V = z.shape
        dense, q, log_q, at, live = targets64(ids, top, top_lse, V, tau)
        z = torch.where(live[:, None], z, 0.0) / tau
        e = torch.as_tensor(z_err, dtype=torch.float64, device=z.device) / tau
        e = torch.where(live, e, 0.0) if e.dim() else e
        mass = dense.sum(1)
        self.live = live
        top_z = z.amax(1, keepdim=True)
        z = z - top_z  # the differences first: values may be near the type's lowest or highest
        from_top = torch.logsumexp(z, 1)
        lse = top_z[:, 0] + from_top
        terms = log_q - z.gather(1, at) + from_top[:, None]
        self.kl = torch.where(live, torch.where(q > 0, q * terms, 0.0).sum(1), 0.0)
        self.lse = torch.where(live, lse, 0.0)
        size = torch.where(q > 0, q * terms.abs(), 0.0).sum(1)
        self.kl_room = torch.where(live, mass * (4e-5 + 2 * e) + 2.2e-5 * size + 2 * U * self.kl.abs(), 0.0) + 1e-30
        self.lse_room = torch.where(live, 2e-5 + e + 2 * U * lse.abs(), 0.0) + 1e-30
        p = (z - from_top[:, None]).exp() * mass[:, None]
        self.dz = torch.where(live[:, None], (p - dense) * (c / tau), 0.0)
        e = e[:, None] if e.dim() else e
        room = abs(c) / tau * (p * (2e-5 + 2 * e) + dense * 2e-5 + 2 * U * torch.maximum(p, dense))
        if codes:
            room = room + abs(c) / tau * torch.where(dense > 0, 0.0, 5.2e-4 * p + mass[:, None] * 2.0 ** -95)
        self.dz_room = torch.where(live[:, None], room, 0.0)
        self.dz_room += (half or HALF[stored]) * (self.dz.abs() + self.dz_room) + torch.where(live[:, None], 1e-37, 0.0)
        self.loss = self.kl.sum() * c
        self.loss_room = abs(c) * (self.kl_room.sum() + 4 * U * self.kl.abs().sum()) + 1e-30

    def rows(self, kl, lse, loss):
        near(kl, self.kl, self.kl_room, "kl")
        if lse is not None:
            near(lse, self.lse, self.lse_room, "lse")
        if loss is not None:
            near(loss.reshape(()), self.loss, self.loss_room, "loss")


def near(got, want, room, name):
    off = (got.to(want.device).double() - want).abs()
    worst = float((off / room).max()) if off.numel() else 0.0
    assert not off.isnan().any() and worst <= 1.0, f"{name}: {worst:.2f} of its bound"


def z_bound(X, W):
    """The bound of every row's logits (the largest over its columns)."""
    d = X.shape[1]
    f = (d / 8 + 8 if X.dtype == torch.bfloat16 else d / 2 + 16) * U
    return f * (X.double().abs().nan_to_num() @ W.double().abs().T).amax(1)


def product_bound(A, B, room, stored, exact):
    """Of A B where A is known within `room` and stored, B exactly.  A sum of dW runs over 32768 tokens at most, and then over these sums."""
    n = min(A.shape[1], 32768 + A.shape[1] // 32768)
    f = (n / 8 + 8 if stored == torch.bfloat16 else n / 2 + 16) * U
    b = B.abs()
    return (room + f * (A.abs() + room)) @ b + HALF[stored] * exact.abs() + 1e-37


class HeadWant(Want):
    def __init__(self, X, W, ids, top, top_lse, tau, c):
        dt = X.dtype
        live = targets64(ids, top, top_lse, W.shape[0], tau)[4]
        x = torch.where(live[:, None], X.double(), 0.0)
        w = W.double()
        two = dt == torch.bfloat16 and int(live.sum()) <= 128
        super().__init__(x @ w.T, ids, top, top_lse, tau, c, z_bound(x.to(dt), W), dt, codes=dt == torch.bfloat16, half=2.0 ** -17 if two else None)
        self.dX, self.dW = self.dz @ w, self.dz.T @ x
        self.dX_room = product_bound(self.dz, w, self.dz_room, dt, self.dX)
        self.dX_room = torch.where(live[:, None], self.dX_room, 1e-300)
        self.dW_room = product_bound(self.dz.T, x, self.dz_room.T, dt, self.dW)

    def check(self, got):
        kl, lse, dX, dW, loss = got
        self.rows(kl, lse, loss)
        if dX is not None:
            near(dX, self.dX, self.dX_room, "dX")
        if dW is not None:
            near(dW, self.dW, self.dW_room, "dW")
