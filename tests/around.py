"""Shared by the tests of norms, token embedding and token loss: tensors between guards, at any element, and 64-bit forms."""
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 40  # elements on each side


class Guarded:
    """A contiguous GPU tensor of `shape` that starts `at` elements behind a 256-byte line, between guards that nothing may write."""

    def __init__(self, shape, dtype, at=0, value=None):
        n = 1
        for s in shape:
            n *= s
        self.buf = torch.full((GUARD + at + n + GUARD + 64,), 7, dtype=dtype, device="cuda")
        self.lo = GUARD + 24 + at
        self.hi = self.lo + n
        if self.hi + GUARD > self.buf.numel():
            self.buf = torch.full((self.hi + GUARD,), 7, dtype=dtype, device="cuda")
        self.t = self.buf[self.lo: self.hi].view(shape)
        self.t.copy_(value) if value is not None else self.t.fill_(float("nan") if dtype.is_floating_point else -77)

    def check(self, what=""):
        assert (self.buf[: self.lo] == 7).all() and (self.buf[self.hi:] == 7).all(), f"{what}: written outside its memory"


def normal(*shape, dtype=torch.float32, seed=0, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std + mean).to(dtype)


def norm_fwd64(kind, X, R, gamma, beta, eps):
    """-> Y, H (as stored), mean, rstd in 64 bits."""
    H = X if R is None else (X.double() + R.double()).to(X.dtype)
    h = H.double()
    mean = h.mean(1) if kind == "layer" else torch.zeros(h.shape[0], dtype=torch.float64)
    c = h - mean[:, None]
    rstd = 1.0 / ((c * c).mean(1) + eps).sqrt()
    y = c * rstd[:, None] * gamma.double()
    return y if beta is None else y + beta.double(), H, mean, rstd


def norm_bwd64(kind, H, dY, dH, gamma, mean, rstd):
    xh, dy = (H.double() - mean[:, None]) * rstd[:, None], dY.double()
    g = dy * gamma.double()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd[:, None]
    return dx if dH is None else dx + dH.double(), (dy * xh).sum(0), dy.sum(0)


def embed_bwd64(dY, ids, V, scale):
    dE = torch.zeros((V, dY.shape[1]), dtype=torch.float64)
    live = (ids >= 0) & (ids < V)
    return dE.index_add_(0, ids[live].long(), dY[live].double()) * scale


def loss64(Z, labels, c):
    """-> nll, lse, dZ, loss in 64 bits; rows without a label are zeros whatever they hold."""
    T, V = Z.shape
    nll, lse, dZ = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64), torch.zeros((T, V), dtype=torch.float64)
    live = torch.nonzero((labels >= 0) & (labels < V))[:, 0]
    z, at = Z[live].double(), labels[live].long()
    lse[live] = torch.logsumexp(z, 1)
    nll[live] = torch.logsumexp(z - z.gather(1, at[:, None]), 1)  # the difference first: values may be near the type's lowest
    p = torch.softmax(z, 1)
    p[torch.arange(len(live)), at] -= 1.0
    dZ[live] = p * c
    return nll, lse, dZ, nll.sum() * c
