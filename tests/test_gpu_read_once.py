"""Norms and token loss on matrices that are read around the caches: 128 MB of input or more, in rows of whole 128-byte lines that start at one.

Other kernels than those of smaller matrices have these, one for every number of waves and pieces of a row.  Each is held against 64 bits on
sampled rows, and against the kernels that read through the caches on all rows: the same data 16 bytes behind a line has to give the same bits,
since the order of every sum is that of the row's shape alone.  Tolerances as in the tests of the smaller matrices, whose sums are as long."""
import pytest
import torch

from around import DT, loss64, norm_bwd64, norm_fwd64

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 1e-5
ONCE = 1 << 27  # bytes of input


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def _room(T, d, dt, behind=0):
    """[T][d], `behind` bytes behind a line of 128."""
    es = torch.tensor([], dtype=dt).element_size()
    buf = torch.empty(T * d + 128, dtype=dt, device="cuda")
    at = (-buf.data_ptr() % 128 + behind) // es
    t = buf[at: at + T * d].view(T, d)
    assert t.data_ptr() % 128 == behind and d * es % 128 == 0
    return t


def _put(x, behind=0):
    return _room(*x.shape, x.dtype, behind).copy_(x)


def _normal(T, d, dt, seed, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _room(T, d, dt).copy_(torch.randn((T, d), generator=g, device="cuda") * std + mean)


def _close_rows(got, want, tol, what):
    """Each row within tol of max(its rms, value)."""
    want = want.to(got.device)
    off = (got.double() - want).abs() / torch.maximum(want.square().mean(1, keepdim=True).sqrt(), want.abs())
    assert off.max() <= tol, f"{what}: {float(off.max()):.2e}"


# widths of every number of waves and pieces, and some that leave lanes and waves without a piece
@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in (64, 512, 1024, 1088, 1536, 2048, 3200, 4096, 8192, 10048, 16384)] +
                         [("f32", d) for d in (32, 256, 512, 768, 1024, 1056, 1536, 2048, 4096, 8192, 9024, 16384)])
def test_norms(sdp, dtype, d):
    dt = DT[dtype]
    es = 2 if dtype == "bf16" else 4
    tol = HALF[dtype] + 1e-5
    gamma, beta = (_normal(1, d, dt, s, std=0.3, mean=m)[0] for s, m in ((1, 1.0), (2, 0.0)))
    # alone, and of two matrices that only together are enough; a row or three more than they need
    for kind, skip in (("layer", False), ("rms", True)):
        T = ONCE // (d * es * (1 + skip)) + (3 if skip else 1)
        print(f"norm {kind} {dtype} T={T} d={d} skip={skip}", flush=True)
        rows = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
        of = lambda t: None if t is None else t[rows].cpu()
        X, R = _normal(T, d, dt, 3, mean=0.7), _normal(T, d, dt, 4, std=0.5) if skip else None
        b = beta if kind == "layer" else None
        st = lambda: torch.empty((T,), device="cuda")
        Y, H, mean, rstd = sdp.norm_fwd(kind, X, gamma, b, residual=R, eps=EPS, out=(_room(T, d, dt), _room(T, d, dt), st(), st()))
        wY, wH, wm, wr = norm_fwd64(kind, of(X), of(R), gamma.cpu(), None if b is None else b.cpu(), EPS)
        assert torch.equal(of(H), wH)
        _close_rows(Y[rows], wY, tol, "Y")
        assert ((of(rstd).double() - wr).abs() <= 1e-5 * wr).all()
        seen = sdp.norm_fwd(kind, _put(X, 16), gamma, b, residual=None if R is None else _put(R, 16), eps=EPS)
        assert torch.equal(seen[0], Y) and torch.equal(seen[1], H) and torch.equal(seen[3], rstd) and (kind == "rms" or torch.equal(seen[2], mean))
        x, r = _put(X), None if R is None else _put(R)
        sdp.norm_fwd(kind, x, gamma, b, residual=r, eps=EPS, out=(x, r, st(), st()))
        assert torch.equal(x, Y) and (r is None or torch.equal(r, H))
        if skip:
            x, r = _put(X), _put(R)
            sdp.norm_fwd(kind, x, gamma, b, residual=r, eps=EPS, out=(r, x, st(), st()))
            assert torch.equal(r, Y) and torch.equal(x, H)
        del x, r, seen, Y, R

        # backward, with two matrices or three: T rows are enough for either
        dY, dH = _normal(T, d, dt, 5), _normal(T, d, dt, 6) if skip else None
        bias = kind == "layer"
        want = sdp.norm_bwd(kind, H, dY, gamma, mean, rstd, dH=dH, out=(_room(T, d, dt), torch.empty_like(gamma), torch.empty_like(gamma) if bias else None))
        wX, _, _ = norm_bwd64(kind, wH, of(dY), of(dH), gamma.cpu(), wm, wr)
        _close_rows(want[0][rows], wX, tol, "dX")
        seen = sdp.norm_bwd(kind, _put(H, 16), _put(dY, 16), gamma, mean, rstd, dH=None if dH is None else _put(dH, 16), bias=bias)
        assert all(torch.equal(a, c) for a, c in zip(seen, want) if c is not None)
        for place in range(3 if skip else 2):
            ops = [_put(t) for t in ((H, dY, dH) if skip else (H, dY))]
            dws = torch.empty_like(gamma), torch.empty_like(gamma) if bias else None
            got = sdp.norm_bwd(kind, ops[0], ops[1], gamma, mean, rstd, dH=ops[2] if skip else None, out=(ops[place], *dws))
            assert all(torch.equal(a, c) for a, c in zip(got, want) if c is not None), place


# a width for every number of waves and pieces: rows as long as they hold (2880: less), but for the values behind the last whole piece
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces", [64, 128, 256, 512, 1024, 1536, 2048, 2880, 4096, 5120, 6144, 7168, 8192, 12288, 16384])
def test_loss(sdp, dtype, pieces):
    dt = DT[dtype]
    es, n = (2, 8) if dtype == "bf16" else (4, 4)
    ldz = pieces * n
    V = ldz - 3
    T = ONCE // (ldz * es) + 2
    print(f"loss {dtype} T={T} V={V} ldz={ldz}", flush=True)
    Z = _normal(T, ldz, dt, 1, std=3.0)
    g = torch.Generator(device="cuda").manual_seed(T)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels[1], labels[T - 2] = -1, V
    labels[0], labels[T - 1] = V - 1, 0
    rows = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    c = 0.5
    st = lambda k=T: torch.empty((k,), device="cuda")
    dZ = _room(T, ldz, dt).fill_(7.0)
    nll, lse, _, loss = sdp.token_loss(Z[:, :V], labels, scale=c, out=(st(), st(), dZ[:, :V], st(1)))
    wn, wl, wz, _ = loss64(Z[rows, :V].cpu(), labels[rows].cpu(), c)
    assert ((nll[rows].cpu().double() - wn).abs() <= 1.5e-5 * wn.clamp(min=1)).all() and ((lse[rows].cpu().double() - wl).abs() <= 1.5e-5 * wl.clamp(min=1)).all()
    live = (wl != 0)[:, None]
    p = torch.where(live, (Z[rows, :V].cpu().double() - wl[:, None]).exp(), 0.0)
    room = HALF[dtype] * wz.abs() + 2e-5 * c * p + 2.0 ** -24 * c * (wz < 0) + 1e-37
    assert ((dZ[rows, :V].cpu().double() - wz).abs() <= room).all()
    assert (dZ[:, V:] == 7.0).all()
    assert abs(float(loss) - c * float(nll.double().sum())) <= 1e-6 * float(loss)
    # through the caches: the same data behind a line's start
    out = _room(T, ldz, dt, 16).fill_(7.0)
    seen = sdp.token_loss(_put(Z, 16)[:, :V], labels, scale=c, out=(st(), st(), out[:, :V], st(1)))
    assert torch.equal(seen[0], nll) and torch.equal(seen[1], lse) and torch.equal(seen[3], loss) and torch.equal(out, dZ)
    # in the logits' place, and without a gradient
    z = _put(Z)
    sdp.token_loss(z[:, :V], labels, scale=c, out=(seen[0], seen[1], z[:, :V], seen[3]))
    assert torch.equal(z[:, :V], dZ[:, :V]) and torch.equal(z[:, V:], Z[:, V:]) and torch.equal(seen[0], nll)
    only = sdp.token_loss(Z[:, :V], labels, scale=c, want_grad=False)
    assert torch.equal(only[0], nll) and torch.equal(only[1], lse) and torch.equal(only[3], loss)
