"""GPU parity of the norms against 64 bits: layer and root-mean-square form, with and without the skip connection's sum and bias,
widths and row counts around every change of tile, matrices that start at any element.

Tolerances (relative to max(rms, value)): an output is rounded once, by at most half a step (2^-8 bf16), on top of fp32 arithmetic.
fp32: a sum of n values adds n roundings of 2^-24 of a partial sum.  A row's sums have at most 32 values a lane, 6 steps of a wave and 16
waves: 54 x 2^-24 = 3.2e-6 each, two of them (mean, squares) and a handful of products: 1e-5.  dgamma, dbeta: partial sums of values of
random sign stay near the result's rms, along at most 5 rows a wave here, 8 waves' rows of a workgroup, 16 of at most 256 workgroups' shares a wave and
16 waves: 45 x 2^-24 = 2.7e-6; with xh's own error, 1e-5, below 2e-5."""
import pytest
import torch

from around import DT, Guarded, norm_bwd64, norm_fwd64, normal
from helpers import assert_close, assert_close_rows

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 1e-5


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def _run(sdp, kind, dtype, T, d, skip, bias, at, seed=1):
    dt = DT[dtype]
    X = normal(T, d, dtype=dt, seed=seed, mean=0.7)
    R = normal(T, d, dtype=dt, seed=seed + 1, std=0.5) if skip else None
    gamma, beta = normal(d, dtype=dt, seed=seed + 2, std=0.3, mean=1.0), normal(d, dtype=dt, seed=seed + 3) if bias else None
    dY, dH = normal(T, d, dtype=dt, seed=seed + 4), normal(T, d, dtype=dt, seed=seed + 5) if skip else None
    put = lambda t: None if t is None else Guarded(t.shape, t.dtype, at, t).t
    room = lambda *s, t=dt: Guarded(s, t, at)
    Y, H = room(T, d), room(T, d) if skip else None
    mean, rstd = room(T, t=torch.float32) if kind == "layer" else None, room(T, t=torch.float32)
    of = lambda g: None if g is None else g.t
    got = sdp.norm_fwd(kind, put(X), put(gamma), put(beta), residual=put(R), eps=EPS, out=(Y.t, of(H), of(mean), rstd.t))
    wY, wH, wmean, wrstd = norm_fwd64(kind, X, R, gamma, beta, EPS)
    dX, dg, db = room(T, d), room(d), room(d) if bias else None
    sdp.norm_bwd(kind, put(wH), put(dY), put(gamma), of(mean), rstd.t, dH=put(dH), out=(dX.t, dg.t, of(db)))
    torch.cuda.synchronize()
    for g in (Y, H, mean, rstd, dX, dg, db):
        if g is not None:
            g.check()
    tol = HALF[dtype] + 1e-5
    assert_close(got[0].cpu().double(), wY, tol, "Y")
    if skip:
        assert torch.equal(got[1].cpu(), wH), "H: the sum of two values of the type, rounded once, has one value"
    if kind == "layer":
        assert_close(mean.t.cpu().double(), wmean, 1e-5, "mean")
    assert_close(rstd.t.cpu().double(), wrstd, 1e-5, "rstd")
    wX, wg, wb = norm_bwd64(kind, wH, dY, dH, gamma, wmean, wrstd)
    assert_close(dX.t.cpu().double(), wX, tol, "dX")
    assert_close(dg.t.cpu().double(), wg, HALF[dtype] + 2e-5, "dgamma")
    if bias:
        assert_close(db.t.cpu().double(), wb, HALF[dtype] + 2e-5, "dbeta")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 6), (1, 8), (3, 5), (5, 64), (7, 255), (64, 256), (65, 257), (33, 511), (33, 512), (20, 513), (9, 768), (257, 1000),
                                 (100, 1024), (31, 1025), (300, 1200), (17, 1536), (9, 1537), (40, 1600), (130, 2048), (6, 2049), (5, 4096), (3, 4100),
                                 (2, 8191), (3, 8192), (2, 8200), (2, 12289), (1, 16383), (2, 16384), (4099, 72), (2500, 264)])
def test_norm_matches_64_bits(sdp, dtype, T, d):
    for kind, skip, bias, at in (("layer", True, True, 0), ("rms", False, False, 1), ("layer", False, False, 3)):
        print(f"norm {kind} {dtype} T={T} d={d} skip={skip} bias={bias} at={at}", flush=True)
        _run(sdp, kind, dtype, T, d, skip, bias, at)
    print(f"norm rms with a sum and a bias {dtype} T={T} d={d}", flush=True)
    _run(sdp, "rms", dtype, T, d, True, True, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(700, 9001), (1100, 12296)])
def test_many_wide_rows(sdp, dtype, T, d):
    """Several turns of every workgroup at widths whose rows are not requested ahead."""
    _run(sdp, "layer", dtype, T, d, True, True, 0)
    _run(sdp, "rms", dtype, T, d, False, False, 1)


def test_norm_of_one_value_and_of_constant_rows(sdp):
    """Width 1 and rows of one value: the layer form gives beta (variance 0, s = 1 / sqrt(eps)) and no gradient by x, exactly."""
    for dtype in ("f32", "bf16"):
        dt = DT[dtype]
        for T, d in ((3, 1), (4, 100)):
            X = torch.full((T, d), 1.5, dtype=dt, device="cuda")
            gamma, beta = (normal(d, dtype=dt, seed=s).cuda() for s in (1, 2))
            Y, H, mean, rstd = sdp.norm_fwd("layer", X, gamma, beta, eps=0.25)
            assert torch.equal(Y, beta.expand(T, d)) and (mean == 1.5).all() and (rstd == 2.0).all()
            dX, dg, db = sdp.norm_bwd("layer", H, torch.ones_like(X), torch.ones_like(gamma), mean, rstd)
            assert (dX == 0).all() and (dg == 0).all() and (db == T).all()


def test_gradients_match_differences(sdp):
    """fp32, central differences of the loss sum(Y W) + sum(H W2) in 64 bits of the same inputs, step 1e-6: error 1e-10 / 1e-6 + 1e-12."""
    T, d = 3, 37
    X, W, W2, gamma = (normal(T, d, seed=s) for s in (1, 2, 3, 4))
    gamma = gamma[0]

    def f(x, g):
        y, _, _, _ = norm_fwd64("layer", x, None, g, None, EPS)
        return float((y * W.double()).sum() + (x.double() * W2.double()).sum())

    Y, H, mean, rstd = sdp.norm_fwd("layer", X.cuda(), gamma.cuda(), eps=EPS)
    dX, dg, _ = sdp.norm_bwd("layer", H, W.cuda(), gamma.cuda(), mean, rstd, dH=W2.cuda(), bias=False)
    x64, g64 = X.double(), gamma.double()
    for t in range(T):
        for e in (0, 5, 36):
            hi, lo = x64.clone(), x64.clone()
            hi[t, e] += 1e-6
            lo[t, e] -= 1e-6
            assert abs((f(hi, g64) - f(lo, g64)) / 2e-6 - float(dX[t, e])) < 1e-4
    for e in (0, 36):
        hi, lo = g64.clone(), g64.clone()
        hi[e] += 1e-6
        lo[e] -= 1e-6
        assert abs((f(x64, hi) - f(x64, lo)) / 2e-6 - float(dg[e])) < 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(37, 200), (300, 2048), (11, 5000), (3, 16000)])
def test_in_place_is_the_same(sdp, dtype, T, d):
    dt = DT[dtype]
    X, R, dY, dH = (normal(T, d, dtype=dt, seed=s).cuda() for s in (1, 2, 3, 4))
    gamma = normal(d, dtype=dt, seed=5).cuda()
    Y, H, mean, rstd = sdp.norm_fwd("layer", X, gamma, residual=R)
    st = lambda: torch.empty((T,), device="cuda")
    for order in (0, 1):
        x, r = X.clone(), R.clone()
        y, h = (x, r) if order else (r, x)
        sdp.norm_fwd("layer", x, gamma, residual=r, out=(y, h, st(), st()))
        assert torch.equal(y, Y) and torch.equal(h, H)
    x = X.clone()
    sdp.norm_fwd("rms", x, gamma, out=(x, None, None, st()))
    assert torch.equal(x, sdp.norm_fwd("rms", X, gamma)[0])
    want = sdp.norm_bwd("layer", H, dY, gamma, mean, rstd, dH=dH)
    for place in range(3):
        ops = [t.clone() for t in (H, dY, dH)]
        got = sdp.norm_bwd("layer", ops[0], ops[1], gamma, mean, rstd, dH=ops[2], out=(ops[place], torch.empty_like(gamma), torch.empty_like(gamma)))
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    only = sdp.norm_bwd("layer", H, dY, gamma, mean, rstd, dH=dH, want_dw=False)
    assert torch.equal(only[0], want[0]) and only[1] is None and only[2] is None
    no_bias = sdp.norm_bwd("layer", H, dY, gamma, mean, rstd, dH=dH, bias=False)
    assert torch.equal(no_bias[1], want[1]) and no_bias[2] is None


def test_empty_batch(sdp):
    for dtype in DT.values():
        X, gamma = torch.empty((0, 24), dtype=dtype, device="cuda"), torch.ones(24, dtype=dtype, device="cuda")
        Y, H, mean, rstd = sdp.norm_fwd("layer", X, gamma)
        assert Y.shape == (0, 24)
        out = (torch.empty_like(X), torch.full_like(gamma, 3.0), torch.full_like(gamma, 3.0))
        sdp.norm_bwd("layer", X, X, gamma, mean, rstd, out=out)
        assert (out[1] == 0).all() and (out[2] == 0).all()


def test_a_bad_row_stays_alone_and_scratch_does_not_matter(sdp):
    """A row of infinities or NaN reaches its own outputs and the weight's gradients only; results do not depend on what the workspace held."""
    T, d = 70, 300
    X, dY = (normal(T, d, dtype=torch.bfloat16, seed=s).cuda() for s in (1, 2))
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    ref = sdp.norm_fwd("layer", X, gamma)
    bad = X.clone()
    bad[5], bad[6, 3] = float("inf"), float("nan")
    got = sdp.norm_fwd("layer", bad, gamma)
    keep = [t for t in range(T) if t not in (5, 6)]
    assert torch.equal(got[0][keep], ref[0][keep]) and got[0][5].isnan().all() and got[0][6].isnan().all()
    dX, _, _ = sdp.norm_bwd("layer", bad, dY, gamma, got[2], got[3])
    want = sdp.norm_bwd("layer", X, dY, gamma, ref[2], ref[3])
    assert torch.equal(dX[keep], want[0][keep])
    n = sdp.norm_bwd_workspace_bytes(X.dtype, T, d)
    for fill in (0, 255, 0x7F):
        again = sdp.norm_bwd("layer", X, dY, gamma, ref[2], ref[3], ws=torch.full((n,), fill, dtype=torch.uint8, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [5, 64, 100, 1200, 2050, 9001])
def test_constant_rows_whose_mean_over_their_deviation_overflows(sdp, dtype, d):
    """Rows of 2^110 throughout have variance 0, s = 1 / sqrt(1e-12) = 1e6 and xh = 0, though mu s = 1.3e39 is no fp32 value: dX, dgamma and
    dbeta are finite.  The mean is exact: a row's partial sums are small integers times 2^110.  Among other rows, alone, and last, whatever share of a
    workgroup's rows is then left without one."""
    dt, eps, half = DT[dtype], 1e-12, HALF[dtype]
    for T, at in ((1, [0]), (3, [2]), (9, [0, 4, 8]), (600, [1, 599])):
        print(f"constant rows {dtype} T={T} d={d}", flush=True)
        X, dY, dH = (normal(T, d, dtype=dt, seed=s) for s in (1, 2, 3))
        X[at] = 2.0 ** 110
        gamma = normal(d, dtype=dt, seed=4, std=0.3, mean=1.0)
        Y, H, mean, rstd = sdp.norm_fwd("layer", X.cuda(), gamma.cuda(), eps=eps)
        wY, _, wm, wr = norm_fwd64("layer", X, None, gamma, None, eps)
        assert (mean.cpu()[at] == 2.0 ** 110).all() and (Y.cpu()[at] == 0).all()
        for skip in (None, dH):
            dX, dg, db = sdp.norm_bwd("layer", H, dY.cuda(), gamma.cuda(), mean, rstd, dH=None if skip is None else skip.cuda())
            wX, wg, wb = norm_bwd64("layer", X, dY, skip, gamma, wm, wr)
            assert_close_rows(dX.cpu().double(), wX, half + 1e-5, "dX")
            if T > len(at):
                assert_close(dg.cpu().double(), wg, half + 2e-5, "dgamma")
            else:
                assert (dg == 0).all()
            assert_close(db.cpu().double(), wb, half + 2e-5, "dbeta")


def _same(got, want, tol, what):
    """Equal where the formula's value is not finite, within tol of it (or of 1) elsewhere."""
    got, fin = got.cpu().double(), want.isfinite()
    assert torch.equal(got[~fin].nan_to_num(nan=7.0), want[~fin].nan_to_num(nan=7.0)), f"{what}: values that are not finite"
    off = (got - want)[fin].abs() / want[fin].abs().clamp(min=1.0)
    assert off.numel() == 0 or off.max() <= tol, f"{what}: {float(off.max()):.2e}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 1000, 2064, 9008])
def test_weights_that_are_not_finite_count_once(sdp, dtype, d):
    """gamma's last value infinite: the root-mean-square form's dX is what the formula gives, infinities of its signs and one NaN a row, whatever
    lanes have no value of the row; dgamma and dbeta do not depend on gamma.  Widths of whole pieces, not of whole waves of them."""
    T, dt = 5, DT[dtype]
    X, dY = (normal(T, d, dtype=dt, seed=s) for s in (1, 2))
    gamma = torch.ones(d, dtype=dt)
    gamma[-1] = float("inf")
    _, H, _, rstd = sdp.norm_fwd("rms", X.cuda(), gamma.cuda(), eps=EPS)
    dX, dg, db = sdp.norm_bwd("rms", H, dY.cuda(), gamma.cuda(), None, rstd, bias=True)
    _, _, wm, wr = norm_fwd64("rms", X, None, gamma, None, EPS)
    wX, wg, wb = norm_bwd64("rms", X, dY, None, gamma, wm, wr)
    assert wX.isinf().sum() == T * (d - 1) and wX[:, -1].isnan().all()
    _same(dX, wX, 0.0, "dX")
    _same(dg, wg, HALF[dtype] + 2e-5, "dgamma")
    _same(db, wb, HALF[dtype] + 2e-5, "dbeta")


def test_a_norm_in_its_tokens_place_leaves_nothing_to_normalise_again(sdp):
    """Without a residual H is X itself.  Where Y takes X's place there is none, and the backward call says so; everywhere else the
    returned tuple is what the backward call takes."""
    T, d = 6, 40
    X, dY = (normal(T, d, seed=s).cuda() for s in (1, 2))
    gamma, st = normal(d, seed=3, mean=1.0).cuda(), lambda: torch.empty((T,), device="cuda")
    Y, H, mean, rstd = sdp.norm_fwd("layer", X, gamma)
    assert H is X
    want = sdp.norm_bwd("layer", H, dY, gamma, mean, rstd)
    Y2, H2, m2, r2 = sdp.norm_fwd("layer", X, gamma, out=(torch.empty_like(X), None, st(), st()))
    assert H2 is X and all(torch.equal(a, b) for a, b in zip(sdp.norm_bwd("layer", H2, dY, gamma, m2, r2), want))
    for view in (lambda x: x, lambda x: x.view(-1).view(T, d)):  # the same memory, the same tensor or not
        x = X.clone()
        y, h, m2, r2 = sdp.norm_fwd("layer", x, gamma, out=(view(x), None, st(), st()))
        assert torch.equal(y, Y) and h is None
        with pytest.raises(TypeError, match="H: expected a tensor"):
            sdp.norm_bwd("layer", h, dY, gamma, m2, r2)
        # with a residual H is a buffer of its own, whatever Y takes the place of
        x, r = X.clone(), dY.clone()
        y, h, m2, r2 = sdp.norm_fwd("layer", x, gamma, residual=r, out=(view(x), r, st(), st()))
        assert h is r and torch.equal(h, X + dY)
    empty = torch.empty((0, d), device="cuda")
    assert sdp.norm_fwd("rms", empty, gamma)[1] is empty
