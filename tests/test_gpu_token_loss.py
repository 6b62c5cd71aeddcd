"""GPU parity of the token loss against 64 bits: vocabularies around every change of tile and beyond what registers hold, rows
that start at any element or lie apart, labels that name no logit, masked logits.

Tolerances: fp32 arithmetic on top of one rounding of dZ.  The exponents (z - max) log2 e are rounded twice, and log2 e once, 2^-24 of at most 64
each (logits within 44 of the maximum; smaller terms are below 2^-64 of the sum), that is 3 x 64 x 2^-24 x ln 2 = 8e-6 relative to such a
term and 2e-6 to those that make up the sum (within 2^-16 of the largest); a sum of positive terms adds at most 128 + 6 + 16 roundings, 9e-6
(rows beyond the registers: 8 values of a piece in fp32, pieces in 64 bits, 1 + 6 + 16 roundings, 2e-6); the hardware's 2^x 1.2e-7.  So lse and nll are within 1.2e-5, dZ's terms within 2e-5 of c p beside their rounding (2^-8 bf16)."""
import math

import pytest
import torch

from around import DT, Guarded, loss64, normal

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
INF = float("inf")


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def _check(got, Z, labels, c, dtype, rows=None):
    nll, lse, dZ, loss = got
    wn, wl, wz, wloss = loss64(Z, labels, c)
    for g, w, name in ((nll, wn, "nll"), (lse, wl, "lse")):
        off = (g.cpu().double() - w).abs() / w.abs().clamp(min=1)
        assert off.max() <= 1.5e-5, f"{name}: {off.max():.2e}"
    if dZ is not None:
        live = ((labels >= 0) & (labels < Z.shape[1]))[:, None]
        p = torch.where(live, (Z.double() - wl[:, None]).exp(), 0.0)
        # at the label dz = (p - 1) c is formed as fl(c p) - fl(c): with c = scale x scale_dev[0] rounded to fp32 that is 2^-24 c more
        # than p's error and the result's rounding; 1e-37: fp32's smallest normal number
        room = HALF[dtype] * wz.abs() + 2e-5 * abs(c) * p + 2.0 ** -24 * abs(c) * (wz * c < 0) + 1e-37
        off = (dZ.cpu().double() - wz).abs()
        assert (off <= room).all(), f"dZ: {float((off / room).max()):.2f} of the bound"
    if loss is not None:
        # the sum of nll's own errors, which share no sign, and one rounding
        assert abs(float(loss) - float(wloss)) <= 1.5e-5 * abs(c) * max(1.0, float(wn.abs().sum())) + 1e-30


CASES = [(1, 1), (1, 2), (3, 7), (5, 8), (2, 9), (17, 100), (64, 1023), (40, 1024), (9, 1025), (33, 2047), (20, 2048), (7, 2049), (11, 4096), (6, 4099),
         (5, 8191), (4, 8192), (3, 8193), (6, 16384), (5, 16385), (3, 32000), (2, 32768), (2, 32769), (3, 50001), (2, 65536), (2, 65537),
         (2, 100003), (1, 131072), (2, 131073), (2, 200001), (1500, 67)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", CASES)
def test_loss_matches_64_bits(sdp, T, V, dtype):
    dt, at, wide = DT[dtype], (T + V) % 5, V % 2 == 0
    Z = normal(T, V, dtype=dt, seed=V, std=3.0)
    g = torch.Generator().manual_seed(T)
    labels = torch.randint(0, V, (T,), generator=g).to(torch.int64 if wide else torch.int32)
    if T > 2:
        labels[1], labels[2] = -1, V
    print(f"loss T={T} V={V} {dtype} at={at}", flush=True)
    dl = labels.cuda()
    Zd, dZ = Guarded((T, V), dt, at, Z), Guarded((T, V), dt, at)
    nll, lse, loss = Guarded((T,), torch.float32, 1), Guarded((T,), torch.float32, 1), Guarded((1,), torch.float32, 1)
    scale = sdp.label_scale(dl, V)
    n = int(((labels >= 0) & (labels < V)).sum())
    assert float(scale) == torch.tensor(1.0 / max(1, n), dtype=torch.float32)
    got = sdp.token_loss(Zd.t, dl, scale=3.0, scale_dev=scale, out=(nll.t, lse.t, dZ.t, loss.t))
    torch.cuda.synchronize()
    for t in (Zd, dZ, nll, lse, loss):
        t.check()
    assert torch.equal(Zd.t.cpu(), Z)
    _check(got, Z, labels, 3.0 * float(scale), dtype)
    # without a gradient, without lse and loss, and in the logits' place: the same bits
    only = sdp.token_loss(Zd.t, dl, scale=3.0, scale_dev=scale, want_grad=False)
    assert torch.equal(only[0], nll.t) and torch.equal(only[1], lse.t) and only[2] is None and torch.equal(only[3], loss.t)
    keep = dZ.t.clone()
    few = torch.empty_like(nll.t)
    sdp.token_loss(Zd.t, dl, scale=3.0, scale_dev=scale, out=(few, None, Zd.t, None))
    assert torch.equal(few, nll.t) and torch.equal(Zd.t, keep)
    Zd.check("in place")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ldz", [(7, 8), (1000, 1003), (2500, 4096), (50001, 50048), (140001, 140010)])
def test_rows_apart_keep_what_lies_between(sdp, dtype, V, ldz):
    T, dt = 5, DT[dtype]
    Z = normal(T, ldz, dtype=dt, seed=1, std=2.0)
    labels = torch.tensor([0, V - 1, -1, V, V // 2])  # V is a column between the rows, and no label
    Zd = Z.cuda()
    got = sdp.token_loss(Zd[:, :V], labels.cuda())
    _check(got, Z[:, :V].contiguous(), labels, 1.0, dtype)
    place = Zd.clone()
    sdp.token_loss(place[:, :V], labels.cuda(), out=(got[0], got[1], place[:, :V], got[3]))
    assert torch.equal(place[:, :V], got[2]) and torch.equal(place[:, V:], Zd[:, V:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 5000, 40000, 140000])
def test_masked_and_bad_logits(sdp, dtype, V):
    dt = DT[dtype]
    low = torch.finfo(dt).min
    Z = normal(10, V, dtype=dt, seed=2)
    labels = torch.tensor([3, 3, 3, 3, 3, -1, 3, 3, 3, 3])
    Z[0, 10:] = -INF  # masked
    Z[1, 3] = -INF  # the label is masked
    Z[2] = -INF  # nothing left
    Z[3, 7] = float("nan")
    Z[4, 7] = INF
    Z[5] = float("nan")  # no label: not looked at
    Z[6, 10:] = low  # masked by the type's lowest value
    Z[7] = low
    Z[8] = torch.finfo(dt).max / 4
    nll, lse, dZ, loss = sdp.token_loss(Z.cuda(), labels.cuda())
    torch.cuda.synchronize()
    clean = torch.tensor([0, 5, 6, 7, 8, 9])
    wn, wl, wz, _ = loss64(Z, labels, 1.0)
    assert torch.allclose(nll.cpu()[clean].double(), wn[clean], rtol=1.5e-5, atol=1.5e-5)
    assert torch.allclose(lse.cpu()[clean].double(), wl[clean], rtol=1.5e-5, atol=1.5e-5)
    assert torch.allclose(dZ.cpu()[clean].double(), wz[clean], rtol=HALF[dtype], atol=1.5e-5)
    assert (dZ[0, 10:] == 0).all() and (dZ[5] == 0).all() and float(nll[5]) == 0 and float(lse[5]) == 0
    assert float(nll[1]) == INF and float(dZ[1, 3]) == -1 and dZ[1].isfinite().all() and abs(float(lse[1]) - float(wl[1])) <= 1.5e-5 * float(wl[1])
    for t in (2, 3, 4):
        assert nll[t].isnan() and dZ[t].isnan().all(), t
    assert loss.isnan()


def test_gradient_matches_differences_and_rows_sum_to_zero(sdp):
    T, V = 4, 300
    Z, labels = normal(T, V, seed=3, std=2.0), torch.tensor([5, 0, 299, 17])
    _, _, dZ, _ = sdp.token_loss(Z.cuda(), labels.cuda(), scale=0.25)
    for t, j in ((0, 5), (0, 6), (1, 0), (2, 299), (3, 100)):
        f = []
        for s in (1e-6, -1e-6):
            z = Z.double()
            z[t, j] += s
            f.append(float(loss64(z, labels, 0.25)[3]))
        assert abs((f[0] - f[1]) / 2e-6 - float(dZ[t, j])) < 1e-6
    assert dZ.double().sum(1).abs().max() < 1e-5


def test_empty_batch_and_no_labels(sdp):
    for dt in DT.values():
        Z = torch.empty((0, 100), dtype=dt, device="cuda")
        labels = torch.empty((0,), dtype=torch.int32, device="cuda")
        loss = torch.full((1,), 3.0, device="cuda")
        nll, lse, dZ, loss = sdp.token_loss(Z, labels, out=(torch.empty(0, device="cuda"), None, Z, loss))
        assert float(loss) == 0 and float(sdp.label_scale(labels, 100)) == 1
        Z = torch.full((300, 100), float("nan"), dtype=dt, device="cuda")
        labels = torch.full((300,), -100, dtype=torch.int64, device="cuda")
        scale = sdp.label_scale(labels, 100)
        nll, lse, dZ, loss = sdp.token_loss(Z, labels, scale_dev=scale)
        assert float(scale) == 1 and float(loss) == 0 and (nll == 0).all() and (dZ == 0).all()


def test_many_rows(sdp):
    """The sums over rows: 100000 of them."""
    T, V = 100000, 9
    Z, labels = normal(T, V, seed=5), torch.arange(T) % 12 - 1
    scale = sdp.label_scale(labels.cuda(), V)
    assert float(scale) == torch.tensor(1.0 / int(((labels >= 0) & (labels < V)).sum()), dtype=torch.float32)
    got = sdp.token_loss(Z.cuda(), labels.cuda(), scale_dev=scale)
    _check(got, Z, labels, float(scale), "f32")


@pytest.mark.parametrize("dtype,V,tops", [("bf16", 2 ** 26 - 3, (4.71875, 1.5)), ("f32", 2 ** 25 - 3, (3.453125, 6.28125))])
def test_sums_of_long_rows_do_not_drift(sdp, dtype, V, tops):
    """Rows of zeros and one larger logit m: V - 1 equal terms exp(-m), whose roundings in a running fp32 sum all fall to the same side (1e-3 off at these
    m and V).  In closed form lse = m + log(1 + (V - 1) exp(-m)).  The sum: 3 roundings of an exponent below 9.1, 3 x 9.1 x 2^-24 x ln 2 = 1.2e-6; the
    hardware's 2^x 1.2e-7; the values of a piece, 7 roundings, 4.2e-7; 64 bits over pieces, exact here; 1 + 6 + 15 over lanes and waves, 1.3e-6: 3.1e-6
    together.  Then lse's own rounding and its logarithm's, 2^-23 of it."""
    dt, c = DT[dtype], 3.0
    Z = torch.zeros((2, V), dtype=dt, device="cuda")
    Z[0, 12345], Z[1, V - 1] = tops
    labels = torch.tensor([12345, 7], device="cuda")
    nll, lse, dZ, loss = sdp.token_loss(Z, labels, scale=c)
    for t, m in enumerate(tops):
        want = m + math.log1p((V - 1) * math.exp(-m))
        room = 3.1e-6 + 2.0 ** -23 * want
        assert abs(float(lse[t]) - want) <= room
        assert abs(float(nll[t]) - (want - float(Z[t, labels[t]]))) <= room
        p = c * math.exp(-want)
        # beside the sum's error: the quotient's, the product's and the result's own roundings
        assert abs(float(dZ[t, 99]) - p) <= (HALF[dtype] + 3.1e-6 + 2.0 ** -22) * p
    assert torch.equal(sdp.token_loss(Z, labels, want_grad=False)[1], lse)
