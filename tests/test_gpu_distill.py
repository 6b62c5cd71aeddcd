"""GPU parity of the divergence from a teacher's top logits against 64 bits: vocabularies around every change of tile and beyond what registers
hold, 1 to 1024 entries, entries that name no token, the same token twice, rows that start at any element or lie apart, masked logits.
Bounds: targets.py."""
import pytest
import torch

from around import DT, Guarded, normal
from targets import HALF, Want, entries, near, rest_of

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


CASES = [(1, 1, 1), (1, 2, 3), (3, 7, 7), (5, 8, 1), (2, 9, 20), (17, 100, 64), (64, 1023, 65), (20, 2048, 5), (7, 2049, 130), (6, 4099, 300), (4, 8192, 1024),
         (3, 8193, 2), (5, 16385, 64), (3, 32000, 64), (2, 32769, 100), (3, 50001, 20), (2, 65537, 64), (1, 131072, 9), (2, 131073, 1000), (1500, 67, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,k", CASES)
def test_matches_64_bits(sdp, T, V, k, dtype):
    dt, at, n = DT[dtype], (T + V) % 5, T + V + k
    tau = (1.0, 2.0, 0.7)[n % 3]
    Z = normal(T, V, dtype=dt, seed=V, std=3.0)
    ids, top = entries(T, V, k, n, pad=0.3 if T > 2 else 0.0, cut=n % 2 == 0, wide=n % 4 < 2, dtype=(torch.float32, torch.bfloat16)[n % 2], twice=n % 5 == 0)
    rest = rest_of(top, ids, V, tau) if n % 3 else None
    print(f"distill T={T} V={V} k={k} {dtype} tau={tau} at={at}", flush=True)
    scale = torch.tensor([0.25], device="cuda")
    Zd, dZ = Guarded((T, V), dt, at, Z), Guarded((T, V), dt, at)
    kl, lse, loss = Guarded((T,), torch.float32, 1), Guarded((T,), torch.float32, 1), Guarded((1,), torch.float32, 1)
    di, dv, dr = cuda(ids, top, rest)
    a = dict(temperature=tau, top_lse=dr, scale=3.0, scale_dev=scale)
    sdp.distill_loss(Zd.t, di, dv, out=(kl.t, lse.t, dZ.t, loss.t), **a)
    torch.cuda.synchronize()
    for t in (Zd, dZ, kl, lse, loss):
        t.check()
    assert torch.equal(Zd.t.cpu(), Z)
    w = Want(Z.double(), ids, top, rest, tau, 0.75, stored=dt)
    w.rows(kl.t, lse.t, loss.t)
    near(dZ.t, w.dz, w.dz_room + 1e-300, "dZ")
    # without a gradient, without lse and loss, and in the logits' place: the same bits
    only = sdp.distill_loss(Zd.t, di, dv, want_grad=False, **a)
    assert torch.equal(only[0], kl.t) and torch.equal(only[1], lse.t) and only[2] is None and torch.equal(only[3], loss.t)
    keep, few = dZ.t.clone(), torch.empty_like(kl.t)
    sdp.distill_loss(Zd.t, di, dv, out=(few, None, Zd.t, None), **a)
    assert torch.equal(few, kl.t) and torch.equal(Zd.t, keep)
    Zd.check("in place")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ldz", [(7, 8), (1000, 1003), (2500, 4096), (50001, 50048), (140001, 140010)])
def test_rows_apart_keep_what_lies_between(sdp, dtype, V, ldz):
    T, dt = 5, DT[dtype]
    Z = normal(T, ldz, dtype=dt, seed=1, std=2.0)
    ids, top = entries(T, V, 6, V)
    ids[1], ids[2, 0], ids[3, 1] = -1, V, V  # V is a column between the rows, and no token
    Zd = Z.cuda()
    di, dv = cuda(ids, top)
    got = sdp.distill_loss(Zd[:, :V], di, dv)
    w = Want(Z[:, :V].double(), ids, top, None, 1.0, 1.0, stored=dt)
    w.rows(got[0], got[1], got[3])
    near(got[2], w.dz, w.dz_room + 1e-300, "dZ")
    place = Zd.clone()
    sdp.distill_loss(place[:, :V], di, dv, out=(got[0], got[1], place[:, :V], got[3]))
    assert torch.equal(place[:, :V], got[2]) and torch.equal(place[:, V:], Zd[:, V:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 5000, 140000])
def test_masked_and_bad_logits(sdp, dtype, V):
    dt = DT[dtype]
    low = torch.finfo(dt).min
    T = 14
    Z = normal(T, V, dtype=dt, seed=2)
    ids, top = torch.tensor([[3, 9, 5]] * T, dtype=torch.int32), torch.tensor([[2.0, 1.0, 0.5]] * T)
    Z[0, 10:] = -INF  # masked
    Z[1, 9] = -INF  # an entry is masked
    Z[2] = -INF  # nothing left
    Z[3, 7], Z[4, 7] = NAN, INF
    Z[5], ids[5] = NAN, -1  # no entry: not looked at
    Z[6, 10:] = low  # masked by the type's lowest value
    Z[7] = low
    Z[8] = torch.finfo(dt).max / 4
    top[9, 1] = -INF  # no entry
    Z[10], top[10] = NAN, -INF
    top[11, 2] = NAN
    ids[12], top[12] = torch.tensor([3, 3, 3]), torch.tensor([1.0, 2.0, 3.0])
    Z[13, 9], top[13, 1] = -INF, -INF  # masked, and no entry
    kl, lse, dZ, loss = sdp.distill_loss(Z.cuda(), *cuda(ids, top))
    torch.cuda.synchronize()
    clean = torch.tensor([0, 5, 6, 7, 8, 9, 10, 12, 13])
    w = Want(Z[clean].double(), ids[clean], top[clean], None, 1.0, 1.0, stored=dt)
    w.rows(kl[clean], lse[clean], None)
    near(dZ[clean], w.dz, w.dz_room + 1e-300, "dZ")
    for t in (5, 10):
        assert float(kl[t]) == 0 and float(lse[t]) == 0 and (dZ[t] == 0).all()
    assert (dZ[0, 10:] == 0).all() and float(kl[1]) == INF and dZ[1].isfinite().all() and float(dZ[1, 9]) < -0.2
    for t in (2, 3, 4, 11):
        assert kl[t].isnan() and dZ[t].isnan().all(), t
    assert loss.isnan()
    # the log-sum of a teacher that is not a number, and one without an end: nothing is known of its entries
    rest = torch.tensor([NAN, INF, 3.0]).cuda()
    kl, lse, dZ, _ = sdp.distill_loss(Z[[0, 0, 0]].cuda(), ids[:3].cuda(), top[:3].cuda(), top_lse=rest)
    assert kl[0].isnan() and dZ[0].isnan().all() and float(kl[1]) == 0 and (dZ[1] == 0).all() and kl[2].isfinite()


def test_gradient_matches_differences_and_rows_sum_to_zero(sdp):
    T, V, tau, c = 4, 300, 2.0, 0.25
    Z = normal(T, V, seed=3, std=2.0)
    ids, top = entries(T, V, 5, 3)
    rest = rest_of(top, ids, V, tau)
    for r in (None, rest):
        dZ = sdp.distill_loss(Z.cuda(), *cuda(ids, top), temperature=tau, top_lse=None if r is None else r.cuda(), scale=c)[2]
        for t, j in ((0, int(ids[0, 0])), (0, 6), (1, int(ids[1, 4])), (2, 299), (3, 100)):
            f = []
            for s in (1e-6, -1e-6):
                z = Z.double()
                z[t, j] += s
                f.append(float(Want(z, ids, top, r, tau, c).loss))
            assert abs((f[0] - f[1]) / 2e-6 - float(dZ[t, j])) < 1e-6
        assert dZ.double().sum(1).abs().max() < 1e-5


def test_one_entry_is_a_label(sdp):
    """A single entry, renormalised, has all the mass: the token loss, to the bounds of both."""
    for dtype, dt in DT.items():
        Z = normal(50, 4099, dtype=dt, seed=4, std=3.0).cuda()
        labels = torch.randint(-1, 4099, (50,), generator=torch.Generator().manual_seed(1)).cuda()
        got = sdp.distill_loss(Z, labels[:, None], torch.full((50, 1), 5.0, device="cuda"), scale=0.5)
        want = sdp.token_loss(Z, labels, scale=0.5)
        assert torch.allclose(got[0], want[0], rtol=4 * 2.0 ** -24, atol=4e-5) and torch.allclose(got[1], want[1], rtol=4 * 2.0 ** -24, atol=4e-5)
        assert torch.allclose(got[2].double(), want[2].double(), rtol=2 * HALF[dt], atol=2e-5)


def test_empty_batch_and_no_teacher(sdp):
    for dt in DT.values():
        Z = torch.empty((0, 100), dtype=dt, device="cuda")
        ids, top = torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), device="cuda")
        loss = torch.full((1,), 3.0, device="cuda")
        assert float(sdp.distill_loss(Z, ids, top, out=(torch.empty(0, device="cuda"), None, Z, loss))[3]) == 0
        Z = torch.full((300, 100), NAN, dtype=dt, device="cuda")
        ids, top = torch.full((300, 4), 100, dtype=torch.int64, device="cuda"), torch.zeros((300, 4), dtype=torch.bfloat16, device="cuda")
        kl, lse, dZ, loss = sdp.distill_loss(Z, ids, top)
        assert float(loss) == 0 and (kl == 0).all() and (lse == 0).all() and (dZ == 0).all()
