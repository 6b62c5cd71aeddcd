"""GPU parity of the token embedding against 64 bits: vocabularies and batches around every change of range and chunk, ids that
name no row, rows that occur in every chunk, both id types.

Tolerances, per row (relative to max(rms of the row, value)): an output is rounded once (2^-8 bf16, 2^-24 fp32); a sum of n rows in
fp32 adds at most n roundings of 2^-24 of partial sums: 16 tokens of a wave's piece, the 8 or 16 pieces of a chunk of 128 or 256 tokens, then the chunks',
one after the other up to 1024 tokens, every fourth a wave beyond: for n <= 4096, 16 + 16 + 4 or 16 + 8 + 8 + 3 of them: 2.1e-6, below 1e-5 where
partial sums are no larger than the result.  Values have one sign in the columns that are compared element by element (mean 1), so they are not."""
import pytest
import torch

from around import DT, Guarded, embed_bwd64, normal
from helpers import assert_close_rows

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def _ids(T, V, pattern, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=g)
    if pattern == "text":  # frequencies fall as 1 / rank
        ids = (V ** torch.rand(T, generator=g, dtype=torch.float64)).long().clamp(1, V) - 1
        ids = torch.randperm(V, generator=g)[ids]
    elif pattern == "one":
        ids[:] = V // 2
    elif pattern == "runs":
        ids = torch.arange(T) // 97 % V
    elif pattern == "last":
        ids = V - 1 - ids % min(V, 3)
    elif pattern == "none":
        ids[:] = -1
    elif pattern == "holes":
        ids[torch.rand(T, generator=g) < 0.5] = -1
        ids[::7] = V
        ids[::11] = -(2 ** 31)
        ids[3::13] = 2 ** 31 - 1
    return ids


CASES = [(1, 1, 1, "text"), (1, 5, 8, "text"), (2, 3, 7, "one"), (31, 300, 24, "text"), (32, 40, 256, "one"), (33, 256, 512, "one"), (64, 257, 520, "runs"),
         (65, 1000, 100, "holes"), (300, 1024, 256, "text"), (1023, 5000, 264, "holes"), (1025, 4096, 513, "last"), (4096, 977, 64, "text"),
         (4097, 32000, 72, "text"), (5000, 50001, 40, "holes"), (777, 300000, 16, "text"), (4000, 3, 1030, "text"), (3333, 2, 1, "text"),
         (2048, 100, 2048, "one"), (100, 512, 33, "none"), (20000, 700, 8, "text"), (700, 64, 1601, "runs")]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,pattern", CASES)
def test_embedding_matches_64_bits(sdp, T, V, d, pattern, dtype, wide):
    print(f"embed T={T} V={V} d={d} {pattern} {dtype} wide={wide}", flush=True)
    dt, at, scale = DT[dtype], (T + d) % 4, 1.0 if V % 2 else 7.25
    ids = _ids(T, V, pattern, T + V)
    if wide and pattern == "holes":
        ids[5::17] = 2 ** 32  # 0 in its lower half
        ids[6::17] = -(2 ** 40)
    ids = ids.to(torch.int64 if wide else torch.int32)
    E, dY = normal(V, d, dtype=dt, seed=1), normal(T, d, dtype=dt, seed=2, std=0.5, mean=1.0)
    put = lambda t: Guarded(t.shape, t.dtype, at, t).t
    Y, dE = Guarded((T, d), dt, at), Guarded((V, d), dt, at)
    dids = Guarded(ids.shape, ids.dtype, 1, ids).t
    sdp.embed_fwd(put(E), dids, scale, out=Y.t)
    sdp.embed_bwd(put(dY), dids, V, scale, out=dE.t)
    torch.cuda.synchronize()
    Y.check("Y"), dE.check("dE")
    live = (ids >= 0) & (ids < V)
    want = (E.float()[torch.where(live, ids, 0).long()] * scale).to(dt) * live[:, None]
    assert torch.equal(Y.t.cpu(), want), "one product, rounded once"
    wE = embed_bwd64(dY, ids, V, scale)
    got = dE.t.cpu().double()
    assert (got[wE.abs().sum(1) == 0] == 0).all(), "rows that do not occur are zeros"
    assert_close_rows(got, wE, HALF[dtype] + 1e-5, "dE")


def test_order_of_the_sum_is_the_tokens(sdp):
    """The same rows in other memory, in other launches: the same bits; a row's sum does not depend on what else is in the batch
    as long as it lies the same way in its chunks."""
    T, V, d = 6000, 900, 260
    ids = _ids(T, V, "text", 3).int().cuda()
    dY = normal(T, d, seed=4).cuda()
    ref = sdp.embed_bwd(dY, ids, V)
    n = sdp.embed_bwd_workspace_bytes(dY.dtype, T, V, d)
    for fill in (0, 255, 0x7F):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(sdp.embed_bwd(dY, ids, V, ws=ws), ref)
        assert torch.equal(sdp.embed_bwd(dY, ids.long(), V, ws=ws), ref)


def test_integers_are_exact(sdp):
    """Sums of small whole numbers have no rounding: every row exact, in both types, hot rows over many chunks among them."""
    T, V, d = 9000, 1300, 96
    for dtype, top in (("f32", 50), ("bf16", 1)):
        ids = _ids(T, V, "text", 5)
        if dtype == "bf16":  # sums up to 256 are whole in bf16
            ids = torch.where(torch.arange(T) % 40 == 0, ids, torch.arange(T) % V)
        g = torch.Generator().manual_seed(6)
        dY = torch.randint(-top, top + 1, (T, d), generator=g).to(DT[dtype])
        got = sdp.embed_bwd(dY.cuda(), ids.int().cuda(), V).cpu().double()
        want = embed_bwd64(dY, ids, V, 1.0)
        assert want.abs().max() <= 2 ** 24 and (dtype == "f32" or want.abs().max() <= 256)
        assert torch.equal(got, want)


def test_empty_batch_and_values_that_are_not_finite(sdp):
    for dt in DT.values():
        ids = torch.empty((0,), dtype=torch.int32, device="cuda")
        assert sdp.embed_fwd(torch.ones((4, 8), dtype=dt, device="cuda"), ids).shape == (0, 8)
        dE = torch.full((5, 8), 3.0, dtype=dt, device="cuda")
        sdp.embed_bwd(torch.empty((0, 8), dtype=dt, device="cuda"), ids, 5, out=dE)
        assert (dE == 0).all()
        # a token without an id reaches nothing, whatever it holds; one with an id only its own row
        ids = torch.tensor([2, -1, 2, 7, 1], dtype=torch.int64, device="cuda")
        dY = torch.ones((5, 8), dtype=dt, device="cuda")
        dY[1], dY[3], dY[4, 0] = float("nan"), float("inf"), float("nan")
        dE = sdp.embed_bwd(dY, ids, 5)
        assert (dE[2] == 2).all() and dE[1, 0].isnan() and (dE[1, 1:] == 1).all() and (dE[[0, 3, 4]] == 0).all()


def test_a_long_batch(sdp):
    """More tokens than one wave's piece fits in its registers, one id for most of them."""
    T, V, d = 300000, 11, 8
    ids = torch.full((T,), 4, dtype=torch.int32)
    ids[::1000] = 9
    dY = torch.ones((T, d), dtype=torch.float32)
    got = sdp.embed_bwd(dY.cuda(), ids.cuda(), V).cpu()
    assert (got[9] == 300).all() and (got[4] == T - 300).all() and got.abs().sum() == T * d


@pytest.mark.parametrize("T,V", [(1000, 50001), (60000, 50001), (60000, 700000)])
def test_ids_of_one_workgroup(sdp, T, V):
    """All tokens belong to the share of ids that one workgroup of the sort has, whatever it is: ids that agree in what deals them out, and, for any
    other deal, neighbours and ids a power of two apart.  dY is small integers: every sum is exact (below 60000 x 8 < 2^24)."""
    g = torch.Generator().manual_seed(T)
    v = torch.arange(V)
    dY = torch.randint(-8, 9, (T, 24), generator=g).float()
    for of in ((v ^ (v >> 8)) % 256 == 5, (v ^ (v >> 10)) % 1024 == 5, v % 1024 == 7, (v >= 1000) & (v < 1200)):
        share = v[of]
        ids = share[torch.randint(0, len(share), (T,), generator=g)]
        want = torch.zeros((V, 24)).index_add_(0, ids, dY)
        got = sdp.embed_bwd(dY.cuda(), ids.int().cuda(), V)
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [255, 256, 257, 271, 511, 512, 513, 767, 769, 1000, 1023, 1024, 1025, 1300])
def test_rows_that_go_over_chunks(sdp, T, dtype):
    """Few ids, so that a row's tokens reach over one, several and all chunks, begin and end at their borders and share them with others.  dY is 0
    and 1 with few enough ones that every sum is exact in both types (at most 256)."""
    g = torch.Generator().manual_seed(T)
    for V, d in ((5, 72), (3000, 67)):
        place = torch.arange(T)
        for ids in (torch.full((T,), 3), place // 256 % V, (place >= 250).long() * 2, (place * 7 // T) % V, torch.randint(0, 3, (T,), generator=g),
                    torch.where(place % 5 == 0, -1, place // 300)):
            ids = ids[torch.randperm(T, generator=g)]  # sorted order differs from theirs
            dY = (torch.rand((T, d), generator=g) < 0.1).to(DT[dtype])
            want = torch.zeros((V, d)).index_add_(0, ids[ids >= 0], dY[ids >= 0].float())
            assert want.max() <= 256
            got = sdp.embed_bwd(dY.cuda(), ids.int().cuda(), V)
            assert torch.equal(got.cpu().float(), want)
