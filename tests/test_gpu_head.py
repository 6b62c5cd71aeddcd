"""GPU parity of the output head's losses (cross-entropy and divergence from a teacher, without the logits in memory) against 64 bits: sizes around
every change of tile, odd vocabularies, tokens without a target, more tokens than one piece takes, and what is not wanted.  Bounds: targets.py."""
import pytest
import torch

from around import DT, Guarded, normal
from targets import HeadWant, entries, rest_of

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


def head(T, V, d, dt, labels, seed=0):
    """X, W: hidden states that point to their token (a logit of about 10 there), logits of deviation 2 elsewhere."""
    W = normal(V, d, dtype=dt, seed=seed + 1, std=2.0 / d ** 0.5)
    g = 2.5 * W[labels.clamp(0, V - 1)].double()
    return (normal(T, d, dtype=torch.float64, seed=seed) + g).to(dt), W


def some_labels(T, V, seed=0, pad=0.2):
    g = torch.Generator().manual_seed(seed)
    labels = torch.randint(0, V, (T,), generator=g)
    none = torch.rand(T, generator=g) < pad
    return torch.where(none, torch.where(torch.rand(T, generator=g) < 0.5, -100, V), labels)


CASES = [(1, 1, 8), (1, 2, 8), (3, 7, 8), (5, 63, 16), (17, 64, 24), (64, 65, 64), (65, 129, 72), (130, 1000, 200), (257, 1023, 256), (300, 5003, 512),
         (513, 2049, 128), (1000, 300, 40), (16, 32000, 256), (2, 50001, 64), (2049, 515, 64), (700, 4096, 1024)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", CASES)
def test_loss_matches_64_bits(sdp, T, V, d, dtype):
    dt, n = DT[dtype], T + V + d
    if dtype == "f32" and n % 2:
        d -= 1
    labels = some_labels(T, V, n, 0.2 if T > 2 else 0.0)
    X, W = head(T, V, d, dt, labels)
    X[(labels < 0) | (labels >= V)] = NAN  # tokens without a label are not looked at
    if n % 3:
        labels = labels.int()
    print(f"head loss T={T} V={V} d={d} {dtype}", flush=True)
    at = 0 if dtype == "bf16" else 1
    Xd, Wd, dX, dW = (Guarded(s, dt, at, v) for s, v in (((T, d), X), ((V, d), W), ((T, d), None), ((V, d), None)))
    nll, lse, loss = Guarded((T,), torch.float32, 1), Guarded((T,), torch.float32, 1), Guarded((1,), torch.float32, 1)
    scale = torch.tensor([0.25], device="cuda")
    ws = Guarded((sdp.head_loss_workspace_bytes(dt, T, V, d),), torch.uint8, -64 % 256, torch.tensor(255, dtype=torch.uint8))
    out = (nll.t, lse.t, dX.t, dW.t, loss.t)
    sdp.head_loss(Xd.t, Wd.t, labels.cuda(), scale=3.0, scale_dev=scale, out=out, ws=ws.t)
    torch.cuda.synchronize()
    for t in (Xd, Wd, dX, dW, nll, lse, loss, ws):
        t.check()
    assert torch.equal(Xd.t.cpu().nan_to_num(7), X.nan_to_num(7)) and torch.equal(Wd.t.cpu(), W)
    want = HeadWant(X.cuda(), W.cuda(), labels.cuda()[:, None], None, None, 1.0, 0.75)
    want.check(out)
    assert (nll.t >= 0).all()
    # what is not wanted: the other outputs to the same bounds, and dX in X's place
    a = dict(scale=3.0, scale_dev=scale)
    for kind in (dict(want_dx=False, want_dw=False), dict(want_dx=False), dict(want_dw=False)):
        got = sdp.head_loss(Xd.t, Wd.t, labels.cuda(), **a, **kind)
        assert (got[2] is None) == ("want_dx" in kind) and (got[3] is None) == ("want_dw" in kind)
        want.check(got)
    sdp.head_loss(Xd.t, Wd.t, labels.cuda(), out=(nll.t, None, Xd.t, dW.t, None), **a)
    want.check((nll.t, None, Xd.t, dW.t, None))
    Xd.check("in place")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,k", [(1, 1, 8, 1), (3, 7, 8, 20), (17, 64, 24, 64), (65, 129, 72, 7), (130, 1000, 200, 130), (257, 1023, 256, 8), (300, 5003, 512, 64),
                                     (16, 32000, 256, 33), (40, 2048, 128, 1024), (2049, 515, 64, 3)])
def test_distillation_matches_64_bits(sdp, T, V, d, k, dtype):
    dt, n = DT[dtype], T + V + d + k
    if dtype == "f32" and n % 2:
        d -= 1
    tau = (1.0, 2.0, 0.7)[n % 3]
    ids, top = entries(T, V, k, n, pad=0.3 if T > 2 else 0.0, cut=n % 2 == 0, wide=n % 4 < 2, dtype=(torch.float32, torch.bfloat16)[n % 2], twice=n % 5 == 0)
    rest = rest_of(top, ids, V, tau) if n % 3 else None
    X, W = head(T, V, d, dt, ids[:, 0].long())
    X[~(((ids >= 0) & (ids < V) & (top != -INF)).any(1))] = NAN
    print(f"head distill T={T} V={V} d={d} k={k} {dtype} tau={tau}", flush=True)
    X, W, ids, top = X.cuda(), W.cuda(), ids.cuda(), top.cuda()
    rest = None if rest is None else rest.cuda()
    a = dict(temperature=tau, top_lse=rest, scale=0.5)
    want = HeadWant(X, W, ids, top, rest, tau, 0.5)
    dX, dW = Guarded((T, d), dt), Guarded((V, d), dt)
    ws = Guarded((sdp.head_distill_workspace_bytes(dt, T, V, d, k),), torch.uint8, -64 % 256, torch.tensor(255, dtype=torch.uint8))
    f = dict(dtype=torch.float32, device="cuda")
    got = sdp.head_distill(X, W, ids, top, out=(torch.empty(T, **f), torch.empty(T, **f), dX.t, dW.t, torch.empty(1, **f)), ws=ws.t, **a)
    torch.cuda.synchronize()
    for t in (dX, dW, ws):
        t.check()
    want.check(got)
    for kind in (dict(want_dx=False, want_dw=False), dict(want_dw=False)):
        want.check(sdp.head_distill(X, W, ids, top, **a, **kind))


def _reference(X, W, ids, top, c):
    want = HeadWant(X, W, ids, top, None, 1.0, c)
    torch.cuda.synchronize()
    return want


@pytest.mark.parametrize("T,V,d", [(4096, 8192, 512), (1111, 30000, 1000), (9000, 3001, 264)])
def test_large_tiles(sdp, T, V, d):
    labels = some_labels(T, V, 1, 0.1)
    X, W = (t.cuda() for t in head(T, V, d, torch.bfloat16, labels))
    _reference(X, W, labels.cuda()[:, None], None, 1.0 / T).check(sdp.head_loss(X, W, labels.cuda(), scale=1.0 / T))


@pytest.mark.parametrize("dtype,T,V,d,live", [("bf16", 10000, 60000, 64, 1.0), ("bf16", 20000, 60000, 48, 0.7), ("bf16", 20000, 60000, 48, 0.02), ("f32", 10000, 30001, 33, 0.6),
                                                ("bf16", 600000, 5, 1000, 0.8), ("bf16", 300, 3000001, 16, 0.9), ("f32", 600, 1000001, 9, 0.9)])
def test_more_tokens_than_a_piece(sdp, dtype, T, V, d, live):
    """Two to three pieces, the later ones without a token that has a label in the third case; tokens of more bytes than their logits; a
    vocabulary that leaves a piece as few as are held in two terms."""
    dt = DT[dtype]
    labels = some_labels(T, V, 2, 1.0 - live)
    X, W = (t.cuda() for t in head(T, V, d, dt, labels))
    labels = labels.cuda()
    got = sdp.head_loss(X, W, labels, scale=1.0 / T)
    _reference(X, W, labels[:, None], None, 1.0 / T).check(got)
    again = sdp.head_loss(X, W, labels, scale=1.0 / T)
    for a, b in zip(got, again):
        assert torch.equal(a, b)


def test_empty_batch_and_no_labels(sdp):
    for dt in DT.values():
        X, W = torch.empty((0, 16), dtype=dt, device="cuda"), normal(100, 16, dtype=dt).cuda()
        labels = torch.empty((0,), dtype=torch.int64, device="cuda")
        nll, lse, dX, dW, loss = sdp.head_loss(X, W, labels)
        assert dX.shape == X.shape and (dW == 0).all() and float(loss) == 0
        for T in (3, 700):
            X = torch.full((T, 16), NAN, dtype=dt, device="cuda")
            nll, lse, dX, dW, loss = sdp.head_loss(X, W, torch.full((T,), -100, dtype=torch.int32, device="cuda"))
            assert (nll == 0).all() and (lse == 0).all() and (dX == 0).all() and (dW == 0).all() and float(loss) == 0
            kl, lse, dX, dW, loss = sdp.head_distill(X, W, torch.zeros((T, 3), dtype=torch.int32, device="cuda"), torch.full((T, 3), -INF, device="cuda"))
            assert (kl == 0).all() and (lse == 0).all() and (dX == 0).all() and (dW == 0).all() and float(loss) == 0
