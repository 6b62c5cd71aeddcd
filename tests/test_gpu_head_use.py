"""The output head's losses and the divergence from a teacher as they are used: behind the embedding and a norm, through the update; against
differences; under graph capture, with other numbers of tokens that have a target in every replay; on other streams and two at once; around the
number of tokens that are held in two terms; on matrices of more than 2^31 values; with values that are not finite.  Bounds: targets.py."""
import pytest
import torch

from around import DT, normal
from targets import HALF, HeadWant, Want, entries, near, rest_of, z_bound
from test_gpu_graph import _replay_against_eager
from test_gpu_head import head, some_labels

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_student_learns_from_labels_and_a_teacher(sdp, dtype):
    """Tokens -> embedding -> norm -> head: the labels' loss and the divergence from a teacher, their gradients added up, through the norm into the embedding, which
    is the head's matrix as well, and its update.  Each loss as the one on logits in memory, and all of it as in 64 bits."""
    dt, T, V, d, k, tau = DT[dtype], 300, 1001, 64, 7, 2.0
    W, gamma = normal(V, d, dtype=dt, seed=1, std=0.3), normal(d, dtype=dt, seed=2, std=0.1, mean=1.0)
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(0, V, (T,), generator=g)
    labels, (tid, top) = some_labels(T, V, 4), entries(T, V, k, 5, pad=0.2)
    Wd, gd, idd, ld, td, vd = (t.cuda() for t in (W, gamma, ids, labels, tid, top))
    n = int(((labels >= 0) & (labels < V)).sum())
    X = sdp.embed_fwd(Wd, idd)
    y, h, _, r = sdp.norm_fwd("rms", X, gd)
    scale = sdp.label_scale(ld, V)
    nll, lse, dy1, dW1, loss1 = sdp.head_loss(y, Wd, ld, scale=0.4, scale_dev=scale)
    kl, lse2, dy2, dW2, loss2 = sdp.head_distill(y, Wd, td, vd, temperature=tau, scale=0.6 * tau * tau / T)
    HeadWant(y, Wd, ld[:, None], None, None, 1.0, 0.4 * float(scale)).check((nll, lse, dy1, dW1, loss1))
    HeadWant(y, Wd, td, vd, None, tau, 0.6 * tau * tau / T).check((kl, lse2, dy2, dW2, loss2))
    # on logits that lie in memory, in fp32: the same losses
    Z = y.float() @ Wd.float().T
    zb = float(z_bound(y, Wd).max())
    assert (sdp.token_loss(Z, ld)[0] - nll).abs().max() <= 4 * zb + 1e-4 and (sdp.distill_loss(Z, td, vd, temperature=tau)[0] - kl).abs().max() <= 4 * zb + 1e-4
    dX, dg, _ = sdp.norm_bwd("rms", h, dy1 + dy2, gd, None, r)
    grad = sdp.embed_bwd(dX, idd, V) + dW1 + dW2
    # 64 bits, by differentiation: of the loss, from the same parameters
    w = W.double().requires_grad_()
    x = w[ids]
    z = (x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma.double()) @ w.T
    on = (labels >= 0) & (labels < V)
    a = torch.where(tid >= 0, top.double(), -INF)
    some = (tid >= 0).any(1)
    q, logp = (a[some] / tau).softmax(1), (z[some] / tau).log_softmax(1)
    want = 0.4 * torch.nn.functional.cross_entropy(z[on], labels[on]) + 0.6 * tau * tau / T * torch.special.xlogy(q, q).sub(q * logp.gather(1, tid[some].long().clamp(min=0))).sum()
    want.backward()
    # a chain of embedding, norm, head and back, each rounded to the type: 8 roundings of half a step, of which an element of the norm's gradient may keep the largest
    # factor, 3 (1e-5 a step in fp32, whose contractions count)
    tol = 24 * HALF[dt] if dtype == "bf16" else 8e-5
    assert abs(float(loss1) + float(loss2) - float(want.detach())) <= tol * abs(float(want.detach()))
    assert float((grad.cpu().double() - w.grad).norm() / w.grad.norm()) <= tol
    mask = torch.ones((1, V), dtype=torch.uint8, device="cuda")
    theta, m, v = Wd.float(), torch.zeros((V, d), device="cuda"), torch.zeros((V, d), device="cuda")
    sdp.coverage_avg_adamw([grad.contiguous()], mask, theta, m, v, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, step=1)
    assert torch.allclose(m, 0.1 * grad.float(), rtol=1e-5, atol=1e-12)


def test_gradients_match_differences(sdp):
    T, V, d, k, tau = 6, 150, 24, 5, 2.0
    X, W = normal(T, d, seed=1), normal(V, d, seed=2, std=0.4)
    labels, (ids, top) = torch.tensor([3, -1, 149, 0, 77, 3]), entries(T, V, k, 3)
    ids[2] = -1
    rest = rest_of(top, ids, V, tau)
    calls = [(lambda x, w: sdp.head_loss(x, w, labels.cuda(), scale=0.5), labels[:, None], None, None, 1.0)]
    for r in (None, rest):
        calls.append((lambda x, w, r=r: sdp.head_distill(x, w, ids.cuda(), top.cuda(), temperature=tau, top_lse=None if r is None else r.cuda(), scale=0.5), ids, top, r, tau))
    for call, i, v, r, t in calls:
        for dt, half in ((torch.float32, 1e-6), (torch.bfloat16, 2.0 ** -8)):
            x, w = X.to(dt).double(), W.to(dt).double()
            _, _, dX, dW, _ = call(X.to(dt).cuda(), W.to(dt).cuda())
            f = lambda a, b: float(Want(a @ b.T, i, v, r, t, 0.5).loss)
            for row, col in ((0, 0), (1, 5), (2, 23), (5, 7), (3, 11)):
                for what, got in ((0, dX), (1, dW)):
                    p = [[x.clone(), w.clone()] for _ in range(2)]
                    at = row if what == 0 else (3, 149, 10, int(ids[0, 1]), 77)[row % 5]
                    p[0][what][at, col] += 1e-6
                    p[1][what][at, col] -= 1e-6
                    slope = (f(*p[0]) - f(*p[1])) / 2e-6
                    # the difference's own error 1e-8; the result's rounding; terms that cancel in it, within 1e-3 (two terms, 2^-17, and a code's 5.2e-4 of each)
                    assert abs(slope - float(got[at, col])) <= half * abs(slope) + (2e-6 if dt == torch.float32 else 1e-3 * float(got.abs().max())) + 1e-8


def _step(sdp, T, V, d, k, dt):
    e = lambda *s, t=dt: torch.empty(s, dtype=t, device="cuda")
    f32 = torch.float32
    X, W, labels, ids, top, rest, Z = e(T, d), e(V, d), e(T, t=torch.int64), e(T, k, t=torch.int32), e(T, k, t=f32), e(T, t=f32), e(T, V)
    one, two, three = ((e(T, t=f32), e(T, t=f32), e(T, d), e(V, d), e(1, t=f32)) for _ in range(3))
    four = (e(T, t=f32), e(T, t=f32), e(T, V), e(1, t=f32))
    scale = e(1, t=f32)
    ws = torch.empty(max(sdp.head_loss_workspace_bytes(dt, T, V, d), sdp.head_distill_workspace_bytes(dt, T, V, d, k)), dtype=torch.uint8, device="cuda")

    def run():
        sdp.label_scale(labels, V, out=scale)
        sdp.head_loss(X, W, labels, scale_dev=scale, out=one, ws=ws)
        sdp.head_distill(X, W, ids, top, temperature=2.0, scale_dev=scale, out=two, ws=ws)  # the same workspace: one call after the other
        sdp.head_distill(X, W, ids, top, temperature=1.5, top_lse=rest, want_dw=False, out=three, ws=ws)
        sdp.distill_loss(Z, ids, top, temperature=2.0, scale_dev=scale, out=four)

    g = torch.Generator(device="cuda").manual_seed(T)

    def draw(live):
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        on = torch.rand(T, generator=g, device="cuda") < live
        lab = torch.where(on, torch.randint(0, V, (T,), generator=g, device="cuda"), -100)
        tid = torch.where(on[:, None], torch.randint(0, V, (T, k), generator=g, device="cuda"), V).int()
        return r(T, d).to(dt), (r(V, d) * 2 / d ** 0.5).to(dt), lab, tid, r(T, k), r(T) + 3.0, r(T, V).to(dt)

    outputs = [scale, *one, *two, *three[:3], three[4], *four]
    return run, (X, W, labels, ids, top, rest, Z), draw, outputs, ws


@pytest.mark.parametrize("T,V,d,k,dt", [(40, 120, 64, 3, torch.float32), (2100, 700, 264, 9, torch.bfloat16), (300, 1077, 72, 70, torch.bfloat16), (100, 2000, 128, 5, torch.bfloat16),
                                        (1500, 900, 33, 4, torch.float32)])
def test_replays_like_eager(sdp, T, V, d, k, dt):
    """Two variants: most tokens have a target, or few (fewer than are held in two terms)."""
    run, inputs, draw, outputs, _ = _step(sdp, T, V, d, k, dt)
    _replay_against_eager(run, inputs, [draw(0.9), draw(0.04)], outputs)


def test_two_graphs_share_a_workspace(sdp):
    steps = [_step(sdp, *s, torch.bfloat16) for s in ((1300, 300, 128, 5), (400, 1900, 72, 9))]
    ws = max((s[4] for s in steps), key=lambda t: t.numel())
    refs, graphs = [], []
    for run, inputs, draw, outputs, own in steps:
        for cell in run.__closure__:
            if cell.cell_contents is own:
                cell.cell_contents = ws
        for dst, src in zip(inputs, draw(0.7)):
            dst.copy_(src)
        run()
        torch.cuda.synchronize()
        refs.append([o.clone() for o in outputs])
    for run, *_ in steps:
        graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            with torch.cuda.graph(graph, stream=s):
                run()
        graphs.append(graph)
    torch.cuda.synchronize()
    for i in (0, 1, 1, 0, 1, 0):
        for o in steps[i][3]:
            o.fill_(NAN)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o.view(torch.uint8), r.view(torch.uint8)) for o, r in zip(steps[i][3], refs[i]))


def test_on_other_streams_two_at_once(sdp):
    steps = [_step(sdp, 1200, 800, 136, 6, torch.bfloat16), _step(sdp, 90, 3000, 64, 6, torch.float32)]
    refs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for run, inputs, draw, outputs, _ in steps:
        for dst, src in zip(inputs, draw(0.8)):
            dst.copy_(src)
        run()
        torch.cuda.synchronize()
        refs.append([o.clone() for o in outputs])
        for o in outputs:
            o.fill_(NAN)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (run, *_) in zip(streams, steps):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, _, _, outputs, _), ref in zip(steps, refs):
        assert all(torch.equal(o, r) for o, r in zip(outputs, ref))


@pytest.mark.parametrize("T,live", [(127, 127), (128, 128), (129, 129), (255, 128), (256, 129), (257, 128), (600, 127), (600, 128), (600, 129), (600, 1), (3000, 100), (33, 5)])
def test_two_terms_for_few_tokens(sdp, T, live):
    """Around the number of tokens whose gradient is held in two terms: to these terms' bounds up to it."""
    V, d = 1003, 200
    labels = torch.full((T,), -1)
    at = torch.randperm(T, generator=torch.Generator().manual_seed(T))[:live]
    labels[at] = torch.randint(0, V, (live,), generator=torch.Generator().manual_seed(live))
    X, W = (t.cuda() for t in head(T, V, d, torch.bfloat16, labels))
    X[labels.cuda() < 0] = NAN
    want = HeadWant(X, W, labels.cuda()[:, None], None, None, 1.0, 1.0 / live)
    got = sdp.head_loss(X, W, labels.cuda(), scale=1.0 / live)
    want.check(got)
    want.check(sdp.head_loss(X, W, labels.cuda(), scale=1.0 / live, want_dx=False))
    want.check(sdp.head_loss(X, W, labels.cuda(), scale=1.0 / live, want_dw=False))
    ids, top = labels[:, None].repeat(1, 3).int(), torch.zeros((T, 3))
    ids[:, 2] = -1  # a teacher that knows one id twice: the label
    ids, top = ids.cuda(), top.cuda()
    again = sdp.head_distill(X, W, ids, top, scale=1.0 / live)
    HeadWant(X, W, ids, top, None, 1.0, 1.0 / live).check(again)  # (kl counts each entry with its own log q)
    near(again[2], want.dX, want.dX_room, "dX")
    near(again[3], want.dW, want.dW_room, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.05, 20.0])
def test_temperatures(sdp, dtype, tau):
    T, V, d, k = 200, 700, 64, 9
    dt = DT[dtype]
    ids, top = entries(T, V, k, 1)
    X, W = (t.cuda() for t in head(T, V, d, dt, ids[:, 0].long()))
    X = (X.float() * min(1.0, tau * 2)).to(dt)  # logits over tau of the size of others
    top = top * min(1.0, tau * 2)
    ids, top = ids.cuda(), top.cuda()
    HeadWant(X, W, ids, top, None, tau, tau * tau).check(sdp.head_distill(X, W, ids, top, temperature=tau, scale=tau * tau))
    Z = (X.float() @ W.float().T).to(dt)
    w = Want(Z.double(), ids, top, None, tau, tau * tau, stored=dt)
    kl, lse, dZ, loss = sdp.distill_loss(Z, ids, top, temperature=tau, scale=tau * tau)
    w.rows(kl, lse, loss)
    near(dZ, w.dz, w.dz_room + 1e-300, "dZ")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales(sdp, dtype):
    """A factor of any size comes in fp32: the gradients of scale 1 times it, to twice the result's rounding."""
    T, V, d, dt = 150, 300, 64, DT[dtype]
    labels = some_labels(T, V, 1)
    X, W = (t.cuda() for t in head(T, V, d, dt, labels))
    one = sdp.head_loss(X, W, labels.cuda())
    for c in (2.0 ** 20, -(2.0 ** -30), 3.0, 0.0):
        got = sdp.head_loss(X, W, labels.cuda(), scale=c)
        assert torch.equal(got[0], one[0]) and abs(float(got[4]) - c * float(one[4])) <= 2.0 ** -22 * abs(c * float(one[4]))
        for a, b in ((got[2], one[2]), (got[3], one[3])):
            room = 2 * HALF[dt] * abs(c) * b.double().abs() + abs(c) * (0.0 if dtype == "bf16" else 1e-5 * float(b.abs().max()))
            assert ((a.double() - c * b.double()).abs() <= room).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [20, 500])
def test_values_that_are_not_finite(sdp, dtype, T):
    """A bad token spoils its own row and dW, which sums over it; a bad row of the head spoils all."""
    V, d, dt = 400, 64, DT[dtype]
    labels = some_labels(T, V, 1, 0.1)
    labels[3], labels[7] = 5, 9
    X, W = (t.cuda() for t in head(T, V, d, dt, labels))
    clean = sdp.head_loss(X, W, labels.cuda())
    bad = X.clone()
    bad[3, 10] = NAN
    bad[7, 0] = INF
    nll, lse, dX, dW, loss = sdp.head_loss(bad, W, labels.cuda())
    others = torch.ones(T, dtype=torch.bool)
    others[[3, 7]] = False
    assert torch.equal(nll.cpu()[others], clean[0].cpu()[others]) and torch.equal(dX.cpu()[others], clean[2].cpu()[others])
    assert nll[3].isnan() and nll[7].isnan() and dX[3].isnan().all() and dX[7].isnan().all() and dW.isnan().all() and loss.isnan()
    bad = W.clone()
    bad[100] = NAN
    nll, lse, dX, dW, loss = sdp.head_loss(X, bad, labels.cuda())
    on = ((labels >= 0) & (labels < V))
    assert nll.cpu()[on].isnan().all() and dX.cpu()[on].isnan().all() and (dX.cpu()[~on] == 0).all() and (nll.cpu()[~on] == 0).all()


def test_one_id_many_times(sdp):
    """1024 entries of one id are the label; of two ids, two."""
    T, V, d = 40, 500, 64
    for dt in DT.values():
        ids = torch.full((T, 1024), 7, dtype=torch.int64)
        ids[:, 600:] = 8 + torch.arange(T)[:, None]
        top = torch.randn((T, 1024), generator=torch.Generator().manual_seed(1))
        X, W = (t.cuda() for t in head(T, V, d, dt, ids[:, 0]))
        ids, top = ids.cuda(), top.cuda()
        HeadWant(X, W, ids, top, None, 1.0, 1.0).check(sdp.head_distill(X, W, ids, top))


def test_offsets_past_32_bits(sdp):
    """Matrices of more than 2^31 values: sampled rows against 64 bits, the last ones among them."""
    big = dict(dtype=torch.bfloat16, device="cuda")
    print("distill 70000 x 32003", flush=True)
    T, V, k = 70000, 32003, 3
    Z = torch.randn((T, V), **big)
    ids = (torch.arange(T * k, device="cuda").view(T, k) * 7919) % V
    top = torch.randn((T, k), device="cuda")
    ids[T - 2] = -1
    kl, lse, dZ, loss = sdp.distill_loss(Z, ids, top, scale=2.0)
    rows = torch.tensor([0, 5, 34999, 67100, 67109, T - 3, T - 2, T - 1]).cuda()
    w = Want(Z[rows].double(), ids[rows], top[rows], None, 1.0, 2.0, stored=torch.bfloat16)
    w.rows(kl[rows], lse[rows], None)
    near(dZ[rows], w.dz, w.dz_room + 1e-300, "dZ")
    assert abs(float(loss) - 2.0 * float(kl.double().sum())) <= 1e-6 * float(loss)
    del Z, dZ, ids, top

    print("head 1050000 x 2040", flush=True)
    V, d, T = 1050000, 2040, 40  # W of 4.28 GB: byte offsets up to 2^32
    W = torch.randn((V, d), **big) * 0.05
    labels = (torch.arange(T, device="cuda") * 26923) % V
    labels[-1], labels[5] = V - 1, -1
    X = torch.randn((T, d), **big)
    nll, lse, dX, dW, loss = sdp.head_loss(X, W, labels, scale=1.0)
    z = torch.cat([X.double() @ W[i: i + 50000].double().T for i in range(0, V, 50000)], 1)
    w = Want(z, labels[:, None], None, None, 1.0, 1.0, float((d / 8 + 8) * 2.0 ** -24 * d * 0.05 * 2), torch.bfloat16, codes=True, half=2.0 ** -17)
    w.rows(nll, lse, loss)
    want = sum(w.dz[:, i: i + 50000] @ W[i: i + 50000].double() for i in range(0, V, 50000))
    room = sum((w.dz_room[:, i: i + 50000] + V / 8 * 2.0 ** -24 * w.dz[:, i: i + 50000].abs()) @ W[i: i + 50000].double().abs() for i in range(0, V, 50000))
    near(dX, want, room + 2.0 ** -8 * want.abs() + 1e-37, "dX")
    for v in (0, 5, 526343, 526345, 1048575, 1048576, V - 2, V - 1, int(labels[7])):
        x = X.double()
        near(dW[v], w.dz[:, v] @ x, (w.dz_room[:, v] + 16 * 2.0 ** -24 * w.dz[:, v].abs()) @ x.abs() + 2.0 ** -8 * (w.dz[:, v] @ x).abs() + 1e-37, f"dW[{v}]")


@pytest.mark.parametrize("T,V,d", [(2932, 348636, 88), (34417, 10808, 336), (38275, 2254, 1872), (130, 3000001, 16)])
def test_a_last_piece_of_fewer_tokens(sdp, T, V, d):
    """Two pieces, the second of so many tokens less that a call of as many would run in other tiles: 1460 after 1472, 17201 after 17216, 19075 after 19200, and
    2 after 128."""
    labels = (torch.arange(T, device="cuda") * 7919) % V
    X, W = normal(T, d, dtype=torch.bfloat16, seed=3).cuda(), normal(V, d, dtype=torch.bfloat16, seed=4, std=1.5 / d ** 0.5).cuda()
    print(f"head T={T} V={V} d={d}", flush=True)
    got = sdp.head_loss(X, W, labels, scale=1.0 / T)
    HeadWant(X, W, labels[:, None], None, None, 1.0, 1.0 / T).check(got)


def test_more_workgroups_than_a_row_of_the_grid(sdp):
    T, V, d = 1200007, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    Z = torch.randn((T, V), generator=g, device="cuda")
    ids = (torch.arange(T, device="cuda") % V)[:, None].int()
    top = torch.zeros((T, 1), device="cuda")
    rows = torch.tensor([0, 1048575, 1048576, T - 1]).cuda()
    kl, lse, dZ, _ = sdp.distill_loss(Z, ids, top)
    w = Want(Z[rows].double(), ids[rows], top[rows], None, 1.0, 1.0)
    w.rows(kl[rows], lse[rows], None)
    near(dZ[rows], w.dz, w.dz_room, "dZ")
    for dt in DT.values():
        X, W = Z.to(dt), torch.randn((V, d), generator=g, device="cuda").to(dt)
        for got in (sdp.head_loss(X, W, ids[:, 0]), sdp.head_distill(X, W, ids, top)):
            w = HeadWant(X[rows], W, ids[rows], None, None, 1.0, 1.0)
            w.rows(got[0][rows], got[1][rows], None)
            # more than 128 tokens: one term
            near(got[2][rows], w.dX, w.dX_room + HALF[dt] * w.dz.abs() @ W.double().abs(), "dX")
            full = HeadWant(X, W, ids, None, None, 1.0, 1.0)
            near(got[3], full.dW, full.dW_room, "dW")
