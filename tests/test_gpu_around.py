"""Norms, embedding and token loss as they are used: around the masked attention and MLP of two workers, through the update; under graph
capture; on another stream; on matrices of more than 2^31 values."""
import math

import numpy as np
import pytest
import torch

import workloads
from around import embed_bwd64, loss64, norm_bwd64, norm_fwd64
from helpers import err_report
from test_gpu_graph import _replay_against_eager

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


Bt, S, d, F, H, hd, V, K = 2, 24, 64, 128, 4, 16, 101, 2
T = Bt * S


def _model(dtype, seed=3):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=0.1, mean=0.0: (torch.randn(s, generator=g, dtype=torch.float64) * std + mean).to(dtype)
    return dict(E=n(V, d, std=0.5), Wqkv=n(3, H * hd, d), WoT=n(H * hd, d), W1=n(F, d), W3=n(F, d), W2T=n(F, d), W=n(V, d, std=0.2),
                g1=n(d, std=0.2, mean=1.0), b1=n(d), g2=n(d, std=0.2, mean=1.0), b2=n(d), g3=n(d, std=0.2, mean=1.0))


def _batch(k, seed=9):
    g = torch.Generator().manual_seed(seed + k)
    ids = torch.randint(0, V, (T,), generator=g)
    labels = torch.randint(0, V, (T,), generator=g)
    ids[T - 3:] = -1  # padding at the end of the last sequence, and positions that are not trained on
    labels[T - 4:] = -1
    labels[:5] = -100
    return ids, labels


def _step(sdp, P, heads, neurons, ids, labels):
    """One worker: embedding -> norm -> attention -> + , norm -> MLP -> +, norm -> logits -> mean loss, and back.  -> loss, gradients."""
    X = sdp.embed_fwd(P["E"], ids, math.sqrt(d))
    y1, h1, m1, r1 = sdp.norm_fwd("layer", X, P["g1"], P["b1"], eps=EPS)
    a, QKV, O, LSE = sdp.masked_attn_fwd("fm", Bt, S, hd, y1, P["Wqkv"], P["WoT"], heads)
    y2, h2, m2, r2 = sdp.norm_fwd("layer", a, P["g2"], P["b2"], residual=h1, eps=EPS)
    f, G, U = sdp.masked_mlp_fwd("fm", y2, P["W1"], P["W3"], P["W2T"], neurons)
    y3, h3, _, r3 = sdp.norm_fwd("rms", f, P["g3"], residual=h2, eps=EPS)
    Z = y3 @ P["W"].T
    _, _, dZ, loss = sdp.token_loss(Z, labels, scale_dev=sdp.label_scale(labels, V))
    dy3, dW = dZ @ P["W"], dZ.T @ y3
    dh3, dg3, _ = sdp.norm_bwd("rms", h3, dy3, P["g3"], None, r3)
    out = lambda *names: tuple(torch.zeros_like(P[n]) for n in names)  # scattered: rows off the masks stay zeros
    dy2, dW1, dW3, dW2T = sdp.masked_mlp_bwd("fm", y2, dh3, P["W1"], P["W3"], P["W2T"], neurons, G, U, dw_layout="scatter",
                                             out=(torch.empty_like(y2),) + out("W1", "W3", "W2T"))
    dh2, dg2, db2 = sdp.norm_bwd("layer", h2, dy2, P["g2"], m2, r2, dH=dh3)
    dy1, dWqkv, dWoT = sdp.masked_attn_bwd("fm", Bt, S, hd, y1, dh2, P["Wqkv"], P["WoT"], heads, QKV, O, LSE, dw_layout="scatter",
                                           out=(torch.empty_like(y1),) + out("Wqkv", "WoT"))
    dX, dg1, db1 = sdp.norm_bwd("layer", h1, dy1, P["g1"], m1, r1, dH=dh2)
    dE = sdp.embed_bwd(dX, ids, V, math.sqrt(d))
    return loss, dict(E=dE, Wqkv=dWqkv, WoT=dWoT, W1=dW1, W3=dW3, W2T=dW2T, W=dW, g1=dg1, b1=db1, g2=dg2, b2=db2, g3=dg3)


def _step64(P, head_mask, neuron_mask, ids, labels):
    """The same in 64 bits with autograd, masks as products."""
    P = {k: v.double().requires_grad_() for k, v in P.items()}
    hm = torch.from_numpy(np.repeat(head_mask, hd).astype(np.float64))[:, None]
    nm = torch.from_numpy(neuron_mask.astype(np.float64))[:, None]
    live = (ids >= 0)[:, None]
    X = P["E"][ids.clamp(min=0)] * math.sqrt(d) * live

    def layer(h, g, b):
        c = h - h.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + EPS).sqrt() * g + b

    y1 = layer(X, P["g1"], P["b1"])
    q, k, v = ((y1 @ (P["Wqkv"][i] * hm).T).view(Bt, S, H, hd).transpose(1, 2) for i in range(3))
    p = (q @ k.transpose(2, 3) / math.sqrt(hd)).masked_fill(torch.ones(S, S).triu(1).bool(), -math.inf).softmax(3)
    h2 = X + (p @ v).transpose(1, 2).reshape(T, H * hd) @ (P["WoT"] * hm)
    y2 = layer(h2, P["g2"], P["b2"])
    G, U = y2 @ (P["W1"] * nm).T, y2 @ (P["W3"] * nm).T
    h3 = h2 + (torch.nn.functional.silu(G) * U) @ (P["W2T"] * nm)
    y3 = h3 / (h3.square().mean(1, keepdim=True) + EPS).sqrt() * P["g3"]
    on = (labels >= 0) & (labels < V)
    loss = torch.nn.functional.cross_entropy(y3[on] @ P["W"].T, labels[on])
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in P.items()}


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 5e-2)])
def test_a_step_of_two_workers_with_its_update(sdp, orc, dtype, tol):
    """fp32: every gradient of a chain of nine operators, each within 1e-5 (1e-5 x 9).  bf16: about 20 roundings of at most 2^-8, 2^-9.6 rms each,
    on the way there and back, amplified by the norms at most tenfold: 20^0.5 x 10 x 2^-9.6 = 5.8e-2 of the norm if all were at the worst place."""
    P = _model(dtype)
    Pd = {k: v.cuda() for k, v in P.items()}
    hmask, heads, _, _ = sdp.make_masks(K, H, 3, 11, True)
    nmask, neurons, _, _ = sdp.make_masks(K, F, 96, 12, True)
    grads, want = [], []
    for k in range(K):
        ids, labels = _batch(k)
        loss, g = _step(sdp, Pd, heads[k], neurons[k], ids.cuda(), labels.int().cuda())
        wloss, wg = _step64(P, hmask[k].cpu().numpy(), nmask[k].cpu().numpy(), ids, labels)
        torch.cuda.synchronize()
        assert abs(float(loss) - wloss) <= tol * wloss
        for name in P:
            assert err_report(g[name].cpu().double(), wg[name])[1] <= tol, name
        grads.append(g)
        want.append(wg)
    # the update of the embedding and of a norm's weight: every worker holds all of them
    for name, shape in (("E", (V, d)), ("g1", (1, d))):
        R, D = shape
        mask = torch.ones((K, R), dtype=torch.uint8, device="cuda")
        theta = P[name].float().view(R, D).cuda()
        m, v = torch.zeros_like(theta), torch.zeros_like(theta)
        bufs = [g[name].view(R, D) for g in grads]
        hp = dict(lr=4e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1)
        scale = sdp.clip_scale(sdp.coverage_grad_sqnorm(bufs, mask), 1.0)
        sdp.coverage_avg_adamw(bufs, mask, theta, m, v, grad_scale_dev=scale, **hp)
        mean = sum(w[name].view(R, D) for w in want) / K
        clip = min(1.0, 1.0 / (float(mean.norm()) + 1e-6))
        assert err_report(m.cpu().double(), 0.1 * clip * mean)[1] <= 2 * tol
        host = [workloads.bf16_bits(b) if dtype == torch.bfloat16 else b.cpu().numpy() for b in bufs]
        wth, _, _, _ = orc.avg_adamw(host, mask.cpu().numpy(), P[name].float().view(R, D).numpy(), np.zeros(shape, np.float32), np.zeros(shape, np.float32),
                                     grad_scale=float(scale), **hp)
        assert err_report(theta.cpu().numpy(), wth)[1] <= 1e-5


def _around_step(sdp, T, V, d, dt):
    """A step's outputs and workspaces, kept, and the calls that fill them."""
    e = lambda *s, t=dt: torch.empty(s, dtype=t, device="cuda")
    E, ids, labels, gamma, dZs = e(V, d), e(T, t=torch.int32), e(T, t=torch.int64), e(d), e(T, V)
    Z, st = e(T, V), torch.float32
    X, Y, H, mean, rstd = e(T, d), e(T, d), e(T, d), e(T, t=st), e(T, t=st)
    nll, lse, loss, scale = e(T, t=st), e(T, t=st), e(1, t=st), e(1, t=st)
    dX, dg, db, dE = e(T, d), e(d), e(d), e(V, d)
    n = max(sdp.norm_bwd_workspace_bytes(dt, T, d), sdp.embed_bwd_workspace_bytes(dt, T, V, d))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def run():
        sdp.embed_fwd(E, ids, 2.0, out=X)
        sdp.norm_fwd("layer", X, gamma, gamma, residual=X, out=(Y, H, mean, rstd))
        sdp.label_scale(labels, V, out=scale)
        sdp.token_loss(Z, labels, scale_dev=scale, out=(nll, lse, dZs, loss))
        sdp.norm_bwd("layer", H, Y, gamma, mean, rstd, dH=X, out=(dX, dg, db), ws=ws)
        sdp.embed_bwd(dX, ids, V, 2.0, out=dE, ws=ws)  # the same workspace: one call after the other

    g = torch.Generator(device="cuda").manual_seed(T)
    draw = lambda: (torch.randn((V, d), generator=g, device="cuda").to(dt), torch.randint(-1, V, (T,), generator=g, device="cuda").int(),
                    torch.randint(-1, V + 1, (T,), generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda").to(dt),
                    torch.randn((T, V), generator=g, device="cuda").to(dt))
    return run, (E, ids, labels, gamma, Z), draw, (X, Y, H, mean, rstd, scale, nll, lse, dZs, loss, dX, dg, db, dE), ws


@pytest.mark.parametrize("T,V,d,dt", [(40, 120, 64, torch.float32), (700, 500, 264, torch.bfloat16), (300, 77, 33, torch.bfloat16)])
def test_replays_like_eager(sdp, T, V, d, dt):
    run, inputs, draw, outputs, _ = _around_step(sdp, T, V, d, dt)
    _replay_against_eager(run, inputs, [draw(), draw()], outputs)


def test_two_graphs_share_a_workspace(sdp):
    """Captured one after the other with one workspace, replayed in turn on one stream: each leaves the other's results as they are."""
    steps = [_around_step(sdp, T, V, d, torch.bfloat16) for T, V, d in ((500, 300, 128), (400, 900, 72))]
    ws = steps[0][4] if steps[0][4].numel() >= steps[1][4].numel() else steps[1][4]
    refs, graphs = [], []
    for run, inputs, draw, outputs, own in steps:
        for cell in run.__closure__:  # both with the larger of the two
            if cell.cell_contents is own:
                cell.cell_contents = ws
        for dst, src in zip(inputs, draw()):
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
            o.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o.view(torch.uint8), r.view(torch.uint8)) for o, r in zip(steps[i][3], refs[i]))


def test_on_another_stream(sdp):
    run, inputs, draw, outputs, _ = _around_step(sdp, 600, 400, 136, torch.bfloat16)
    for dst, src in zip(inputs, draw()):
        dst.copy_(src)
    run()
    torch.cuda.synchronize()
    refs = [o.clone() for o in outputs]
    for o in outputs:
        o.fill_(float("nan"))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outputs, refs))


def test_offsets_past_32_bits(sdp):
    """Matrices of more than 2^31 values: sampled rows against 64 bits, the last ones among them."""
    big = dict(dtype=torch.bfloat16, device="cuda")
    print("loss 70000 x 32003", flush=True)
    T, V = 70000, 32003
    Z = torch.randn((T, V), **big)
    labels = torch.arange(T, device="cuda") % V
    labels[5], labels[T - 2] = -1, -1
    nll, lse, dZ, loss = sdp.token_loss(Z, labels, scale=2.0)
    rows = torch.tensor([0, 5, 34999, 67100, 67109, T - 3, T - 2, T - 1])
    wn, wl, wz, _ = loss64(Z[rows.cuda()].cpu(), labels[rows.cuda()].cpu(), 2.0)
    assert (nll.cpu()[rows].double() - wn).abs().max() <= 1.5e-5 * 12 and (lse.cpu()[rows].double() - wl).abs().max() <= 1.5e-5 * 12
    assert torch.allclose(dZ[rows.cuda()].cpu().double(), wz, rtol=2.0 ** -8 + 2e-5, atol=1e-12)
    assert abs(float(loss) - 2.0 * float(nll.double().sum())) <= 1e-6 * float(loss)
    del Z, dZ

    print("embedding 1100000 x 2000", flush=True)
    V, d, T = 1100000, 2000, 3000
    E = torch.randn((V, d), **big)
    ids = (torch.arange(T, device="cuda") * 367) % V
    ids[-1] = V - 1
    Y = sdp.embed_fwd(E, ids)
    assert torch.equal(Y, E[ids])
    dE = sdp.embed_bwd(Y, ids, V, 3.0, out=E)
    uniq, inv = torch.unique(ids.cpu(), return_inverse=True)
    want = embed_bwd64(Y.cpu(), inv, len(uniq), 3.0)
    assert torch.allclose(dE[uniq.cuda()].cpu().double(), want, rtol=2.0 ** -8 + 1e-5, atol=1e-6)
    dE[uniq.cuda()] = 0
    assert not dE.any()
    del E, dE

    print("norm 1100000 x 2000", flush=True)
    T = 1100000
    X, dY = torch.randn((T, d), **big), torch.randn((T, d), **big)
    gamma = torch.randn(d, **big)
    Y, H, mean, rstd = sdp.norm_fwd("layer", X, gamma, eps=EPS)
    dX, dg, db = sdp.norm_bwd("layer", H, dY, gamma, mean, rstd)
    rows = torch.tensor([0, 536870, 1073740, 1073742, T - 2, T - 1])
    r = rows.cuda()
    wY, _, wm, wr = norm_fwd64("layer", X[r].cpu(), None, gamma.cpu(), None, EPS)
    wX, _, _ = norm_bwd64("layer", X[r].cpu(), dY[r].cpu(), None, gamma.cpu(), wm, wr)
    assert torch.allclose(Y[r].cpu().double(), wY, rtol=2.0 ** -8, atol=2e-5) and torch.allclose(dX[r].cpu().double(), wX, rtol=2.0 ** -8, atol=2e-5)
    # sums over 1.1e6 rows: rounded to bf16, after 2149 + 2 + 16 + 16 additions (two rows at a time on 256 workgroups) of 2^-24 of partial sums that are
    # below 6 x 1.1e6^0.5 = 6300
    wb = sum(dY[i: i + 50000].double().sum(0) for i in range(0, T, 50000))
    assert ((db.double() - wb).abs() <= 2.0 ** -8 * wb.abs() + 2183 * 2.0 ** -24 * 6300).all()


def test_more_workgroups_than_a_row_of_the_grid(sdp):
    """Beyond 2^20 workgroups a launch has a second dimension: the last rows, and nothing behind them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    T, d = 5000003, 8
    X = torch.randn((T, d), generator=g, device="cuda")
    gamma = torch.ones(d, device="cuda")
    rows = torch.tensor([0, 4194303, 4194304, T - 1])
    Y, H, mean, rstd = sdp.norm_fwd("rms", X, gamma, eps=EPS)
    # relative: eight squares, their sum and mean, the root and two products, fewer than 20 roundings of 2^-24 = 1.2e-6
    assert torch.allclose(Y[rows.cuda()].cpu().double(), norm_fwd64("rms", X[rows.cuda()].cpu(), None, gamma.cpu(), None, EPS)[0], rtol=1.2e-6, atol=1e-12)
    V = 20000011
    ids = torch.arange(T, device="cuda") * 4
    E = torch.randn((V, d), generator=g, device="cuda")
    assert torch.equal(sdp.embed_fwd(E, ids), E[ids])
    dE = sdp.embed_bwd(X, ids, V, out=E)
    assert torch.equal(dE[ids], X)
    dE[ids] = 0
    assert not dE.any()
    few = ids[-200:]
    dE = sdp.embed_bwd(X[-200:], few, V, out=E)
    assert torch.equal(dE[few], X[-200:])
    dE[few] = 0
    assert not dE.any()
    T = 1200007
    nll, lse, dZ, loss = sdp.token_loss(X[:T], torch.arange(T, device="cuda") % d)
    rows = torch.tensor([0, 1048575, 1048576, T - 1])
    wn, _, wz, _ = loss64(X[rows.cuda()].cpu(), rows % d, 1.0)
    # eight terms of one lane's: exponents 3 roundings of at most 16 (logits within 11), 3 x 16 x 2^-24 x ln 2 = 2e-6, a sum of 7 + 6 roundings 8e-7,
    # 2^x 1.2e-7; log2 and the label's own value, at most 11, two roundings more: below 1.5e-5, and dZ, at most 1, below 2e-5
    assert ((nll.cpu()[rows].double() - wn).abs() <= 1.5e-5 * wn.clamp(min=1)).all()
    assert ((dZ.cpu()[rows].double() - wz).abs() <= 2e-5).all()
