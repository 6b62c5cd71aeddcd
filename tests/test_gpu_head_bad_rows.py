"""GPU: a token whose logits or teacher hold something that is no number has NaN for its whole gradient, logits of -inf and logits far below the others included, so
that dW, which sums over it, is NaN throughout, whichever tokens are beside it."""
import pytest
import torch

from around import DT, normal
from targets import entries
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
@pytest.mark.parametrize("T", [20, 500, 1500])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_a_token_alone(sdp, bad, T, dtype):
    """X of one token: its logits are +inf and -inf side by side."""
    V, d, dt = 400, 64, DT[dtype]
    labels = some_labels(T, V, 1, 0.1)
    labels[7] = 9
    X, W = (t.cuda() for t in head(T, V, d, dt, labels))
    clean = sdp.head_loss(X, W, labels.cuda())
    X[7, 3] = bad
    nll, lse, dX, dW, loss = sdp.head_loss(X, W, labels.cuda())
    others = torch.arange(T) != 7
    assert torch.equal(nll.cpu()[others], clean[0].cpu()[others]) and torch.equal(dX.cpu()[others], clean[2].cpu()[others])
    assert nll[7].isnan() and lse[7].isnan() and loss.isnan() and dX[7].isnan().all() and dW.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [20, 500, 1500])
def test_far_logits_beside_a_bad_one(sdp, T, dtype):
    """A bad row of W spoils one logit of every token; the others lie hundreds apart, most of them further below their neighbours than 16 bits of distance say."""
    V, d, dt = 400, 64, DT[dtype]
    X, W = (normal(n, d, dtype=torch.float64, seed=n, std=s).to(dt).cuda() for n, s in ((T, 30.0), (V, 3.0)))
    W[301] = NAN
    nll, lse, dX, dW, loss = sdp.head_loss(X, W, (torch.arange(T) % V).cuda())
    assert nll.isnan().all() and lse.isnan().all() and loss.isnan() and dX.isnan().all() and dW.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [20, 500, 1500])
@pytest.mark.parametrize("bad", [INF, NAN])
def test_a_teacher_alone(sdp, bad, T, dtype):
    """One entry of one token; logits far apart."""
    V, d, k, dt = 400, 64, 5, DT[dtype]
    ids, top = entries(T, V, k, 1)
    X, W = (normal(n, d, dtype=torch.float64, seed=n, std=s).to(dt).cuda() for n, s in ((T, 30.0), (V, 3.0)))
    top[7, 2] = bad
    kl, lse, dX, dW, loss = sdp.head_distill(X, W, ids.cuda(), top.cuda())
    others = torch.arange(T) != 7
    assert not kl.cpu()[others].isnan().any() and not dX.cpu()[others].isnan().any()
    assert kl[7].isnan() and loss.isnan() and dX[7].isnan().all() and dW.isnan().all()
