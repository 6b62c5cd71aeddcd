"""GPU parity of the output head on tokens so wide that all of dX's tiles are more than its cut tiles are otherwise.  Bounds: targets.py."""
import pytest
import torch

from targets import Want, near, product_bound, z_bound
from test_gpu_head import head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,V,d", [(5, 2000, 81920), (128, 8000, 98304), (300, 200, 163840)])
def test_two_terms_of_very_wide_tokens(sdp, T, V, d):
    """Few tokens' gradient is held in two terms however many columns dX has: to these terms' bounds.  The last batch has 100 tokens with a target."""
    n, c = 64, 0.1  # X has so many columns that are not zero: bounds of their products alone, the others add exact zeros
    labels = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(T))
    x, w = head(T, V, n, torch.bfloat16, labels)
    labels[100 if T == 300 else T:] = -1
    g = torch.Generator(device="cuda").manual_seed(1)
    X, W = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda"), torch.randn((V, d), generator=g, device="cuda").mul_(0.25).bfloat16()
    X[:, :n], W[:, :n] = x, w
    labels = labels.cuda()
    print(f"head loss T={T} V={V} d={d}", flush=True)
    x, w = X[:, :n].double(), W.double()
    want = Want(x @ w[:, :n].T, labels[:, None], None, None, 1.0, c, z_bound(X[:, :n], W[:, :n]), torch.bfloat16, codes=True, half=2.0 ** -17)
    dX, dW = want.dz @ w, want.dz.T @ x
    dX_room, dW_room = product_bound(want.dz, w, want.dz_room, torch.bfloat16, dX), product_bound(want.dz.T, x, want.dz_room.T, torch.bfloat16, dW)
    for kind in (dict(), dict(want_dx=False), dict(want_dw=False)):
        nll, lse, gx, gw, loss = sdp.head_loss(X, W, labels, scale=c, **kind)
        want.rows(nll, lse, loss)
        if gx is not None:
            near(gx, dX, torch.where(want.live[:, None], dX_room, 1e-300), "dX")
        if gw is not None:
            near(gw[:, :n], dW, dW_room, "dW")
            assert (gw[:, n:] == 0).all()
