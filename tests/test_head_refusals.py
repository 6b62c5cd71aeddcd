"""CPU: what the calls of the output head and of learning from a teacher refuse, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2507_09029_amd as sdp

INVALID, SHAPE, WORKSPACE = -1, -2, -3
NAN, INF = float("nan"), float("inf")


def at(i):  # buffers far apart; never dereferenced
    return ctypes.c_void_p(0x100000000 * (i + 1))


def odd(n):
    return ctypes.c_void_p(0x1000 + n)


def call(fn, args, **change):
    for k in change:
        assert k in args
    return fn(*[change.get(n, v) for n, v in args.items()])


@pytest.fixture(scope="module")
def L():
    return sdp.lib()


def test_distillation(L):
    a = dict(dtype=1, id_type=0, top_dtype=0, T=4, V=10, k=3, ldz=10, temperature=1.0, scale=1.0, Z=at(0), ids=at(1), top=at(2), top_lse=at(3), scale_dev=at(4),
             kl=at(5), lse=at(6), dZ=at(7), loss=at(8), stream=None)
    f = lambda **c: call(L.sdp_distill_loss, a, **c)
    for bad in (dict(dtype=2), dict(id_type=2), dict(top_dtype=2), dict(top_dtype=-1), dict(T=-1), dict(V=0), dict(k=0), dict(temperature=0.0), dict(temperature=-1.0),
                dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-7), dict(scale=INF), dict(Z=None), dict(ids=None), dict(top=None), dict(kl=None),
                dict(Z=odd(1)), dict(dtype=0, Z=odd(2)), dict(ids=odd(2)), dict(id_type=1, ids=odd(4)), dict(top=odd(2)), dict(top_dtype=1, top=odd(1)),
                dict(top_lse=odd(2)), dict(kl=odd(1)), dict(dZ=ctypes.c_void_p(0x100000000 + 2)), dict(dZ=at(1)), dict(dZ=at(2)), dict(kl=at(3)), dict(lse=at(5)),
                dict(loss=at(5)), dict(loss=at(4)), dict(kl=at(0)), dict(loss=at(7))):
        assert f(**bad) == INVALID, bad
    assert f(ldz=9) == SHAPE and f(T=(1 << 30) + 1) == SHAPE and f(k=1025) == SHAPE
    assert f(T=0, Z=None, ids=None, top=None, top_lse=None, kl=None, lse=None, dZ=None, loss=None, scale_dev=None) == 0


def test_head_loss(L):
    a = dict(dtype=1, id_type=0, T=4, V=10, d=16, scale=1.0, X=at(0), W=at(1), labels=at(2), scale_dev=at(3), nll=at(4), lse=at(5), dX=at(6), dW=at(7), loss=at(8),
             ws=at(9), ws_bytes=1 << 30, stream=None)
    f = lambda **c: call(L.sdp_head_loss, a, **c)
    for bad in (dict(dtype=3), dict(id_type=-1), dict(T=-1), dict(V=0), dict(d=0), dict(scale=NAN), dict(X=None), dict(W=None), dict(labels=None), dict(nll=None),
                dict(X=odd(8)), dict(W=odd(2)), dict(dX=odd(8)), dict(dW=odd(8)), dict(labels=odd(2)), dict(id_type=1, labels=odd(4)), dict(nll=odd(2)),
                dict(dW=at(1)), dict(dX=at(1)), dict(dW=at(0)), dict(dX=ctypes.c_void_p(0x100000000 + 16)), dict(dX=at(7)), dict(nll=at(5)), dict(loss=at(4)),
                dict(loss=at(3)), dict(lse=at(2)), dict(nll=at(0)), dict(ws=at(0)), dict(ws=at(6)), dict(ws=at(8))):
        assert f(**bad) == INVALID, bad
    assert f(d=12) == SHAPE and f(V=1 << 22) == SHAPE and f(V=1 << 20, d=1 << 11) == SHAPE and f(T=(1 << 26) + 1) == SHAPE
    assert f(dtype=0, V=1 << 22) == SHAPE and f(V=5, d=(1 << 20) + 8) == SHAPE
    assert f(ws=None) == WORKSPACE and f(ws_bytes=64) == WORKSPACE and f(ws=odd(0x80)) == WORKSPACE
    w = L.sdp_head_loss_workspace_bytes
    assert f(ws_bytes=w(1, 4, 10, 16, 1, 1) - 1) == WORKSPACE
    assert w(1, 0, 10, 16, 1, 1) == 0 and w(1, 4, 0, 16, 1, 1) == 0 and w(2, 4, 10, 16, 1, 1) == 0 and w(1, 4, 10, 12, 1, 1) == 0 and w(1, 4, 1 << 22, 16, 1, 1) == 0
    # whatever the tokens, a piece of their logits
    assert w(1, 16384, 32000, 2048, 0, 0) < w(1, 16384, 32000, 2048, 1, 1) < 3 << 29
    assert w(1, 1 << 20, 128256, 4096, 1, 1) < (1 << 30) * 4.5 and w(0, 1 << 20, 32000, 1024, 1, 1) < 1.3 * (1 << 30)
    assert sdp.head_loss_workspace_bytes(torch.bfloat16, 16384, 32000, 2048, want_dw=False) == w(1, 16384, 32000, 2048, 1, 0)


def test_head_distillation(L):
    a = dict(dtype=1, id_type=0, top_dtype=0, T=4, V=10, d=16, k=3, temperature=2.0, scale=1.0, X=at(0), W=at(1), ids=at(2), top=at(3), top_lse=at(4),
             scale_dev=at(5), kl=at(6), lse=at(7), dX=at(8), dW=at(9), loss=at(10), ws=at(11), ws_bytes=1 << 30, stream=None)
    f = lambda **c: call(L.sdp_head_distill, a, **c)
    for bad in (dict(dtype=3), dict(id_type=-1), dict(top_dtype=-1), dict(top_dtype=2), dict(T=-1), dict(V=0), dict(d=0), dict(k=0), dict(temperature=0.0),
                dict(temperature=NAN), dict(scale=NAN), dict(X=None), dict(W=None), dict(ids=None), dict(top=None), dict(kl=None), dict(X=odd(8)), dict(W=odd(2)),
                dict(top=odd(2)), dict(top_lse=odd(1)), dict(dW=at(3)), dict(dX=at(4)), dict(kl=at(2)), dict(loss=at(6)), dict(ws=at(3))):
        assert f(**bad) == INVALID, bad
    assert f(d=12) == SHAPE and f(V=1 << 22) == SHAPE and f(k=1025) == SHAPE
    assert f(ws=None) == WORKSPACE and f(ws_bytes=L.sdp_head_distill_workspace_bytes(1, 4, 10, 16, 3, 1, 1) - 1) == WORKSPACE
    assert L.sdp_head_distill_workspace_bytes(1, 4, 10, 16, 1025, 1, 1) == 0


def test_binding_refuses_what_does_not_fit():
    X, W, labels = torch.zeros(4, 16), torch.zeros(10, 16), torch.zeros(4, dtype=torch.int32)
    Z, ids, top = torch.zeros(4, 10), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    with pytest.raises(TypeError, match="X: expected a contiguous torch.float32 tensor on the GPU"):
        sdp.head_loss(X, W, labels)
    with pytest.raises(TypeError, match="X: expected torch.float32 or torch.bfloat16"):
        sdp.head_loss(X.half(), W, labels)
    with pytest.raises(TypeError, match="labels: expected torch.int32 or torch.int64"):
        sdp.head_loss(X, W, labels.short())
    with pytest.raises(ValueError, match="W"):
        sdp.head_loss(X, W[:, :8], labels)
    with pytest.raises(ValueError, match="labels"):
        sdp.head_loss(X, W, labels[:3])
    with pytest.raises(ValueError, match="dX: expected a tensor"):
        sdp.head_loss(X, W, labels, out=(Z, None, None, W, None))
    with pytest.raises(ValueError, match="dW: expected a tensor"):
        sdp.head_loss(X, W, labels, out=(Z, None, X, None, None))
    with pytest.raises(ValueError, match="ids"):
        sdp.head_distill(X, W, labels, top)
    with pytest.raises(ValueError, match="top"):
        sdp.head_distill(X, W, ids, top[:, :2])
    with pytest.raises(TypeError, match="top: expected torch.float32 or torch.bfloat16"):
        sdp.head_distill(X, W, ids, top.half())
    with pytest.raises(ValueError, match="ids"):
        sdp.distill_loss(Z, labels, top)
    with pytest.raises(ValueError, match="top_lse"):
        sdp.distill_loss(Z, ids, top, top_lse=torch.zeros(3))
    with pytest.raises(ValueError, match="dZ: expected a tensor"):
        sdp.distill_loss(Z, ids, top, out=(top, None, None, None))
    with pytest.raises(TypeError, match="Z: expected a contiguous"):
        sdp.distill_loss(Z, ids, top)
