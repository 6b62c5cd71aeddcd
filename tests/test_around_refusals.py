"""CPU: what the norm, embedding and loss calls refuse, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2507_09029_amd as sdp

INVALID, SHAPE, WORKSPACE = -1, -2, -3
NAN, INF = float("nan"), float("inf")


def at(i):  # buffers far apart; never dereferenced
    return ctypes.c_void_p(0x100000000 * (i + 1))


def call(fn, args, **change):
    names = list(args)
    for k, v in change.items():
        assert k in names
    return fn(*[change.get(n, args[n]) for n in names])


@pytest.fixture(scope="module")
def L():
    return sdp.lib()


def test_norm_forward(L):
    a = dict(kind=0, dtype=1, T=4, d=16, eps=1e-5, X=at(0), R=at(1), gamma=at(2), beta=at(3), H=at(4), Y=at(5), mean=at(6), rstd=at(7), stream=None)
    f = lambda **c: call(L.sdp_norm_fwd, a, **c)
    for bad in (dict(kind=2), dict(kind=-1), dict(dtype=2), dict(T=-1), dict(d=0), dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF), dict(X=None),
                dict(gamma=None), dict(Y=None), dict(rstd=None), dict(mean=None), dict(H=None), dict(R=None), dict(kind=1),
                dict(X=ctypes.c_void_p(0x1001)), dict(rstd=ctypes.c_void_p(0x1002)), dict(dtype=0, Y=ctypes.c_void_p(0x1002)),
                dict(H=at(5)), dict(Y=at(2)), dict(Y=ctypes.c_void_p(0x100000000 + 32)), dict(mean=at(7)), dict(rstd=at(0)), dict(H=at(3))):
        assert f(**bad) == INVALID, bad
    assert f(d=16385) == SHAPE and f(T=(1 << 30) + 1) == SHAPE
    assert f(T=0, X=None, R=None, H=None, Y=None, mean=None, rstd=None) == 0


def test_norm_backward(L):
    a = dict(kind=0, dtype=1, T=4, d=16, H=at(0), dY=at(1), dH=at(2), gamma=at(3), mean=at(4), rstd=at(5), dX=at(6), dgamma=at(7), dbeta=at(8), ws=at(9),
             ws_bytes=1 << 30, stream=None)
    f = lambda **c: call(L.sdp_norm_bwd, a, **c)
    for bad in (dict(kind=7), dict(dtype=-1), dict(T=-1), dict(d=-4), dict(H=None), dict(dY=None), dict(gamma=None), dict(mean=None), dict(rstd=None),
                dict(dX=None), dict(dgamma=None), dict(kind=1), dict(dX=ctypes.c_void_p(0x1001)), dict(dX=ctypes.c_void_p(0x100000000 + 16)),
                dict(dgamma=at(0)), dict(dgamma=at(8)), dict(dbeta=at(6)), dict(dX=at(3)), dict(dgamma=at(3)), dict(dX=at(5))):
        assert f(**bad) == INVALID, bad
    assert f(d=40000) == SHAPE
    assert f(ws=None) == WORKSPACE and f(ws_bytes=8) == WORKSPACE and f(ws=ctypes.c_void_p(0x1004)) == WORKSPACE
    assert f(T=0, H=None, dY=None, dH=None, gamma=None, mean=None, rstd=None, dX=None, dgamma=None, dbeta=None, ws=None, ws_bytes=0) == 0
    w = L.sdp_norm_bwd_workspace_bytes
    assert w(1, 0, 16) == 0 and w(1, 5, 0) == 0 and w(1, -1, 8) == 0 and w(3, 4, 8) == 0 and w(1, 4, 40000) == 0
    assert 2 * 16 * 4 <= w(1, 4, 16) <= w(1, 100000, 16) <= w(1, 100000, 2048)
    assert sdp.norm_bwd_workspace_bytes(torch.bfloat16, 4, 16) == w(1, 4, 16)


def test_embedding(L):
    a = dict(dtype=1, id_type=0, T=4, V=10, d=16, scale=1.0, E=at(0), ids=at(1), Y=at(2), stream=None)
    f = lambda **c: call(L.sdp_embed_fwd, a, **c)
    for bad in (dict(dtype=2), dict(id_type=2), dict(T=-1), dict(V=0), dict(d=0), dict(scale=NAN), dict(scale=INF), dict(E=None), dict(ids=None), dict(Y=None),
                dict(E=ctypes.c_void_p(0x1001)), dict(ids=ctypes.c_void_p(0x1002)), dict(id_type=1, ids=ctypes.c_void_p(0x1004)), dict(Y=at(0)), dict(Y=at(1))):
        assert f(**bad) == INVALID, bad
    assert f(T=(1 << 30) + 1) == SHAPE
    assert f(T=0, ids=None, Y=None) == 0
    a = dict(dtype=1, id_type=0, T=4, V=10, d=16, scale=1.0, dY=at(0), ids=at(1), dE=at(2), ws=at(3), ws_bytes=1 << 30, stream=None)
    f = lambda **c: call(L.sdp_embed_bwd, a, **c)
    for bad in (dict(dtype=2), dict(id_type=-1), dict(T=-1), dict(V=0), dict(d=0), dict(scale=INF), dict(dY=None), dict(ids=None), dict(dE=None),
                dict(dE=at(0)), dict(dE=at(1)), dict(dtype=0, dY=ctypes.c_void_p(0x1002))):
        assert f(**bad) == INVALID, bad
    assert f(T=(1 << 30) + 1) == SHAPE and f(ws=None) == WORKSPACE and f(ws_bytes=64) == WORKSPACE
    assert f(V=1 << 30, d=1 << 30) == SHAPE and f(T=1000, V=1 << 30, d=1 << 20) == SHAPE
    w = L.sdp_embed_bwd_workspace_bytes
    assert w(1, 4, 0, 16) == 0 and w(2, 4, 10, 16) == 0 and w(1, -1, 10, 16) == 0
    assert w(1, 0, 10, 16) >= 11 * 4 and w(1, 1000, 10, 16) >= 2 * 4000


def test_loss(L):
    a = dict(dtype=1, id_type=0, T=4, V=10, ldz=10, scale=1.0, Z=at(0), labels=at(1), scale_dev=at(2), nll=at(3), lse=at(4), dZ=at(5), loss=at(6), stream=None)
    f = lambda **c: call(L.sdp_token_loss, a, **c)
    for bad in (dict(dtype=4), dict(id_type=9), dict(T=-1), dict(V=0), dict(scale=NAN), dict(Z=None), dict(labels=None), dict(nll=None),
                dict(Z=ctypes.c_void_p(0x1001)), dict(nll=ctypes.c_void_p(0x1002)), dict(scale_dev=ctypes.c_void_p(0x1002)),
                dict(dZ=ctypes.c_void_p(0x100000000 + 2)), dict(dZ=at(1)), dict(lse=at(3)), dict(loss=at(3)), dict(loss=at(2)), dict(nll=at(0)), dict(loss=at(5))):
        assert f(**bad) == INVALID, bad
    assert f(ldz=9) == SHAPE and f(T=(1 << 30) + 1) == SHAPE
    assert f(T=0, Z=None, labels=None, nll=None, lse=None, dZ=None, loss=None, scale_dev=None) == 0
    a = dict(id_type=1, T=4, V=10, labels=at(0), scale=at(1), stream=None)
    f = lambda **c: call(L.sdp_label_scale, a, **c)
    for bad in (dict(id_type=2), dict(T=-1), dict(V=0), dict(labels=None), dict(scale=None), dict(labels=ctypes.c_void_p(0x1004)), dict(scale=at(0))):
        assert f(**bad) == INVALID, bad
    assert f(T=(1 << 30) + 1) == SHAPE


def test_binding_refuses_what_does_not_fit():
    X, g, ids = torch.zeros(4, 16), torch.ones(16), torch.zeros(4, dtype=torch.int32)
    st = torch.zeros(4)
    with pytest.raises(TypeError, match="X: expected a contiguous torch.float32 tensor on the GPU"):
        sdp.norm_fwd("layer", X, g)
    with pytest.raises(KeyError):
        sdp.norm_fwd("batch", X, g)
    with pytest.raises(TypeError, match="X: expected torch.float32 or torch.bfloat16"):
        sdp.norm_fwd("layer", X.half(), g)
    with pytest.raises(ValueError, match="gamma"):
        sdp.norm_fwd("layer", X, g[:8])
    with pytest.raises(ValueError, match="residual"):
        sdp.norm_fwd("layer", X, g, residual=X[:2])
    with pytest.raises(ValueError, match="Y"):
        sdp.norm_fwd("layer", X, g, out=(X[:1], None, st, st))
    with pytest.raises(ValueError, match="dY"):
        sdp.norm_bwd("layer", X, X[:, :8], g, st, st)
    with pytest.raises(ValueError, match="dgamma"):
        sdp.norm_bwd("rms", X, X, g, None, st, out=(X, None, None))
    with pytest.raises(TypeError, match="H: expected a contiguous"):
        sdp.norm_bwd("rms", X, X, g, None, st, ws=torch.zeros(1 << 16, dtype=torch.uint8))
    with pytest.raises(TypeError, match="E: expected a contiguous"):
        sdp.embed_fwd(X, ids)
    with pytest.raises(TypeError, match="ids: expected torch.int32 or torch.int64"):
        sdp.embed_fwd(X, ids.short())
    with pytest.raises(ValueError, match="ids"):
        sdp.embed_bwd(X, ids[:3], 10)
    with pytest.raises(ValueError, match="dE"):
        sdp.embed_bwd(X, ids, 10, out=X)
    with pytest.raises(ValueError, match="labels"):
        sdp.token_loss(X, ids[:3])
    with pytest.raises(ValueError, match="strides of Z"):
        sdp.token_loss(X, ids, out=(st, None, torch.zeros(4, 20)[:, :16], None))
    with pytest.raises(TypeError, match="Z: expected a contiguous"):
        sdp.token_loss(X, ids)
    with pytest.raises(TypeError, match="labels: expected a contiguous"):
        sdp.label_scale(ids, 10)
