"""GPU parity of the output head where a call takes a form of a kernel that the other tests' sizes do not: a teacher's logits by whole waves (bf16, d > 512) with one and with several
workgroups a token, short rows of codes by a wave each with more entries than lanes, codes of 512 MB and more with a teacher; and the same bits whatever the
workspace held before.  Bounds: targets.py."""
import pytest
import torch

from around import DT
from targets import HeadWant, entries, rest_of
from test_gpu_head import head, some_labels

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,V,d,k", [(5, 1500, 520, 1), (5, 1500, 520, 100), (600, 1500, 520, 1), (600, 1500, 520, 100), (5, 1501, 2048, 1), (5, 1501, 2048, 100), (600, 1501, 2048, 1),
                                     (600, 1501, 2048, 100), (76, 2000, 832, 84), (511, 900, 1200, 17), (512, 900, 1200, 17), (1500, 3000, 64, 130), (1024, 4096, 72, 65),
                                     (1024, 4097, 72, 65)])
def test_distillation_of_wide_tokens_and_short_rows(sdp, T, V, d, k):
    """bf16.  d = 520: 65 pieces of eight values, one more than a wave; fewer than 512 tokens: several workgroups each."""
    n = T + V + d + k
    tau = (1.0, 2.0, 0.7)[n % 3]
    ids, top = entries(T, V, k, n, pad=0.2, cut=n % 2 == 0, wide=n % 4 < 2, dtype=(torch.float32, torch.bfloat16)[n % 2], twice=n % 5 == 0)
    ids[0, 0] = V - 1  # (not a batch without a target)
    top[0, 0] = 5.0
    rest = rest_of(top, ids, V, tau).cuda() if n % 3 else None
    X, W = (t.cuda() for t in head(T, V, d, torch.bfloat16, ids[:, 0].long()))
    ids, top = ids.cuda(), top.cuda()
    X[~(((ids >= 0) & (ids < V) & (top != -float("inf"))).any(1))] = NAN
    print(f"head distill T={T} V={V} d={d} k={k} tau={tau}", flush=True)
    a = dict(temperature=tau, top_lse=rest, scale=0.5)
    want = HeadWant(X, W, ids, top, rest, tau, 0.5)
    for kind in (dict(), dict(want_dw=False), dict(want_dx=False), dict(want_dx=False, want_dw=False)):
        want.check(sdp.head_distill(X, W, ids, top, **a, **kind))


def test_distillation_with_codes_of_half_a_gigabyte(sdp):
    """bf16, 9001 x 30001: rows around the caches, with several entries a lane."""
    T, V, d, k = 9001, 30001, 520, 70
    ids, top = entries(T, V, k, 1, pad=0.02, twice=True)
    ids[-1, -1], ids[0, 0] = V - 1, 0
    X, W = (t.cuda() for t in head(T, V, d, torch.bfloat16, ids[:, 0].long()))
    ids, top = ids.cuda(), top.cuda()
    HeadWant(X, W, ids, top, None, 2.0, 1.0 / T).check(sdp.head_distill(X, W, ids, top, temperature=2.0, scale=1.0 / T))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,k", [(1, 1, 8, 1), (5, 63, 16, 3), (17, 65, 24, 5), (65, 129, 72, 7), (130, 1001, 200, 9), (130, 9001, 64, 9), (257, 1023, 256, 8), (2049, 515, 64, 3), (1100, 5003, 40, 4),
                                     (20000, 60001, 16, 2)])
def test_any_bytes_in_the_workspace(sdp, T, V, d, k, dtype):
    """All outputs, from workspaces of zeros (code 0: a block's largest), of ones (code 65535: nothing; NaN) and of the byte 63 (numbers): the same bits.  The last batch takes
    several pieces."""
    dt = DT[dtype]
    labels = some_labels(T, V, 1, 0.2 if T > 2 else 0.0)
    ids, top = entries(T, V, k, 2, pad=0.2 if T > 2 else 0.0, twice=True)
    X, W = (t.cuda() for t in head(T, V, d, dt, labels))
    X[0] *= 40  # logits further apart than codes say
    labels, ids, top = labels.cuda(), ids.cuda(), top.cuda()
    print(f"head T={T} V={V} d={d} {dtype}", flush=True)
    for kind in (dict(), dict(want_dx=False), dict(want_dw=False), dict(want_dx=False, want_dw=False)):
        for call, size in ((lambda w: sdp.head_loss(X, W, labels, ws=w, **kind), sdp.head_loss_workspace_bytes(dt, T, V, d, **kind)),
                           (lambda w: sdp.head_distill(X, W, ids, top, ws=w, **kind), sdp.head_distill_workspace_bytes(dt, T, V, d, k, **kind))):
            ws = torch.empty((size,), dtype=torch.uint8, device="cuda")
            first = None
            for fill in (0, 255, 63):
                ws.fill_(fill)
                got = call(ws)
                first = first or got
                assert not any(t.isnan().any() for t in got if t is not None)
                assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, first)), (kind, fill)
