"""The embedding's gradient of more tokens than one launch takes (sort, sums, join, through a workspace), and of more than the sort keeps in
registers, as programs use it: captured and replayed, by two graphs with one workspace, on another stream; with no token that has an id, neighbours in
runs, one id, ids of 64 bits.  Sums of whole numbers up to 2^24 (2^8 in bf16) are exact: results are compared for equality."""
import pytest
import torch

import test_gpu_around as steps
from around import DT, Guarded
from test_gpu_graph import _replay_against_eager

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def sdp():
    import paper_2507_09029_amd as m

    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,V,d,dt", [(1025, 120, 64, F32), (1500, 500, 264, BF16), (3000, 77, 33, BF16), (20000, 1300, 40, BF16), (17000, 40, 9, F32)])
def test_replays_like_eager(sdp, T, V, d, dt):
    run, inputs, draw, outputs, _ = steps._around_step(sdp, T, V, d, dt)
    _replay_against_eager(run, inputs, [draw(), draw()], outputs)


def test_graphs_share_a_workspace(sdp):
    """Three, captured one after the other with one workspace, replayed in turn on one stream: each leaves the others' results as they are."""
    made = [steps._around_step(sdp, T, V, d, BF16) for T, V, d in ((1500, 300, 128), (3000, 900, 72), (18000, 200, 24))]
    shared = max((m[4] for m in made), key=torch.Tensor.numel)
    refs, graphs = [], []
    for run, inputs, draw, outputs, own in made:
        for cell in run.__closure__:
            if cell.cell_contents is own:
                cell.cell_contents = shared
        for dst, src in zip(inputs, draw()):
            dst.copy_(src)
        run()
        torch.cuda.synchronize()
        refs.append([o.clone() for o in outputs])
    for run, *_ in made:
        graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            with torch.cuda.graph(graph, stream=s):
                run()
        graphs.append(graph)
    torch.cuda.synchronize()
    for i in (0, 1, 2, 1, 1, 0, 2, 0):
        for o in made[i][3]:
            o.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o.view(torch.uint8), r.view(torch.uint8)) for o, r in zip(made[i][3], refs[i])), i


@pytest.mark.parametrize("T", [3000, 20000])
def test_on_another_stream(sdp, T):
    run, inputs, draw, outputs, _ = steps._around_step(sdp, T, 400, 136, BF16)
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


def _ids(T, V, pattern, g):
    place = torch.arange(T)
    if pattern == "none":
        return torch.where(place % 2 == 0, -1, V)
    if pattern == "last":  # one token has an id
        return torch.where(place == T - 1, V - 1, -100)
    if pattern == "one":
        return torch.full((T,), V // 2)
    if pattern == "runs":
        return place // 97 % V
    if pattern == "mostly":  # one id but for every thousandth token
        return torch.where(place % 1000 == 0, V - 1, V // 3)
    return torch.randint(-1, V + 1, (T,), generator=g)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(1025, 100, 33), (1500, 64, 1601), (2000, 50001, 24), (16384, 5, 8), (16385, 700, 40), (70000, 300, 17)])
def test_patterns(sdp, T, V, d, dtype, wide):
    dt, g = DT[dtype], torch.Generator().manual_seed(T + V)
    for pattern in ("none", "last", "one", "runs", "mostly", "any"):
        print(f"embed_bwd {pattern} {dtype} T={T} V={V} d={d} wide={wide}", flush=True)
        ids = _ids(T, V, pattern, g)
        if dtype == "bf16":  # at most 256 ones of a column, whichever rows they fall into
            dY = torch.zeros((T, d))
            dY[torch.randint(0, T, (256, d), generator=g), torch.arange(d)] = 1.0
        else:
            dY = torch.randint(-8, 9, (T, d), generator=g).float()
        if wide:
            ids[3] += 2 ** 32  # its lower half names a row, it does not
        live = (ids >= 0) & (ids < V)
        want = torch.zeros((V, d)).index_add_(0, ids[live], dY[live])
        dE = Guarded((V, d), dt, 1)
        sdp.embed_bwd(dY.to(dt).cuda(), (ids if wide else ids.int()).cuda(), V, out=dE.t)
        torch.cuda.synchronize()
        dE.check("dE")
        assert torch.equal(dE.t.cpu().float(), want)


@pytest.mark.parametrize("T,V", [(1100, 50001), (2000, 700000)])
def test_ids_of_one_workgroup(sdp, T, V):
    """All tokens belong to the share of ids that one workgroup of the sort has, dealt out to 256 workgroups or 1024, or lie next to each other."""
    g = torch.Generator().manual_seed(T)
    v = torch.arange(V)
    dY = torch.randint(-8, 9, (T, 24), generator=g).float()
    for of in ((v ^ (v >> 8)) % 256 == 5, (v ^ (v >> 10)) % 1024 == 5, v % 1024 == 7, (v >= 1000) & (v < 1200)):
        share = v[of]
        ids = share[torch.randint(0, len(share), (T,), generator=g)]
        want = torch.zeros((V, 24)).index_add_(0, ids, dY)
        assert torch.equal(sdp.embed_bwd(dY.cuda(), ids.int().cuda(), V).cpu(), want)
