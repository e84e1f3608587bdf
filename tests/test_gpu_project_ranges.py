"""The products whose rows choose their weights at the ends of their ranges: many matrices, the narrowest ones, scales
of matrices without adapters, uneven loads, members beside one another beyond what the workspace has room for."""
import pytest
import torch

import project_reference as R
from test_gpu_project import Case, bounds, close, i32, matrices, normal, pj, room  # noqa: F401
from test_gpu_route_ranges import alone

pytestmark = pytest.mark.gpu


def check_experts(pj, loads, width, out, dtype, gated=False, gathered=False, scale=None, seed=0):  # noqa: F811
    g = torch.Generator().manual_seed(seed + len(loads))
    start = bounds(loads)
    w, own, values = matrices(g, len(loads), out, width, dtype)
    if scale is not None:
        own = torch.tensor(scale, device="cuda")
        values = w.cpu().view(torch.float8_e4m3fn).double() * own.cpu().double()[:, None, None]
    x = normal(g, 77 if gathered else start[-1], width).bfloat16()
    rows = torch.randint(-1, 78, (start[-1],), generator=g).tolist() if gathered else None
    weights = pj.es_weights_create(w, own)
    space = room(pj, weights, start[-1])
    y, again = (torch.empty(start[-1], out // 2 if gated else out, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for to in (y, again):
        pj.es_project_experts(weights, x.cuda(), to, i32(start), space, rows=None if rows is None else i32(rows), gated=gated)
    assert not pj.es_project_gave_up(space)
    close(y, *R.experts(x, values, start, rows, gated))
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("count", [256, 257, 512, 513, 1024])
@pytest.mark.parametrize("most", [1, 9, 130])
def test_many_matrices(pj, count, most, dtype):  # noqa: F811
    """More segments than a block has threads; tiles of up to 64 rows and of up to 256."""
    loads = [(i * 7919 % (most + 2)) * (i % 5 != 3) for i in range(count)]
    loads[-1] += 2
    check_experts(pj, loads, 48, 32, dtype, gated=most == 9, gathered=most == 130)


@pytest.mark.parametrize("count", [300, 1024])
def test_many_matrices_whose_rows_are_all_of_the_last_or_the_first(pj, count):  # noqa: F811
    for loads in ([0] * (count - 1) + [5], [17] + [0] * (count - 1), [0] * (count // 2) + [3] + [0] * (count - count // 2 - 1)):
        check_experts(pj, loads, 64, 16, "bf16")


@pytest.mark.parametrize("rows", [1, 20, 70, 300])
@pytest.mark.parametrize("out", [8, 16, 136])
def test_rows_of_eight(pj, rows, out):  # noqa: F811
    Case(pj, [rows, 2, 1], [1, -1, 0], 8, out, seed=rows + out).check()
    if out % 16 == 0:
        check_experts(pj, [rows, 0, 3], 8, out, "bf16", gated=True)
    check_experts(pj, [rows, 0, 3], 8, out, "bf16", gathered=True)


@pytest.mark.parametrize("rows", [3, 40, 200])
def test_scales_without_adapters(pj, rows):  # noqa: F811
    """Each matrix's own; one that is subnormal is taken as it is."""
    scale = [0.0, 1e-39, 1.2e-38, -0.5, 1e30, 3e-7]
    check_experts(pj, [rows, 2, rows, 1, rows, 5], 320, 144, "e4m3", scale=scale)
    check_experts(pj, [rows, 2, rows, 1, rows, 5], 320, 144, "e4m3", scale=[0.0, 1e-39, 1.2e-38, -0.5, 1e15, 3e-7], gated=True)
    for s in scale:
        g = torch.Generator().manual_seed(rows)
        w, own, _ = matrices(g, 1, 136, 320, "e4m3")
        own.fill_(s)
        x = normal(g, rows, 320).bfloat16()
        weights = pj.es_weights_create(w, own)
        y = torch.empty(rows, 136, dtype=torch.bfloat16, device="cuda")
        pj.es_project(weights, x.cuda(), y, room(pj, weights, rows))
        close(y, *R.project(x, w[0].cpu().view(torch.float8_e4m3fn).double() * float(own.double())))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("loads", [[0, 3000] + [3] * 30, [1] * 63 + [3100], [900] + [0] * 15, [130] + [2] * 3])
def test_most_rows_in_one_matrix(pj, loads, dtype):  # noqa: F811
    """Above and below the mean load at which tiles grow."""
    check_experts(pj, loads, 192, 144, dtype, gated=True, gathered=True)


@pytest.mark.parametrize("dtype,rank", [("bf16", 64), ("e4m3", 48)])
def test_single_rows_of_members_beyond_the_workspaces_room(pj, dtype, rank):  # noqa: F811
    counts = [1] * 1200
    Case(pj, counts, [i % 7 - 1 for i in range(len(counts))], 64, 28008, count=6, rank=rank, dtype=dtype).check()


@pytest.mark.parametrize("loads", [[65] * 40, [257] * 9 + [1], [1] * 80, [64, 1, 129] * 20, [256, 513, 1, 1, 257]])
def test_most_tiles_that_rows_have(pj, loads):  # noqa: F811
    """Each matrix has a tile of a single row at most behind its full ones."""
    check_experts(pj, loads, 64, 136, "bf16")


@pytest.mark.parametrize("groups,slots", [(1024, 900), (1024, 60000), (33, 16), (5, 4000)])
def test_starts_that_decrease(pj, groups, slots):  # noqa: F811
    """What is written then is not said, but it ends, and nothing is written around y."""
    w = torch.ones(groups, 16, 16, dtype=torch.bfloat16, device="cuda")
    weights = pj.es_weights_create(w)
    x = torch.ones(slots, 16, dtype=torch.bfloat16, device="cuda")
    around = torch.full((slots + 20, 16), 3.0, dtype=torch.bfloat16, device="cuda")
    space = room(pj, weights, slots)
    for start in ([slots * (g % 2) for g in range(groups + 1)], [slots - g * slots // groups for g in range(groups + 1)],
                  [(g * 7919) % (2 * slots) - slots // 2 for g in range(groups + 1)]):
        for rows in (None, i32(list(range(slots)))):
            around.fill_(3.0)
            pj.es_project_experts(weights, x, around[10:-10], i32(start), space, rows=rows)
            assert not pj.es_project_gave_up(space)
            assert (around[:10] == 3).all() and (around[-10:] == 3).all()
            if rows is None:
                assert ((around == 3) | (around == 16)).all()


CAPTURED = """
    import sys
    sys.path[:0] = [{root!r}, {tests!r}]
    import torch
    from paper_2608_17310_gb300 import project as pj
    from test_gpu_project import Case, Layer, close, i32
    torch.cuda.init()
    if {kind!r} == "layer":
        layer = Layer(pj, {size})
        call, check = layer.run, layer.check
    else:
        c = Case(pj, [40, 1, {size}], [0, 1, 2], 320, 264, dtype={kind!r})
        adapter, start = i32(c.members), i32(c.start)
        y = torch.empty(c.n, c.out, dtype=torch.bfloat16, device="cuda")
        call = lambda: pj.es_project(c.weights, c.xc, y, c.workspace, adapters=c.adapters, adapter=adapter, start=start)
        check = lambda: close(y, *c.want())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    graph.replay()
    torch.cuda.synchronize()
    check()
    print("fine")
"""


@pytest.mark.parametrize("kind,size", [("layer", 5), ("layer", 700), ("bf16", 300), ("e4m3", 3)])
def test_a_programs_first_calls_can_be_captured(pj, kind, size):  # noqa: F811
    alone(CAPTURED, kind=kind, size=size)


def test_calls_without_adapters_and_named_rows_take_a_small_workspace(pj, es):  # noqa: F811
    """One that was made for adapters serves them too, and so does its head alone; nothing smaller does."""
    c = Case(pj, [90, 10], [0, 1], 512, 136, rank=8)
    y = torch.empty(c.n, c.out, dtype=torch.bfloat16, device="cuda")
    head = torch.zeros(pj.ES_PROJECT_GAVE_UP + 256, dtype=torch.uint8, device="cuda")
    for space in (c.workspace, head):
        pj.es_project(c.weights, c.xc, y, space)
        close(y, *R.project(c.x, c.values[0]))
        pj.es_project_experts(c.weights, c.xc, y, i32([0, c.n]), space)
        close(y, *R.experts(c.x, c.values, [0, c.n]))
    for call in (lambda: pj.es_project(c.weights, c.xc, y, head[:-1]),
                 lambda: pj.es_project_experts(c.weights, c.xc, y, i32([0, c.n]), head[:-1]),
                 lambda: pj.es_project_experts(c.weights, c.xc, y, i32([0, c.n]), head, rows=i32(list(range(c.n))))):
        with pytest.raises(es.EsError) as e:
            call()
        assert e.value.status == es.ES_ERR_INVALID_ARG
