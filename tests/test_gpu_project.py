"""The products whose rows choose their weights against their definitions in 64 bits. Tolerances and
their reasons: project_reference.py."""
import numpy as np
import pytest
import torch

import project_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pj(es):
    from paper_2608_17310_gb300 import project
    return project


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def bounds(counts):
    return [0] + np.cumsum(counts).astype(int).tolist()


def normal(g, *shape):
    return torch.randn(*shape, generator=g)


def matrices(g, groups, out, width, dtype):
    """(stored, scale, values) of matrices: values are what the stored ones stand for, in 64 bits."""
    w = normal(g, groups, out, width) * width ** -0.5
    if dtype == "bf16":
        w = w.bfloat16()
        return w.cuda(), None, w.double()
    scale = w.abs().amax((1, 2)) / 448
    codes = (w / scale[:, None, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).cuda(), scale.cuda(), codes.double() * scale.double()[:, None, None]


def room(pj, w, rows, adapters=None):
    return torch.zeros(pj.es_project_workspace(w, rows, adapters), dtype=torch.uint8, device="cuda")


def close(got, want, off, what=""):
    d = (got.double().cpu() - want).abs()
    bad = ~(d <= off)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((d / off).max()):.2f} of what is allowed"


class Case:
    """Requests of some rows each, their adapters, and the shared matrix."""

    def __init__(self, pj, counts, members, width=512, out=256, count=3, rank=16, dtype="bf16", seed=0, spare=0,
                 scaled=True):
        g = torch.Generator().manual_seed(seed)
        self.pj, self.counts, self.members, self.count = pj, counts, members, count
        self.start = bounds(counts)
        self.n = self.start[-1]
        self.w, self.w_scale, self.values = matrices(g, 1, out, width, dtype)
        self.x = normal(g, self.n + spare, width).bfloat16()
        self.a = (normal(g, count, rank, width) * width ** -0.5).bfloat16()
        self.b = (normal(g, count, out, rank) * 0.3).bfloat16()
        self.scale = (normal(g, count) * 0.5 + 1).float() if scaled else None
        self.weights = pj.es_weights_create(self.w, self.w_scale)
        self.adapters = pj.es_adapters_create(self.a.cuda(), self.b.cuda(), None if self.scale is None else self.scale.cuda())
        self.workspace = room(pj, self.weights, self.n + spare, self.adapters)
        self.xc = self.x.cuda()
        self.out = out

    def member_of_rows(self):
        return [m if 0 <= m < self.count else -1 for m, c in zip(self.members, self.counts) for _ in range(c)]

    def want(self):
        return R.project(self.x[:self.n], self.values[0], self.a, self.b, self.scale, self.member_of_rows())

    def run(self, y=None, start=True, **kw):
        y = torch.full((len(self.x), self.out), 7.0, dtype=torch.bfloat16, device="cuda") if y is None else y
        self.pj.es_project(self.weights, self.xc, y, self.workspace, adapters=self.adapters, adapter=i32(self.members),
                           start=i32(self.start) if start else None, **kw)
        return y

    def check(self, what=""):
        y = self.run()
        again = self.run()
        assert not self.pj.es_project_gave_up(self.workspace)
        assert torch.equal(y.view(torch.int16), again.view(torch.int16)), "two calls differ"
        want, off = self.want()
        close(y[:self.n], want, off, what)
        assert (y[self.n:] == 7).all(), "rows behind the last request were written"


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("width,out", [(16, 8), (48, 136), (512, 256), (1264, 1000), (720, 2072), (4096, 192)])
@pytest.mark.parametrize("counts,members", [
    ([1], [0]), ([1, 1, 1, 1, 1], [2, -1, 0, 1, 7]), ([3, 0, 17, 1, 0, 43], [1, 0, 2, -1, 1, 0])])
def test_project_small(pj, dtype, width, out, counts, members):
    Case(pj, counts, members, width, out, dtype=dtype, spare=3).check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rank", [8, 16, 40, 64, 72, 128])
def test_project_ranks(pj, dtype, rank):
    Case(pj, [1, 70, 1, 1, 16, 33], [0, 1, 2, -1, 2, 0], 320, 264, rank=rank, dtype=dtype, scaled=rank != 16).check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("counts", [[64], [65], [1] * 200, [130, 255, 1, 16, 300], [256, 256], [15, 241, 512, 7],
                                    [1] * 33 + [700] + [2] * 40])
def test_project_many_rows(pj, dtype, counts):
    n = len(counts)
    Case(pj, counts, [i % 5 - 1 for i in range(n)], 576, 392, count=4, rank=32, dtype=dtype, spare=5).check()


@pytest.mark.parametrize("rows", [1, 16, 63, 300])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_project_without_adapters(pj, rows, dtype):
    g = torch.Generator().manual_seed(3)
    w, scale, values = matrices(g, 1, 520, 2064, dtype)
    x = normal(g, rows, 2064).bfloat16()
    weights = pj.es_weights_create(w[0], scale)
    y = torch.empty(rows, 520, dtype=torch.bfloat16, device="cuda")
    pj.es_project(weights, x.cuda(), y, room(pj, weights, rows))
    close(y, *R.project(x, values[0]))


def test_one_row_a_request_without_start(pj):
    c = Case(pj, [1] * 9, [0, 1, 2, -1, 0, 0, 2, 1, 1])
    y = c.run(start=False)
    close(y, *c.want())
    assert torch.equal(y, c.run())


def test_requests_of_no_rows_alone(pj):
    c = Case(pj, [0, 0], [0, 1], spare=4)
    assert (c.run() == 7).all()


def test_nonfinite_adapters_stay_with_their_rows(pj):
    """Members share 16-row blocks and tiles; one has infinities and NaN in A and B, one request a NaN in x."""
    counts = [1, 1, 5, 40, 1, 30, 100, 3]
    c = Case(pj, counts, [0, 1, 2, 1, 0, 2, 0, 2], 512, 264, rank=16)
    clean = c.run()
    want, off = c.want()
    b = c.b.clone()
    b[1, ::3, 5] = float("nan")
    b[1, 1::3, 2] = float("inf")
    a = c.a.clone()
    a[1, 3, 7] = float("inf")
    c.adapters = pj.es_adapters_create(a.cuda(), b.cuda(), c.scale.cuda())
    x = c.xc.clone()
    x[c.start[4], 3] = float("nan")
    c.xc = x
    y = c.run()
    mine = torch.tensor(c.member_of_rows())
    other = (mine != 1)
    other[c.start[4]] = False
    close(y.cpu()[other], want[other], off[other])
    assert torch.equal(y.cpu()[other], clean.cpu()[other])
    assert not torch.isfinite(y[c.start[4]]).any()
    assert not torch.isfinite(y.cpu()[mine == 1][:, ::3]).any()


def test_strides_and_surroundings(pj):
    g = torch.Generator().manual_seed(5)
    rows, width, out, count, rank = 37, 336, 200, 2, 24
    big = normal(g, 1, out + 2, width + 40).bfloat16().cuda()
    w = big[:, 1:out + 1, 8:8 + width]
    x_all = normal(g, rows, width + 24).bfloat16().cuda()
    x = x_all[:, 16:16 + width]
    y_all = torch.full((rows + 2, out + 48), 5.0, dtype=torch.bfloat16, device="cuda")
    y = y_all[1:rows + 1, 32:32 + out]
    a_all = normal(g, count, 2, rank, width).bfloat16().cuda() * 0.05
    b_all = normal(g, count, 2, out, rank).bfloat16().cuda() * 0.05
    a, b = a_all[:, 1], b_all[:, 0]
    weights, adapters = pj.es_weights_create(w), pj.es_adapters_create(a, b)
    member = [1] * 20 + [-1] * 6 + [0] * 11
    pj.es_project(weights, x, y, room(pj, weights, rows, adapters), adapters=adapters, adapter=i32([1, -1, 0]),
                  start=i32([0, 20, 26, 37]))
    close(y, *R.project(x.cpu(), w[0].cpu(), a.cpu(), b.cpu(), None, member))
    y.fill_(5.0)
    assert (y_all == 5).all()


def test_offsets_past_32_bits(pj):
    g = torch.Generator().manual_seed(6)
    stride = 2 ** 31 + 8
    x = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 64), (stride, 1))
    y = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 64), (stride, 1))
    w = torch.empty(2 * 2 ** 31 + 64 * 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 64, 64), (2 ** 31, 64, 1))
    xs, ws = normal(g, 3, 64).bfloat16(), (normal(g, 3, 64, 64) / 8).bfloat16()
    x.copy_(xs), w.copy_(ws)
    weights = pj.es_weights_create(w)
    pj.es_project_experts(weights, x, y, i32([0, 0, 1, 3]), room(pj, weights, 3))
    close(y, *R.experts(xs, ws, [0, 0, 1, 3]))
    pj.es_project_experts(weights, x, y, i32([0, 1, 2, 3]), room(pj, weights, 3), rows=i32([2, 2, 1]))
    close(y, *R.experts(xs, ws, [0, 1, 2, 3], [2, 2, 1]))
    one = pj.es_weights_create(w[2])
    pj.es_project(one, x, y, room(pj, one, 3))
    close(y, *R.project(xs, ws[2]))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gathered", [False, True])
@pytest.mark.parametrize("width,out,loads", [
    (16, 16, [1]), (64, 16, [0, 3, 0, 0, 1]), (512, 272, [5, 0, 16, 17, 1, 0]), (1264, 1456, [2, 2, 0, 1]),
    (320, 400, [300, 0, 1, 64, 65, 257]), (880, 144, [7] * 60)])
def test_experts(pj, dtype, gated, gathered, width, out, loads):
    g = torch.Generator().manual_seed(len(loads) + out)
    start = bounds(loads)
    slots, spare = start[-1], 4
    w, scale, values = matrices(g, len(loads), out, width, dtype)
    rows = None
    x = normal(g, 50 if gathered else slots + spare, width).bfloat16()
    if gathered:
        rows = torch.randint(-2, 52, (slots + spare,), generator=g).tolist()
        rows[0] = 49
    weights = pj.es_weights_create(w, scale)
    outs = out // 2 if gated else out
    workspace = room(pj, weights, slots + spare)
    y, again = (torch.full((slots + spare, outs), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for to in (y, again):
        pj.es_project_experts(weights, x.cuda(), to, i32(start), workspace, rows=None if rows is None else i32(rows), gated=gated)
    assert not pj.es_project_gave_up(workspace)
    close(y[:slots], *R.experts(x, values, start, rows, gated))
    assert (y[slots:] == 7).all()
    assert torch.equal(y, again)


def test_experts_nan_in_absent_and_other_rows(pj):
    """Rows that an expert does not have do not reach those it has, nor does another expert's matrix."""
    g = torch.Generator().manual_seed(9)
    w = (normal(g, 3, 144, 128) / 11).bfloat16()
    w[1] = float("nan")
    x = normal(g, 20, 128).bfloat16()
    x[13:] = float("inf")
    start = [0, 4, 9, 13]
    weights = pj.es_weights_create(w.cuda())
    y = torch.empty(20, 144, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x.cuda(), y, i32(start), room(pj, weights, 20))
    want, off = R.experts(x, w, start)
    for lo, hi in ((0, 4), (9, 13)):
        close(y[lo:hi], want[lo:hi], off[lo:hi])
    assert torch.isnan(y[4:9]).all()


def test_starts_out_of_range_stay_within_the_buffers(pj):
    """Starts beyond the slots are bounded; nothing around y changes."""
    g = torch.Generator().manual_seed(10)
    w = (normal(g, 3, 64, 64) / 8).bfloat16()
    x = normal(g, 30, 64).bfloat16()
    weights = pj.es_weights_create(w.cuda())
    around = torch.full((90, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x.cuda(), around[30:60], i32([-5, 10, 25, 2 ** 31 - 1]), room(pj, weights, 30))
    close(around[30:60], *R.experts(x, w, [0, 10, 25, 30]))
    assert (around[:30] == 3).all() and (around[60:] == 3).all()


@pytest.mark.parametrize("count,top", [(1, 1), (5, 2), (32, 4), (33, 8), (64, 6), (128, 8), (200, 1), (600, 32), (1024, 5)])
@pytest.mark.parametrize("tokens", [1, 3, 96, 257, 5000])
@pytest.mark.parametrize("dtype,normalise", [(torch.bfloat16, True), (torch.float32, False)])
def test_route(pj, count, top, tokens, dtype, normalise):
    if tokens * count > 2e6:
        tokens = 1999
    g = torch.Generator().manual_seed(count * 7 + tokens)
    scores = (1.5 * normal(g, tokens, count + 3)).to(dtype)
    if tokens > 2:
        scores[tokens // 2] = -float("inf")           # a padded token
        scores[1, :max(1, count // 2)] = 0.5          # ties
        scores[2, ::2] = float("nan")
        scores[0, 0] = float("inf")
        if count > 2:
            scores[-1, 1:] = -float("inf")            # fewer than top are left
    x = scores[:, :count]                             # rows of an odd stride
    chosen, places = (torch.empty(tokens, top, dtype=torch.int32, device="cuda") for _ in range(2))
    weights = torch.empty(tokens, top, device="cuda")
    start = torch.empty(count + 1, dtype=torch.int32, device="cuda")
    rows = torch.full((tokens * top,), -7, dtype=torch.int32, device="cuda")
    space = torch.randint(0, 255, (pj.es_route_workspace(tokens, count, top),), dtype=torch.uint8, device="cuda")
    pj.es_route(scores.cuda()[:, :count], chosen, weights, start, rows, places, space, normalise=normalise)
    want = R.route(x, top, normalise)
    assert chosen.tolist() == want[0]
    assert start.tolist() == want[2]
    assert rows.tolist() == want[3] + [-7] * (tokens * top - len(want[3]))
    assert places.tolist() == want[4]
    w = torch.tensor(want[1], dtype=torch.float64)
    close(weights, w, (2.0 ** -20 + count * 2.0 ** -23) * w + 1e-44)


def test_route_of_no_tokens_writes_the_starts(pj):
    e = torch.empty(0, 4, dtype=torch.int32, device="cuda")
    start = torch.full((9,), 5, dtype=torch.int32, device="cuda")
    pj.es_route(torch.empty(0, 8, device="cuda"), e, torch.empty(0, 4, device="cuda"), start, e.view(-1), e.clone(),
                torch.empty(pj.es_route_workspace(0, 8, 4), dtype=torch.uint8, device="cuda"))
    assert start.tolist() == [0] * 9


@pytest.mark.parametrize("tokens,top,features,slots", [(1, 1, 8, 1), (7, 4, 1000, 20), (96, 6, 2560, 576), (3, 32, 264, 50),
                                                       (5, 2, 16, 0), (1200, 3, 136, 2000)])
@pytest.mark.parametrize("added", [False, True])
def test_combine(pj, tokens, top, features, slots, added):
    g = torch.Generator().manual_seed(tokens + top)
    y = normal(g, slots, features).bfloat16()
    places = torch.randint(-2, slots + 2, (tokens, top), generator=g)
    weights = normal(g, tokens, top)
    add = normal(g, tokens, features).bfloat16() if added else None
    out = torch.empty(tokens, features, dtype=torch.bfloat16, device="cuda")
    pj.es_combine(y.cuda(), places.int().cuda(), weights.cuda(), out, add=None if add is None else add.cuda())
    want = R.combine(y, places.tolist(), weights, add)
    close(out, *want)
    if added:  # in place
        both = add.cuda()
        pj.es_combine(y.cuda(), places.int().cuda(), weights.cuda(), both, add=both)
        assert torch.equal(both, out)


def test_combine_leaves_absent_rows_out(pj):
    """NaN in rows that no place names does not reach a token, and strided rows have their surroundings left alone."""
    g = torch.Generator().manual_seed(2)
    y_all = normal(g, 10, 80).bfloat16().cuda()
    y_all[3] = float("nan")
    out_all = torch.full((4, 96), 2.0, dtype=torch.bfloat16, device="cuda")
    places = [[0, -1], [9, 2], [-1, -1], [7, 10]]
    weights = normal(g, 4, 2)
    pj.es_combine(y_all[:, 8:72], i32(places), weights.cuda(), out_all[:, 16:80])
    close(out_all[:, 16:80], *R.combine(y_all[:, 8:72].cpu(), places, weights))
    assert (out_all[:, :16] == 2).all() and (out_all[:, 80:] == 2).all()


class Layer:
    """The layer of experts as a program runs it."""

    def __init__(self, pj, tokens, count=12, top=3, width=256, inner=136, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.pj, self.tokens, self.top, self.width, self.inner = pj, tokens, top, width, inner
        self.up = (normal(g, count, 2 * inner, width) * width ** -0.5).bfloat16()
        self.down = (normal(g, count, width, inner) * inner ** -0.5).bfloat16()
        self.up_handle, self.down_handle = pj.es_weights_create(self.up.cuda()), pj.es_weights_create(self.down.cuda())
        self.x = normal(g, tokens, width).bfloat16().cuda()
        self.scores = normal(g, tokens, count).cuda()
        n = tokens * top
        empty = lambda *s, dtype: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.chosen, self.places = empty(tokens, top, dtype=torch.int32), empty(tokens, top, dtype=torch.int32)
        self.weights, self.start = empty(tokens, top, dtype=torch.float32), empty(count + 1, dtype=torch.int32)
        self.rows = empty(n, dtype=torch.int32)
        self.h, self.z = empty(n, inner, dtype=torch.bfloat16), empty(n, width, dtype=torch.bfloat16)
        self.out = empty(tokens, width, dtype=torch.bfloat16)
        self.route_space = empty(pj.es_route_workspace(tokens, count, top), dtype=torch.uint8)
        self.workspace = room(pj, self.up_handle, n)

    def run(self, stream=None):
        pj = self.pj
        pj.es_route(self.scores, self.chosen, self.weights, self.start, self.rows, self.places, self.route_space, stream=stream)
        pj.es_project_experts(self.up_handle, self.x, self.h, self.start, self.workspace, rows=self.rows, gated=True, stream=stream)
        pj.es_project_experts(self.down_handle, self.h, self.z, self.start, self.workspace, stream=stream)
        pj.es_combine(self.z, self.places, self.weights, self.out, add=self.x, stream=stream)

    def check(self):
        """Each step against the definition, on what the step before has made."""
        chosen, weights, start, rows, places = R.route(self.scores.cpu(), self.top, True)
        assert self.chosen.tolist() == chosen and self.places.tolist() == places and self.start.tolist() == start
        n = start[-1]
        close(self.h[:n], *R.experts(self.x.cpu(), self.up, start, rows, True), "up")
        close(self.z[:n], *R.experts(self.h.cpu(), self.down, start), "down")
        close(self.out, *R.combine(self.z.cpu(), places, self.weights.cpu(), self.x.cpu()), "combine")


@pytest.mark.parametrize("tokens", [1, 5, 96, 700])
def test_layer_of_experts(pj, tokens):
    layer = Layer(pj, tokens)
    layer.scores[tokens // 2, :] = -float("inf") if tokens > 1 else 0.0
    layer.run()
    layer.check()


def test_layer_in_a_graph_with_other_scores(pj):
    """Row counts are read when the graph runs; two graphs share one workspace."""
    first, second = Layer(pj, 64), Layer(pj, 33, seed=1)
    second.workspace = first.workspace
    stream = torch.cuda.Stream()
    graphs = []
    for layer in (first, second):
        with torch.cuda.stream(stream):
            layer.run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.run()
        graphs.append(graph)
    for seed in range(3):
        for layer, graph in zip((first, second), graphs):
            layer.scores.copy_(torch.randn(layer.scores.shape, generator=torch.Generator().manual_seed(seed)))
            layer.x.mul_(1.5)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        first.check()
        second.check()


def test_project_in_a_graph_with_other_requests(pj):
    c = Case(pj, [40, 1, 30], [0, 1, 2], 320, 264)
    start, adapter = i32(c.start), i32(c.members)
    y = torch.full((c.n, c.out), 7.0, dtype=torch.bfloat16, device="cuda")
    call = lambda: pj.es_project(c.weights, c.xc, y, c.workspace, adapters=c.adapters, adapter=adapter, start=start)  # noqa: E731
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for counts, members in (([0, 50, 3], [2, -1, 0]), ([1, 1, 1], [2, 1, 0]), ([71, 0, 0], [1, 0, 0])):
        c.counts, c.members, c.start, c.n = counts, members, bounds(counts), sum(counts)
        start.copy_(i32(c.start)), adapter.copy_(i32(members))
        y.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        close(y[:c.n], *c.want())
        assert (y[c.n:] == 7).all()


def test_two_streams_with_their_workspaces(pj):
    cases = [Case(pj, [100, 7, 1], [0, 1, 2], 1264, 1000, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]
    results = [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for k, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                results[k].append(c.run())
    torch.cuda.synchronize()
    for c, ys in zip(cases, results):
        for y in ys:
            close(y, *c.want())
            assert torch.equal(y, ys[0])


def test_weights_change_between_calls(pj, es):
    """A handle reads its matrices when a call runs: es_perturb and es_restore between calls."""
    c = Case(pj, [5, 20], [0, -1], 512, 256)
    before = c.run()
    plan = es.plan_from_tensors([c.w.view(-1)])
    es.es_perturb(plan, 5, 0.05)
    c.values = c.w.cpu().double()
    close(c.run(), *c.want())
    assert not torch.equal(c.run(), before)
    plan.close()


def test_one_workspace_serves_calls_of_any_shape(pj):
    big = Case(pj, [300, 9, 1, 1], [0, 1, 2, 0], 1264, 1000, rank=64)
    small = Case(pj, [1, 2], [1, 0], 512, 256, rank=8, seed=4)
    small.workspace = big.workspace
    for c in (small, big, small, big):
        close(c.run(), *c.want())


def test_refusals(pj, es):
    c = Case(pj, [3, 2], [0, 1])
    y = torch.empty(c.n, c.out, dtype=torch.bfloat16, device="cuda")
    adapter, start = i32([0, 1]), i32(c.start)

    def refused(error, call, status=None):
        with pytest.raises(error) as e:
            call()
        if status is not None:
            assert e.value.status == status

    go = lambda **kw: pj.es_project(**(dict(weights=c.weights, x=c.xc, y=y, workspace=c.workspace, adapters=c.adapters,  # noqa: E731
                                            adapter=adapter, start=start) | kw))
    go()
    refused(ValueError, lambda: go(x=c.xc.float()))
    refused(ValueError, lambda: go(x=c.xc.cpu()))
    refused(ValueError, lambda: go(y=y[:, :-8]))
    refused(ValueError, lambda: go(y=y[:-1]))
    refused(ValueError, lambda: go(start=i32([0, 5])))
    refused(ValueError, lambda: go(adapter=adapter.long()))
    refused(es.EsError, lambda: go(adapters=None), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: go(adapter=None), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: go(start=None), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: go(workspace=c.workspace[:-1]), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: go(workspace=c.workspace[:0]), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: go(adapters=Case(pj, [1], [0], 512, 264).adapters), es.ES_ERR_INVALID_ARG)
    two = pj.es_weights_create(torch.zeros(2, 256, 512, dtype=torch.bfloat16, device="cuda"))
    refused(es.EsError, lambda: go(weights=two), es.ES_ERR_INVALID_ARG)
    x = torch.zeros(c.n, 516, dtype=torch.bfloat16, device="cuda")
    refused(es.EsError, lambda: go(x=x[:, :512]), es.ES_ERR_ALIGNMENT)
    x = torch.zeros(c.n, 520, dtype=torch.bfloat16, device="cuda")
    refused(es.EsError, lambda: go(x=x[:, 4:516]), es.ES_ERR_ALIGNMENT)
    w = torch.zeros(2, 24, 64, dtype=torch.bfloat16, device="cuda")
    weights = pj.es_weights_create(w)
    x = torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    z = torch.zeros(5, 12, dtype=torch.bfloat16, device="cuda")
    space = room(pj, weights, 5)
    refused(es.EsError, lambda: pj.es_project_experts(weights, x, z, i32([0, 2, 5]), space, gated=True), es.ES_ERR_INVALID_ARG)
    z = torch.zeros(5, 24, dtype=torch.bfloat16, device="cuda")
    refused(ValueError, lambda: pj.es_project_experts(weights, x, z, i32([0, 2]), space))
    refused(es.EsError, lambda: pj.es_project_experts(weights, x, z[:4], i32([0, 2, 4]), space), es.ES_ERR_INVALID_ARG)
    refused(ValueError, lambda: pj.es_weights_create(w.float()))
    refused(ValueError, lambda: pj.es_weights_create(w.cpu()))
    refused(ValueError, lambda: pj.es_weights_create(w.transpose(1, 2)))
    refused(es.EsError, lambda: pj.es_weights_create(w[:, :20]), es.ES_ERR_INVALID_ARG)
    refused(es.EsError, lambda: pj.es_weights_create(w.view(torch.uint8)), es.ES_ERR_INVALID_ARG)
    refused(ValueError, lambda: pj.es_adapters_create(c.a, c.b))
    refused(ValueError, lambda: pj.es_adapters_create(c.a.cuda(), c.b.cuda()[:2]))
    refused(es.EsError, lambda: pj.es_adapters_create(c.a.cuda()[:, :4].contiguous(), c.b.cuda()[:, :, :4].contiguous()), es.ES_ERR_INVALID_ARG)


def test_calls_of_no_rows(pj):
    c = Case(pj, [3, 2], [0, 1])
    none = torch.empty(0, 512, dtype=torch.bfloat16, device="cuda")
    pj.es_project(c.weights, none, torch.empty(0, 256, dtype=torch.bfloat16, device="cuda"), c.workspace, adapters=c.adapters,
                  adapter=i32([0, 1]), start=i32([0, 0, 0]))
    y = torch.full((3, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(c.weights, none, y, i32([0, 2]), c.workspace, rows=i32([0, 1, 2]))
    assert (y[:2] == 0).all() and (y[2] == 7).all()
    pj.es_combine(none, i32([]).view(0, 2), torch.empty(0, 2, device="cuda"), none)
