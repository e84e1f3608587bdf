"""The products whose rows choose their weights where they take other ways than the small cases: many rows
with members beside one another, many requests, every E4M3 code, scales that are zero, many rows that do not exist."""
import pytest
import torch

import project_reference as R
from test_gpu_project import Case, bounds, close, i32, matrices, normal, pj, room  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_many_rows_of_members_beside_one_another(pj, dtype, rank):  # noqa: F811
    """B h of mixed blocks of many rows."""
    counts = [1, 7, 40, 3, 0, 16, 90, 2] * 8 + [33]
    Case(pj, counts, [i % 6 - 1 for i in range(len(counts))], 320, 392, count=5, rank=rank, dtype=dtype, spare=7).check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rank", [8, 40])
def test_members_beside_one_another_through_many_features(pj, dtype, rank):  # noqa: F811
    """With more than 2^25 results B h of mixed blocks has no room and is made where they are written."""
    counts = [1, 7, 40, 3, 0, 16, 90, 2, 1] * 7
    Case(pj, counts, [i % 6 - 1 for i in range(len(counts))], 64, 30008, count=5, rank=rank, dtype=dtype, spare=3).check()


@pytest.mark.parametrize("requests", [127, 128, 129, 1000, 4096])
def test_many_requests(pj, requests):  # noqa: F811
    """Requests are looked up 32 at a time; many of them have no rows."""
    counts = [(0, 1, 0, 0, 2, 0, 1)[i % 7] if requests > 500 else i % 3 for i in range(requests)]
    Case(pj, counts, [(i * 7) % 12 - 1 for i in range(requests)], 128, 136, count=11, rank=16, seed=requests, spare=2).check()


def test_empty_requests_between_rows(pj):  # noqa: F811
    counts = [0] * 70 + [5] + [0] * 90 + [1] + [0] * 3 + [40] + [0] * 200
    Case(pj, counts, [i % 4 for i in range(len(counts))], 128, 136, count=4, spare=2).check()


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_every_code(pj, rows):  # noqa: F811
    """A row of x that is 1 in one place picks a column of codes: each comes back as the number that it is, times
    the scale, exactly where that is a power of two; NaN stays NaN and stays with its feature."""
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    w = torch.stack([codes.roll(7 * k) for k in range(64)], 1).contiguous()      # [256, 64]
    nan = (w & 0x7F) == 0x7F
    keep = torch.where(nan, torch.zeros_like(w), w)
    weights = pj.es_weights_create(w.cuda(), torch.tensor([0.25], device="cuda"))
    clean = pj.es_weights_create(keep.cuda(), torch.tensor([0.25], device="cuda"))
    x = torch.zeros(rows, 64, dtype=torch.bfloat16)
    pick = torch.arange(rows) % 64
    x[torch.arange(rows), pick] = 1
    y, z = (torch.empty(rows, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    space = room(pj, weights, rows)
    pj.es_project(weights, x.cuda(), y, space)
    pj.es_project(clean, x.cuda(), z, space)
    want = 0.25 * keep.view(torch.float8_e4m3fn).double()[:, pick].T
    assert torch.equal(z.cpu().double(), want)
    has_nan = nan.any(1)
    assert torch.isnan(y.cpu()[:, has_nan]).all()
    assert torch.equal(y.cpu()[:, ~has_nan].double(), want[:, ~has_nan])


@pytest.mark.parametrize("counts", [[3, 2], [40, 30], [200, 100]])
@pytest.mark.parametrize("scale", [0.0, 1e-39, -0.5])
def test_scales_of_zero_and_below(pj, counts, scale):  # noqa: F811
    """With adapters a scale without a finite reciprocal counts as 0, and the adapters' part stays."""
    c = Case(pj, counts, [1, -1], 320, 264, dtype="e4m3")
    c.w_scale.fill_(scale)
    c.weights = pj.es_weights_create(c.w, c.w_scale)
    exact = 0.0 if scale == 1e-39 else scale
    c.values = c.w.cpu().view(torch.float8_e4m3fn).double() * exact
    c.check()


@pytest.mark.parametrize("gated", [False, True])
def test_many_slots_without_rows(pj, gated):  # noqa: F811
    g = torch.Generator().manual_seed(4)
    w, _, _ = matrices(g, 2, 160, 64, "bf16")
    weights = pj.es_weights_create(w)
    y = torch.full((300, 80 if gated else 160), 7.0, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x, y, i32([0, 150, 290]), room(pj, weights, 300), rows=i32(list(range(300))), gated=gated)
    assert (y[:290] == 0).all() and (y[290:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_experts_of_many_and_few_rows_at_once(pj, dtype):  # noqa: F811
    """Column tiles of one expert beside those of others, over several bands of tiles and rounds of blocks."""
    g = torch.Generator().manual_seed(8)
    loads = [0, 700, 3, 0, 257, 256, 1, 512, 64, 0, 33, 900]
    start = bounds(loads)
    w, scale, values = matrices(g, len(loads), 784, 192, dtype)
    x = normal(g, 600, 192).bfloat16()
    rows = torch.randint(-1, 601, (start[-1],), generator=g).tolist()
    weights = pj.es_weights_create(w, scale)
    y = torch.empty(start[-1], 392, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x.cuda(), y, i32(start), room(pj, weights, start[-1]), rows=i32(rows), gated=True)
    close(y, *R.experts(x, values, start, rows, True))


@pytest.mark.parametrize("rows", [17, 64, 65, 200, 256, 257])
@pytest.mark.parametrize("width,out", [(4104, 264), (64, 8200)])
def test_rows_around_the_tiles(pj, rows, width, out):  # noqa: F811
    """Both sides of where tiles of other sizes begin, with a depth that blocks share and with many features."""
    Case(pj, [rows - 5, 5], [0, 1], width, out, seed=rows).check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("each,width,out", [(169, 2560, 1280), (78, 2432, 640), (20, 1280, 1280)])
def test_calls_over_cold_weights_agree(pj, dtype, each, width, out):  # noqa: F811
    """Many calls whose copies come in in any order: bit-identical. (A team of warps once took a stage's barrier
    for the one of five stages later, where a copy came in after the one behind it: one call of some thousand.)"""
    groups = 16
    w = [torch.randn(groups, out, width, device="cuda", dtype=torch.bfloat16).mul_(0.02) for _ in range(3)]
    if dtype == "e4m3":
        scale = torch.full((groups,), 2.0 ** -11, device="cuda")
        handles = [pj.es_weights_create((v * 2 ** 11).to(torch.float8_e4m3fn), scale) for v in w]
    else:
        handles = [pj.es_weights_create(v) for v in w]
    start = i32(bounds([each + (7 * i) % 13 - 6 for i in range(groups)]))
    slots = int(start[-1])
    x = torch.randn(slots, width, device="cuda").bfloat16()
    space = room(pj, handles[0], slots)
    first, flush = [], torch.empty(192 << 20, dtype=torch.uint8, device="cuda")
    for i in range(450):
        y = torch.empty(slots, out, dtype=torch.bfloat16, device="cuda")
        pj.es_project_experts(handles[i % 3], x, y, start, space)
        if i % 5 == 0:
            flush.zero_()
        if i < 3:
            first.append(y)
        elif not torch.equal(y.view(torch.int16), first[i % 3].view(torch.int16)):
            raise AssertionError(f"call {i} differs")
