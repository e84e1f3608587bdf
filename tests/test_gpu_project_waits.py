"""Waits of the products' kernel that run out: the call is flagged, nothing hangs, and the workspace
serves again once it has been zeroed. The limit is set to nothing by a hook of the library's."""
import pytest
import torch

import project_reference as R
from test_gpu_project import Case, bounds, i32, matrices, normal, pj, room, close  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_tries(es):
    import ctypes
    es.lib().es_project_wait_tries.argtypes = [ctypes.c_int]
    es.lib().es_project_wait_tries.restype = None
    yield lambda n: es.lib().es_project_wait_tries(n)
    es.lib().es_project_wait_tries(-1)


# one row and a share each, several rows whose depth is shared, pairs, pairs with rows of several members
@pytest.mark.parametrize("counts", [[1], [30, 7], [300], [90, 1, 1, 200]])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_waits_that_run_out_are_told(pj, no_tries, counts, dtype):  # noqa: F811
    c = Case(pj, counts, [0, 1, -1, 2][:len(counts)], 2048, 520, dtype=dtype)
    for tries in (0, 1):
        no_tries(tries)
        c.run()
        torch.cuda.synchronize()
        if tries == 0:
            assert pj.es_project_gave_up(c.workspace)
        no_tries(-1)
        c.workspace.zero_()
        close(c.run(), *c.want())
        assert not pj.es_project_gave_up(c.workspace)


def test_experts_whose_waits_run_out(pj, no_tries):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    w, _, values = matrices(g, 4, 272, 512, "bf16")
    x = normal(g, 20, 512).bfloat16()
    rows = [3, 19, 0, 7, 7, 2, 11, 5, 6, 1]
    start = bounds([3, 0, 5, 2])
    weights = pj.es_weights_create(w)
    space = room(pj, weights, 10)
    y = torch.empty(10, 136, dtype=torch.bfloat16, device="cuda")
    no_tries(0)
    pj.es_project_experts(weights, x.cuda(), y, i32(start), space, rows=i32(rows), gated=True)
    assert pj.es_project_gave_up(space)
    no_tries(-1)
    space.zero_()
    pj.es_project_experts(weights, x.cuda(), y, i32(start), space, rows=i32(rows), gated=True)
    close(y, *R.experts(x, values, start, rows, True))
    assert not pj.es_project_gave_up(space)
