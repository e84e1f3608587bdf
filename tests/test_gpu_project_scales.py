"""FP8 matrices with scales far from 1, with adapters beside them and without. Definitions and tolerances:
project_reference.py. With adapters, a scale whose reciprocal is infinite counts as 0; results here are all finite."""
import pytest
import torch

import project_reference as R
from test_gpu_project import Case, bounds, close, i32, matrices, normal, pj, room  # noqa: F401

pytestmark = pytest.mark.gpu

# zero, subnormal, the smallest normal numbers, both sides of 2^-32 and 2^32, large
SCALES = [1.2e-38, 1e-36, 1e-20, -1e-25, 2.0 ** -33, 2.0 ** -32, 2.0 ** -31, 2.0 ** 32, -2.0 ** 33, 1e30]


def rescaled(pj, c, scale):  # noqa: F811
    """A third of the features have codes of zero, so that the adapters' part is all that they are."""
    c.w[:, ::3] = 0
    c.w_scale.fill_(scale)
    c.weights = pj.es_weights_create(c.w, c.w_scale)
    c.values = c.w.cpu().view(torch.float8_e4m3fn).double() * c.w_scale.double().cpu()[:, None, None]
    return c


# rows of one adapter and beside others', one request, many rows, with and without a second block of rows
@pytest.mark.parametrize("counts,members", [([3, 2], [1, -1]), ([1], [2]), ([40], [0]), ([40, 30, 1, 1, 9], [1, -1, 0, 2, 1]),
                                            ([200, 100], [1, -1]), ([300], [1]), ([90, 1, 1, 200], [0, 1, -1, 2])])
@pytest.mark.parametrize("scale", SCALES)
def test_adapters_beside_matrices_of_any_scale(pj, counts, members, scale):  # noqa: F811
    rescaled(pj, Case(pj, counts, members, 320, 264, dtype="e4m3"), scale).check()


@pytest.mark.parametrize("rank", [8, 40, 128])
def test_ranks_beside_a_small_scale(pj, rank):  # noqa: F811
    rescaled(pj, Case(pj, [40, 30, 1, 1, 9], [1, -1, 0, 2, 1], 320, 264, rank=rank, dtype="e4m3"), 1.2e-38).check()


@pytest.mark.parametrize("counts,members", [([3, 2], [1, -1]), ([40], [0]), ([90, 1, 1, 200], [0, 1, -1, 2])])
@pytest.mark.parametrize("scale", [1e38, -3.4e38])
def test_adapters_beside_codes_of_zero_and_the_largest_scales(pj, counts, members, scale):  # noqa: F811
    c = Case(pj, counts, members, 320, 264, dtype="e4m3")
    c.w.zero_()
    rescaled(pj, c, scale).check()


def test_a_scale_that_is_no_number_reaches_every_result(pj):  # noqa: F811
    for scale in (float("nan"), float("inf")):
        c = rescaled(pj, Case(pj, [40, 3], [1, -1], 320, 264, dtype="e4m3"), scale)
        assert not torch.isfinite(c.run()).any()
