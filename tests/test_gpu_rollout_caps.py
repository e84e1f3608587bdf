"""es_attention with capped scores over the whole range of caps: both kernels against the
definition in 64 bits, with the tolerances of rollout_reference.py (scores within 1e-4)."""
import pytest

from test_gpu_rollout import Setup, check

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "e4m3"]


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1, 1], [2, 1, 2], [70, 3, 33]])
@pytest.mark.parametrize("cap", [1e-6, 0.3, 50.0, 1e3, 1e4, 1e6, 1e8])
def test_caps_of_every_size(ro, dtype, new, cap):
    check(Setup(ro, [200, 90, 333], new, 2, 128, 32, dtype, seed=21), 8, softcap=cap)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap", [2.0 ** 90, 2.0 ** 110, 3e38])
@pytest.mark.parametrize("new", [[1, 1], [40, 20]])
def test_caps_near_the_largest_number(ro, dtype, cap, new):
    check(Setup(ro, [90, 64], new, 2, 64, 16, dtype, seed=22), 8, softcap=cap)
