"""es_attention over FP8 caches whose scales differ in sign: both kernels against the definition in 64
bits, with the tolerances of rollout_reference.py."""
import pytest
import torch

from test_gpu_rollout import Setup, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


NEW = [[1, 1], [2, 3], [40, 7]]


@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("signs", ["negative", "mixed", "one"])
def test_scales_of_either_sign(ro, new, d, signs):
    s = Setup(ro, [150, 75], new, 2, d, 32, "e4m3", seed=31)
    g = torch.Generator().manual_seed(32)
    for t in (s.ks, s.vs):
        sign = torch.where(torch.rand(t.shape, generator=g) < 0.5, -1.0, 1.0) if signs == "mixed" else -torch.ones(t.shape)
        if signs == "one":  # one value's scale alone, eight times the others'
            sign = torch.ones(t.shape)
            page, slot = s.pages[0][20 // 32], 20 % 32
            sign[page, :, slot] = -8.0
        t.mul_(sign.cuda())
    check(s, 4)
    check(s, 4, softcap=30.0, window=60)
