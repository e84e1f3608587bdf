"""es_attention with capped scores over the whole range of caps: both kernels against the
definition in 64 bits, with the tolerances of rollout_reference.py (scores within 1e-4)."""
import pytest
import torch

from test_gpu_rollout import Setup, attend, check

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


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [70, 33]])
def test_unseen_keys_leave_capped_scores_as_they_are(ro, dtype, new):
    # the keys that no row but the last of a sequence sees become 2^6 as large: scores near the cap
    # beside small ones, and not a bit of the other rows changes
    s = Setup(ro, [100, 80], new, 2, 128, 32, dtype, seed=23)
    first = torch.full((s.tokens,), 9, dtype=torch.int32)
    last = torch.tensor([l - n + i + 1 for l, n in zip(s.seq_len, s.new) for i in range(n)], dtype=torch.int32)
    if max(new) == 1:
        last -= 1
    args = dict(first=first, last=last, softcap=100.0)
    q, out, lse = attend(s, 8, **args)
    for b, l in enumerate(s.seq_len):
        for p in (2, l - 1):
            page, slot = s.pages[b][p // 32], p % 32
            if dtype == "bf16":
                s.k[page, :, slot] *= 64
            else:
                s.ks[page, :, slot] *= 64
    _, out2, lse2 = attend(s, 8, q=q, **args)
    rows = [t for t in range(s.tokens) if max(new) == 1 or t + 1 not in s.start]
    assert torch.equal(out[rows].view(torch.int16), out2[rows].view(torch.int16)) and torch.equal(lse[rows], lse2[rows])
