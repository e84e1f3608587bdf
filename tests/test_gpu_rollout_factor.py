"""es_attention with factors of the scores that are negative, zero and small, in both kernels, against the
definition in 64 bits with the tolerances of rollout_reference.py."""
import math

import pytest
import torch

import rollout_reference as R
from test_gpu_rollout import DTYPES, Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [2, 3], [60, 20]])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 1e-6])
@pytest.mark.parametrize("kw", [{}, {"softcap": 4.0}, {"slopes": True, "window": 40}], ids=["plain", "cap", "slopes"])
def test_factors_of_the_scores(ro, dtype, new, scale, kw):
    kw = dict(kw)
    s = Setup(ro, [300, 75], new, 2, 128, 32, dtype, seed=71)
    slopes = 2.0 ** -torch.arange(1, 9, dtype=torch.float32) if kw.pop("slopes", None) else None
    q = (1.5 * torch.randn(s.tokens, 8, 128, generator=s.g)).bfloat16().cuda()
    out, lse = torch.empty_like(q), torch.empty(s.tokens, 8, device="cuda")
    ws = torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")
    ro.es_attention(s.cache, s.batch, q, out, ws, scale=scale, lse=lse, slopes=None if slopes is None else slopes.cuda(), **kw)
    k, v = s.dense()
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, scale, slopes=slopes, **kw)
    assert ((out.cpu().double() - want).abs() <= (2.0 ** -7 + 2.0 ** -12) * size).all()
    assert (want_lse > -math.inf).all() and ((lse.cpu().double() - want_lse).abs() <= 1e-4).all()
