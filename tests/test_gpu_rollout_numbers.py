"""Numbers that the C structures do not hold are refused by the binding, as a ValueError, not cut."""
import pytest
import torch

from test_gpu_rollout import Setup, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


def test_numbers_out_of_range(es, ro):
    s = Setup(ro, [20, 20], [2, 3], 2, 128, 16, "bf16")
    q = torch.zeros(5, 4, 128, dtype=torch.bfloat16, device="cuda")
    out, ws = torch.zeros_like(q), torch.zeros(ro.es_attention_workspace(s.cache, 4), dtype=torch.uint8, device="cuda")
    for kw in (dict(window=2 ** 31), dict(window=-2 ** 40), dict(window=1.5), dict(scale=None)):
        with pytest.raises(ValueError):
            ro.es_attention(s.cache, s.batch, q, out, ws, **dict(dict(scale=1.0), **kw))
    qkv = torch.zeros(5, 8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        ro.es_cache_append(s.cache, s.batch, qkv, q, interleaved=2 ** 32)
    # floats past fp32's range arrive as infinities, which the library refuses
    for kw in (dict(softcap=1e39), dict(scale=1e300)):
        with pytest.raises(es.EsError) as e:
            ro.es_attention(s.cache, s.batch, q, out, ws, **dict(dict(scale=1.0), **kw))
        assert e.value.status == es.ES_ERR_NONFINITE
    for kw in (dict(max_new=2 ** 32 + 1), dict(tokens=2 ** 32 + 5), dict(max_new=-2 ** 32 + 3)):
        with pytest.raises(ValueError):
            ro.Batch(i32(s.pages), i32(s.seq_len), i32(s.start), **dict(dict(tokens=5, max_new=3), **kw))
