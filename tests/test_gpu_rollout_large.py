"""es_cache_append and es_cache_read of 2,048 tokens and more, whose kernels take eight tokens a block,
with the tolerances of rollout_reference.py."""
import pytest
import torch

import rollout_reference as R
from test_gpu_rollout import Setup, append_case, assert_appended

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "e4m3"]


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


NEW, LENS = (1500, 0, 1, 700, 13), (1503, 3, 40, 690, 13)  # 2,214 tokens; ten of the fourth have no place


def turns(n=sum(NEW)):
    return [(7 * i) % 50 for i in range(n)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,rotary,interleaved", [(128, 128, False), (128, 32, False), (128, 48, True), (128, 0, False),
                                                  (64, 64, False), (64, 16, True), (64, 32, False)])
def test_append_of_many_tokens(ro, dtype, d, rotary, interleaved):
    assert_appended(*append_case(ro, dtype, d, rotary, interleaved, new=NEW, lens=LENS, positions=turns(), page=64))


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_of_many_tokens_options(ro, dtype):
    many = dict(new=NEW, lens=LENS, page=128)
    assert_appended(*append_case(ro, dtype, 128, 128, in_place=True, positions=turns(), **many))
    assert_appended(*append_case(ro, dtype, 64, 64, in_place=True, wide=40, positions=turns(), **many))
    assert_appended(*append_case(ro, dtype, 128, 64, weights=False, positions=turns(), q_heads=16, kv_heads=1, **many))
    assert_appended(*append_case(ro, dtype, 64, 32, q_heads=3, kv_heads=3, positions=turns(), **many))
    # positions without a rope row
    assert_appended(*append_case(ro, dtype, 128, 128, positions=([49, 50, -1, 2 ** 31 - 1, 0] * 443)[:sum(NEW)], **many))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv_heads", [1, 3])
def test_read_of_many_tokens(ro, dtype, d, kv_heads):
    s = Setup(ro, LENS, NEW, kv_heads, d, 32, dtype, seed=3)
    s.pages[0][7] = -1
    s.pages[3][2] = 10 ** 9
    s.remake()
    k, v = (torch.full((s.tokens, kv_heads, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ro.es_cache_read(s.cache, s.batch, k, v)
    for pair in ((k, None), (None, v)):
        only = [None if t is None else torch.full_like(t, 6.0) for t in pair]
        ro.es_cache_read(s.cache, s.batch, *only)
        assert all(t is None or torch.equal(t, o) for t, o in zip(pair, only))
    stored = [R.e4m3(t.cpu()) * sc.cpu().double()[..., None] if sc is not None else t.cpu().double()
              for t, sc in ((s.k, s.ks), (s.v, s.vs))]
    spots = R.places(s.pages, 32, s.seq_len, s.new)
    for got, want in zip((k, v), stored):
        w = torch.stack([want[sp[2], :, sp[3]] if sp and 0 <= sp[2] < want.shape[0] else torch.zeros(kv_heads, d).double()
                         for sp in spots])
        assert ((got.cpu().double() - w).abs() <= (2.0 ** -8 * w.abs() if dtype == "e4m3" else 0)).all()
