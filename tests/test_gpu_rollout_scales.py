"""es_attention over FP8 caches whose scales differ in sign and in size, and with queries whose
elements do: both kernels against the definition in 64 bits.

Tolerances: those of rollout_reference.py (A = sum p |v|), and where scales differ in size what the
f16 numbers of the few-rows kernel leave out: exp(x) times a value's scale is held there in units in
which the row's largest such product is at least 2^12, and f16 numbers below 2^-14 are 2^-24 apart, so
each key's is off by 2^-37 of the largest, times a code of up to 448."""
import pytest
import torch

import rollout_reference as R
from test_gpu_rollout import Setup, assert_attention, attend, check

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


def assert_spread(s, q, out, lse):
    k, v = s.dense()
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, s.d ** -0.5)
    heads = q.shape[1]
    extra = torch.zeros(s.tokens, heads, 1, dtype=torch.float64)
    t = 0
    for b, n in enumerate(s.new):
        l = s.seq_len[b]
        scale = torch.stack([s.vs.cpu().double()[s.pages[b][p // s.page], :, p % s.page] for p in range(l)]).abs()
        for i in range(n):
            seen = l - n + i + 1
            for h in range(heads):
                g = h // (heads // s.kv_heads)
                w = torch.softmax((k[b][:seen, g] @ q[t, h].cpu().double()) * s.d ** -0.5, 0)
                extra[t, h] = seen * 2.0 ** -37 * 448 * (w * scale[:seen, g]).max()
            t += 1
    err = (out.cpu().double() - want).abs()
    bound = (2.0 ** -7 + 2.0 ** -12) * size + extra
    assert (err <= bound).all(), f"off by {(err / bound.clamp_min(1e-300)).max():.3g} of the bound"
    assert ((lse.cpu().double() - want_lse).abs() <= 1e-4).all()


@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("bits", [10, 40])
def test_value_scales_of_very_different_size(ro, new, bits):
    s = Setup(ro, [150, 75], new, 2, 128, 32, "e4m3", seed=33)
    g = torch.Generator().manual_seed(34)
    power = torch.randint(-bits, bits + 1, s.vs.shape, generator=g)
    s.vs.mul_(torch.pow(2.0, power.float()).cuda())
    q, out, lse = attend(s, 4)
    assert_spread(s, q, out, lse)


@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("at", [3, 70, 140])
@pytest.mark.parametrize("weight", [3.0, 6.0])
@pytest.mark.parametrize("power", [-40, 40])
def test_the_weight_on_a_key_whose_value_scale_differs(ro, new, at, weight, power):
    # queries along one key, whose value's scale is 2^power of the others'
    s = Setup(ro, [150], new[:1], 2, 128, 32, "e4m3", seed=35)
    page, slot = s.pages[0][at // 32], at % 32
    s.vs[page, :, slot] *= 2.0 ** power
    k, _ = s.dense()
    q = (weight * k[0][at].repeat_interleave(2, 0)).bfloat16().expand(s.tokens, 4, 128).contiguous().cuda()
    q, out, lse = attend(s, 4, q=q)
    assert_spread(s, q, out, lse)


@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("d", [64, 128])
def test_queries_with_one_large_element(ro, new, d):
    # an element 2^22 times the others, at which every key is 0: the others decide
    s = Setup(ro, [150, 75], new, 2, d, 32, "e4m3", seed=36)
    s.k.view(torch.uint8)[..., 5] = 0
    q = 1.5 * torch.randn(s.tokens, 4, d, generator=s.g)
    q[..., 5] = 2.0 ** 22
    q, out, lse = attend(s, 4, q=q.bfloat16().cuda())
    assert_attention(s, q, out, lse)
