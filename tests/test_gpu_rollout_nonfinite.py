"""es_attention over values that are infinities and NaN for some rows and unseen by others: few of them
and so many that the kernel of many rows no longer lists them, against the definition in 64 bits (with the
tolerances of rollout_reference.py where that is finite), and what one of them costs."""
import math

import numpy as np
import pytest
import torch

import rollout_reference as R
from test_gpu_rollout import DTYPES, Setup, attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


def spoil(s, share, seed):
    """Infinities, NaN and (FP8) scales that are either, in a share of the values."""
    g = torch.Generator().manual_seed(seed)
    pages, heads, page, d = s.v.shape
    hit = torch.rand(pages, heads, page, generator=g) < share
    where = torch.randint(0, d, (pages, heads, page, 1), generator=g)
    at = (torch.arange(d) == where) & hit[..., None]
    kind = torch.randint(0, 3, (pages, heads, page), generator=g)
    bad = torch.tensor([math.inf, -math.inf, math.nan])[kind]
    if s.dtype == "bf16":
        s.v.copy_(torch.where(at, bad[..., None], s.v.cpu().float()).bfloat16())
    else:
        codes = s.v.view(torch.uint8)
        codes.copy_(torch.where(at, torch.tensor(0xFF, dtype=torch.uint8), codes.cpu()))
        of_scale = hit & (torch.rand(hit.shape, generator=g) < 0.2)
        s.vs.copy_(torch.where(of_scale, bad, s.vs.cpu()))


def assert_as_defined(s, q, out, lse, first, last):
    k, v = s.dense()
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, s.d ** -0.5, first=first, last=last)
    got = out.cpu().double()
    assert torch.equal(torch.isnan(want), torch.isnan(got))
    endless = torch.isinf(want)
    assert torch.equal(endless, torch.isinf(got)) and torch.equal(want[endless], got[endless])
    fine = torch.isfinite(want)
    assert ((got - want).abs()[fine] <= ((2.0 ** -7 + 2.0 ** -12) * size)[fine]).all()
    hit = want_lse > -math.inf
    assert torch.equal(hit, lse.cpu() > -math.inf)
    assert ((lse.cpu().double() - want_lse)[hit].abs() <= 1e-4).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("share", [0.004, 0.5])
@pytest.mark.parametrize("new", [[1, 2], [70, 40], [150, 3]])
def test_values_that_some_rows_see(ro, dtype, d, share, new):
    s = Setup(ro, [700, 150], new, 2, d, 32, dtype, seed=51)
    spoil(s, share, 52)
    rng = np.random.default_rng(53)
    first = torch.tensor(rng.integers(-20, 120, s.tokens), dtype=torch.int32)
    last = torch.tensor(rng.integers(60, 720, s.tokens), dtype=torch.int32)
    first[-1] = 1000  # sees nothing
    q, out, lse = attend(s, 4, first=first, last=last)
    assert_as_defined(s, q, out, lse, first, last)


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_such_value_costs_little(ro, dtype):
    # the last tokens alone see it; at first every value of the unit was read again for each row
    s = Setup(ro, [20000, 9000], [40, 30], 1, 128, 64, dtype, seed=54)
    first = torch.zeros(s.tokens, dtype=torch.int32, device="cuda")
    first[3] = 10 ** 6  # sees nothing
    q = torch.randn(s.tokens, 8, 128, generator=s.g).bfloat16().cuda()
    out, ws = torch.empty_like(q), torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")

    def ms():
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ro.es_attention(s.cache, s.batch, q, out, ws, scale=s.d ** -0.5, first=first)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    clean = ms()
    assert torch.isfinite(out.float()).all()
    at = s.seq_len[0] - 20
    page, slot = s.pages[0][at // 64], at % 64
    if dtype == "bf16":
        s.v[page, 0, slot, 9] = math.inf
    else:
        s.v.view(torch.uint8)[page, 0, slot, 9] = 0x7F
    spoiled = ms()
    assert not torch.isfinite(out[20:40, :, 9].float()).any()
    other = out.float()
    other[20:40, :, 9] = 0
    assert torch.isfinite(other).all()
    assert spoiled <= 3 * clean + 1.0, f"{spoiled:.2f} ms in place of {clean:.2f}"


def test_an_empty_row_costs_little(ro):
    # a row that sees nothing makes no tile one whose values have to be looked through
    sequences, new, length = 24, 60, 8192
    pages = sequences * length // 64
    k, v = (torch.randn(pages, 8, 64, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = ro.es_cache_create(k, v)
    table = torch.arange(pages, device="cuda", dtype=torch.int32).view(sequences, -1)
    start = torch.arange(0, sequences * new + 1, new, device="cuda", dtype=torch.int32)
    batch = ro.Batch(table, torch.full((sequences,), length, dtype=torch.int32, device="cuda"), start, sequences * new, new)
    q = torch.randn(sequences * new, 32, 128, device="cuda").bfloat16()
    out, ws = torch.empty_like(q), torch.zeros(ro.es_attention_workspace(cache, 32), dtype=torch.uint8, device="cuda")
    first = torch.zeros(sequences * new, dtype=torch.int32, device="cuda")

    def us():
        times = []
        for _ in range(9):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                ro.es_attention(cache, batch, q, out, ws, scale=128 ** -0.5, first=first)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b) * 100)
        return sorted(times)[4]

    us()
    without = us()
    first[3::new] = 10 ** 6
    with_one = us()
    assert (out[3::new] == 0).all()
    assert with_one <= 1.4 * without, f"{with_one:.0f} us in place of {without:.0f}"


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_cache_of_nan_costs_little(ro, dtype):
    # as a member whose parameters went wrong leaves it: every value of every token is NaN
    n = 3001
    s = Setup(ro, [n], [n], 2, 128, 64, dtype, seed=55)
    q = torch.randn(n, 8, 128, generator=s.g).bfloat16().cuda()
    out, ws = torch.empty_like(q), torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")

    def ms():
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ro.es_attention(s.cache, s.batch, q, out, ws, scale=s.d ** -0.5)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    clean = ms()
    assert torch.isfinite(out.float()).all()
    if dtype == "bf16":
        s.v.fill_(math.nan)
    else:
        s.v.view(torch.uint8).fill_(0x7F)
    spoiled = ms()
    assert torch.isnan(out.float()).all()
    assert spoiled <= 3 * clean + 1.0, f"{spoiled:.2f} ms in place of {clean:.2f}"
