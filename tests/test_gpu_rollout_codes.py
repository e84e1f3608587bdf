"""The numbers that an FP8 append writes, to the spacing of the codes, and what a rotation without its row
leaves.

Tolerances of the codes, from the roundings made: a value's y = x / scale passes three fp32 roundings
(the scale, its reciprocal, the product), 2^-22 of it at most; a key's also those of its norm and
rotation, 2^-20 of the vector's size, which is 448 in codes; then half a step of the grid."""
import pytest
import torch

import rollout_reference as R
from test_gpu_rollout import DTYPES, append_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


def turns(n):
    return [(7 * i) % 50 for i in range(n)]


def assert_codes(s, want, spots):
    """Scales and codes to the bounds above."""
    for of_keys, store, scale, w in ((True, s.k, s.ks, want[1]), (False, s.v, s.vs, want[2])):
        for t, sp in enumerate(spots):
            if sp is None or sp[2] < 0:
                continue
            got = R.e4m3(store.view(torch.uint8)[sp[2], :, sp[3]].cpu())
            fin = (w[t].abs().amax(-1) / 448).clamp_min(2.0 ** -126)
            assert ((scale[sp[2], :, sp[3]].cpu().double() - fin).abs() <= (2.0 ** -20 if of_keys else 2.0 ** -23) * fin).all()
            y = (w[t] / fin[:, None]).clamp(-448, 448)
            slack = 448 * 2.0 ** -20 if of_keys else 2.0 ** -22 * y.abs()
            assert ((got - y).abs() <= R.half_step(y) + slack).all()


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_are_the_nearest(ro, many, d):
    # elements of all sizes down to far below the smallest code
    new, lens = ((2000, 60), (2000, 70)) if many else ((19, 5), (30, 5))
    n = sum(new)
    g = torch.Generator().manual_seed(41)
    x = torch.randn(n, 10 * d, generator=g) * torch.pow(2.0, -torch.randint(0, 22, (n, 10 * d), generator=g).float())
    case = append_case(ro, "e4m3", d, d, new=new, lens=lens, x=x, page=64, positions=turns(n))
    assert_codes(case[0], case[2], case[3])


@pytest.mark.parametrize("n", [3, 2051])
def test_codes_of_a_scale_of_one(ro, n):
    # the largest element is 448, so scale and reciprocal are 1: every bf16 number goes to its nearest
    # code, ties to the even one, those below the smallest normal code included
    d = 128
    values = torch.arange(0x3800, 0x43E0).to(torch.int16).view(torch.bfloat16).float()  # 2^-15 and up to 448
    values = torch.cat([values, -values])
    x = torch.zeros(n, 10, d)
    x[:, 8:] = values[torch.arange(n * 2 * d).remainder(values.numel())].view(n, 2, d)
    x[:, 8:, 7] = 448
    s, _, _, spots, _ = append_case(ro, "e4m3", d, 0, new=(n,), lens=(n,), x=x.view(n, -1), weights=False, page=64)
    want = x[:, 8:].to(torch.float8_e4m3fn).double()
    pg, sl = (torch.tensor(v) for v in zip(*[(sp[2], sp[3]) for sp in spots]))
    assert (s.vs.cpu()[pg, :, sl] == 1).all()
    assert torch.equal(R.e4m3(s.v.view(torch.uint8).cpu())[pg, :, sl], want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_a_rotation_without_its_row_leaves_the_other_elements(ro, dtype, interleaved):
    # 32 of 128 elements turn: NaN without a row, the norm's result in the rest
    positions = [0, 49, 50, -1, 2 ** 31 - 1] * 5
    s, q, (wq, wk, _), spots, _ = append_case(ro, dtype, 128, 32, interleaved, positions=positions)
    for t, p in enumerate(positions):
        missing = not 0 <= p < 50
        got = q[t].cpu().double()
        assert torch.isnan(got[:, :32]).all() == missing and not torch.isnan(got[:, 32:]).any()
        if spots[t] is not None:
            key = s.k.view(torch.uint8) if dtype == "e4m3" else s.k
            key = key[spots[t][2], :, spots[t][3]].cpu()
            key = R.e4m3(key) if dtype == "e4m3" else key.double()
            assert torch.isnan(key[:, :32]).all() == missing and not torch.isnan(key[:, 32:]).any()
    s0, q0, (w0, _, _), _, _ = append_case(ro, dtype, 128, 32, interleaved, positions=[0] * 25)
    assert torch.equal(q[:, :, 32:], q0[:, :, 32:])  # the same seed: the same inputs, turned elsewhere
