"""The gate of es_project_experts, silu(v) = v / (1 + exp(-v)), over the whole range of its argument. One element of x
is 1 and the others are 0, so both products are single numbers and exact.

Tolerance: 2^-20 of the result for exp, the divisions and the product in fp32, half a step of the smallest fp32 numbers for silu itself
(2^-150; 2^-149 for the two roundings of it) times the other factor, and the result's own bf16 rounding."""
import pytest
import torch

from project_reference import bf16_off
from test_gpu_project import i32, pj, room  # noqa: F401

pytestmark = pytest.mark.gpu

GATES = [float(v) for v in torch.arange(-104, 104.5, 0.5)] + [0.0, -0.0, 2.0 ** -20, -2.0 ** -126, 2.0 ** -133, -300.0, 3e4, -1e30, 1e30]


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("factor", [1.0, -2.0 ** 60, 1.5 * 2.0 ** -10, 2.0 ** 110])
def test_gates_of_any_size(pj, rows, factor):  # noqa: F811
    gate = torch.tensor([v for v in GATES if abs(v) * abs(factor) < 2.0 ** 127] + [0.0] * 7).bfloat16()
    n = len(gate) // 8 * 8
    gate = gate[:n]
    w = torch.zeros(1, 2 * n, 64, dtype=torch.bfloat16)
    w[0, :n, 5], w[0, n:, 5] = gate, factor
    x = torch.zeros(rows, 64, dtype=torch.bfloat16)
    x[:, 5] = 1
    weights = pj.es_weights_create(w.cuda())
    y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x.cuda(), y, i32([0, rows]), room(pj, weights, rows), gated=True)
    v, q = gate.double(), float(torch.tensor(factor).bfloat16())
    silu = torch.where(v < 0, v * torch.exp(v) / (1 + torch.exp(v)), v / (1 + torch.exp(-v)))
    want = silu * q
    off = 2.0 ** -20 * want.abs() + 2.0 ** -149 * abs(q) + bf16_off(want)
    bad = (y.double().cpu() - want).abs() > off
    assert not bad.any(), [(float(gate[i]), float(y[r, i]), float(want[i])) for r, i in bad.nonzero().tolist()[:8]]


def test_gates_that_are_no_numbers(pj):  # noqa: F811
    """silu(inf) = inf, and -inf / inf and NaN are NaN."""
    gate = torch.tensor([float("inf"), -float("inf"), float("nan"), 1, 1, 1, 1, 1]).bfloat16()
    w = torch.zeros(1, 16, 64, dtype=torch.bfloat16)
    w[0, :8, 5], w[0, 8:, 5] = gate, 2.0
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    x[:, 5] = 1
    weights = pj.es_weights_create(w.cuda())
    y = torch.empty(3, 8, dtype=torch.bfloat16, device="cuda")
    pj.es_project_experts(weights, x.cuda(), y, i32([0, 3]), room(pj, weights, 3), gated=True)
    assert (y[:, 0] == float("inf")).all() and torch.isnan(y[:, 1:3]).all() and torch.isfinite(y[:, 3:]).all()
