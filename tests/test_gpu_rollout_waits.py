"""Waits of the kernel of many rows that run out: the call returns, says so in its workspace, and the
workspace serves again once it has been zeroed. No wait outlasts the test; the limit is set to nothing."""
import ctypes

import pytest
import torch

from test_gpu_rollout import DTYPES, Setup, assert_attention, attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


@pytest.fixture
def wait_tries(es):
    call = es.lib().es_attention_wait_tries
    call.argtypes, call.restype = [ctypes.c_int], None
    yield call
    call(-1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[40, 3], [300, 129]])
def test_a_given_up_wait_is_told(ro, wait_tries, dtype, d, new):
    s = Setup(ro, [400, 150], new, 2, d, 32, dtype, seed=61)
    q, out, lse = attend(s, 8)
    ws = torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)

    def call():
        ro.es_attention(s.cache, s.batch, q, got, ws, scale=s.d ** -0.5, lse=got_lse)
        return ro.es_attention_gave_up(ws)

    assert not call()
    wait_tries(0)
    assert call()
    wait_tries(-1)
    assert ro.es_attention_gave_up(ws)  # until it is zeroed
    ws.zero_()
    assert not call()
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    assert_attention(s, q, got, got_lse)


def test_few_rows_wait_for_nothing(ro, wait_tries):
    s = Setup(ro, [400, 150], [1, 1], 2, 128, 32, "bf16", seed=62)
    wait_tries(0)
    q, out, lse = attend(s, 8)
    assert_attention(s, q, out, lse)
