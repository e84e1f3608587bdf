"""The example of a population rolled out in one batch tells its members apart: with the same prompts for all, each
sequence's logits are those of a plain model with its own member's adapters, and far from any other member's."""
import pytest
import torch

from test_gpu_project_example import ex, plain_logits  # noqa: F401

pytestmark = pytest.mark.gpu


def test_each_members_logits_are_its_own(ex):  # noqa: F811
    members, each, n = 4, 2, 12
    model, roll = ex.Model(members), ex.Rollout(members, each, 32)
    model.perturb(list(range(1, members + 1)), 0.1)
    prompts = torch.randint(0, ex.VOCAB, (each, n), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    tokens = prompts.repeat(members, 1)
    roll.seq_len.fill_(n)
    start = torch.arange(0, members * each * n + 1, n, dtype=torch.int32, device="cuda")
    batch = ex.ro.Batch(roll.table, roll.seq_len, start, members * each * n, n)
    got = roll.forward(model, tokens.reshape(-1), batch, start).view(members * each, n, -1).double()
    want = plain_logits(ex, model, roll, tokens, each)
    size = want.norm(dim=-1)
    # bf16 roundings of every step; a token whose gating scores are near to one another may go to other experts
    assert ((got - want).norm(dim=-1) / size < 0.05).double().mean() > 0.9
    for other in range(1, members):
        moved = want.roll(other * each, 0)
        # plain models of two members differ by some 0.7 to 1.4 at this perturbation, ten times what is allowed above
        assert ((want - moved).norm(dim=-1) / size).min() > 0.5
        assert ((got - moved).norm(dim=-1) / size).min() > 0.25
