"""The example of a population rolled out in one batch: it runs, all of its members' logits are those of a plain
model with each member's adapters, and an update moves the adapters that it is for."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex(es):
    import es_members
    return es_members


def plain_logits(ex, model, roll, tokens, each):
    """Logits of every position of every sequence, in 64 bits, each member by itself."""
    out = []
    for m in range(len(tokens) // each):
        x = model.embed.double()[tokens[m * each:(m + 1) * each]]
        n = x.shape[1]
        mask = torch.ones(n, n, device="cuda").triu(1).bool()
        turn = torch.view_as_complex(roll.rope.double())[:n, None]

        def norm(x):
            return x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + ex.EPS)

        def rotated(v):
            half = ex.HEAD_DIM // 2
            z = torch.complex(v[..., :half], v[..., half:]) * turn
            return torch.cat([z.real, z.imag], -1)

        for i in range(ex.LAYERS):
            w = model.qkv[i][0].double() + model.member_b[i][m].double() @ model.member_a[i][m].double()
            h = (norm(x) @ w.T).view(each, n, -1, ex.HEAD_DIM)
            q, k, v = h.split([ex.Q_HEADS, ex.KV_HEADS, ex.KV_HEADS], 2)
            q, k = rotated(q), rotated(k)
            k, v = (t.repeat_interleave(ex.Q_HEADS // ex.KV_HEADS, 2) for t in (k, v))
            s = torch.einsum("bihd,bjhd->bhij", q, k) * ex.HEAD_DIM ** -0.5
            o = torch.einsum("bhij,bjhd->bihd", s.masked_fill(mask, -torch.inf).softmax(-1), v).reshape(each, n, -1)
            x = x + o @ model.out[i].double().T
            y = norm(x)
            p = (y @ model.gate[i].double().T).softmax(-1)
            top = p.topk(ex.TOP, -1)[0][..., -1:]
            p = torch.where(p >= top, p, torch.zeros_like(p))
            p = p / p.sum(-1, keepdim=True)
            for e in range(ex.EXPERTS):
                z = y @ model.up[i][0][e].double().T
                z = torch.nn.functional.silu(z[..., :ex.INNER]) * z[..., ex.INNER:]
                x = x + p[..., e:e + 1] * (z @ model.down[i][0][e].double().T)
        out.append(norm(x) @ model.embed.double().T)
    return torch.cat(out)


def test_members_logits_are_a_plain_models(ex):
    members, each, n = 5, 3, 20
    model, roll = ex.Model(members), ex.Rollout(members, each, 32)
    model.perturb(list(range(1, members + 1)), 0.05)
    tokens = torch.randint(0, ex.VOCAB, (members * each, n), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    roll.seq_len.fill_(n)
    start = torch.arange(0, members * each * n + 1, n, dtype=torch.int32, device="cuda")
    batch = ex.ro.Batch(roll.table, roll.seq_len, start, members * each * n, n)
    got = roll.forward(model, tokens.reshape(-1), batch, start).view(members * each, n, -1).double()
    want = plain_logits(ex, model, roll, tokens, each)
    # bf16 roundings of every step; a token whose gating scores are near to one another may go to other experts
    off = (got - want).norm(dim=-1) / want.norm(dim=-1)
    assert (off < 0.05).double().mean() > 0.9, off
    # members differ by more than that
    assert (want[0] - want[each]).norm() > 0.2 * want[0].norm() or not torch.equal(tokens[0], tokens[each])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_generations_run_and_move_the_adapters(ex, dtype):
    history, model, _ = ex.generations(2, members=6, each=4, prompt=10, new_tokens=4, dtype=dtype)
    assert len(history) == 2 and all(0 <= r <= 1 for r in history)
    assert any(b.abs().sum() > 0 for b in model.b)
