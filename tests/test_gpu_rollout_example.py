"""The example that rolls members out with the rollout operators: its model's logits against the
same model in plain 32-bit torch over whole sequences, and its generations."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex(es):
    spec = importlib.util.spec_from_file_location("es_rollout_example", os.path.join(ROOT, "examples", "es_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(ex, p, tokens):
    """Logits of whole sequences [b, n] in 32 bits; activations are rounded where the model's are."""
    b, n = tokens.shape
    table = ex.rope_table(n)
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    f = lambda t: t.float()  # noqa: E731

    def turned(x, w):
        x = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + ex.EPS) * f(w)
        a, d = x.chunk(2, -1)
        return torch.cat([a * c - d * s, d * c + a * s], -1)

    x = p["embed"][tokens]
    for i in range(ex.LAYERS):
        qkv = (ex.norm(x, p[f"{i}.norm1"]) @ p[f"{i}.qkv"].T).view(b, n, -1, ex.HEAD_DIM).float()
        q = turned(qkv[:, :, :ex.Q_HEADS], p[f"{i}.q_norm"])
        k = turned(qkv[:, :, ex.Q_HEADS:-ex.KV_HEADS], p[f"{i}.k_norm"])
        v = qkv[:, :, -ex.KV_HEADS:]
        k, v = (t.repeat_interleave(ex.Q_HEADS // ex.KV_HEADS, 2) for t in (k, v))
        score = torch.einsum("bihd,bjhd->bhij", q, k) * ex.HEAD_DIM ** -0.5
        score = score.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -math.inf)
        out = torch.einsum("bhij,bjhd->bihd", score.softmax(-1), v).bfloat16()
        x = x + out.reshape(b, n, -1) @ p[f"{i}.out"].T
        x = x + torch.nn.functional.silu(ex.norm(x, p[f"{i}.norm2"]) @ p[f"{i}.up"].T) @ p[f"{i}.down"].T
    return x @ p["embed"].T


@pytest.mark.parametrize("dtype,bound", [("bf16", 0.05), ("e4m3", 0.25)])
def test_logits_match_the_plain_model(ex, dtype, bound):
    # logits are of size 1 and pass two layers; each bf16 rounding of an activation is worth
    # 2^-9 of it, about forty of them in a chain 0.03; E4M3 keys and values 2^-5 each, 0.15
    p = ex.make_params(3)
    roll = ex.Rollout(5, 40, dtype)
    prompts = torch.randint(0, ex.VOCAB, (5, 21), device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    start = torch.arange(0, 106, 21, dtype=torch.int32, device="cuda")
    roll.seq_len.fill_(21)
    got = [roll.forward(p, prompts.reshape(-1), ex.ro.Batch(roll.table, roll.seq_len, start, 105, 21)).view(5, 21, -1)]
    more = torch.randint(0, ex.VOCAB, (5, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    for i in range(4):  # the rest a token at a time
        roll.seq_len += 1
        got.append(roll.forward(p, more[:, i], roll.step)[:, None])
    got = torch.cat(got, 1).float()
    want = plain_logits(ex, p, torch.cat([prompts, more], 1)).float()
    assert (got - want).norm() <= bound * want.norm()
    k, v = roll.cached(0)
    assert k.shape == (125, ex.KV_HEADS, ex.HEAD_DIM) and torch.isfinite(k.float()).all() and (v != 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_generations_run(ex, dtype):
    first, _ = ex.generations(2, members=4, sequences=8, prompt=9, new_tokens=5, dtype=dtype)
    again, _ = ex.generations(2, members=4, sequences=8, prompt=9, new_tokens=5, dtype=dtype)
    assert len(first) == 2 and all(0.0 <= r <= 1.0 for r in first)
    assert first == again  # noise, rollouts and update are the same from run to run
