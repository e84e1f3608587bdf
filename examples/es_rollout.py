"""An ES generation whose members are rolled out with the rollout operators.

A small decoder (random bf16 weights) is perturbed in place for each member; the
perturbed model reads a batch of prompts and writes some tokens to each, over a paged
key/value cache; the reward is the share of written tokens with an even number. Then the
generation's update.

    python examples/es_rollout.py [--generations N] [--cache e4m3]

The model's products are torch's; head norms, rotation, cache and attention are
es_cache_append and es_attention, and es_cache_read shows what a layer's cache holds.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17310_gb300 import esopt as es  # noqa: E402
from paper_2608_17310_gb300 import rollout as ro  # noqa: E402

VOCAB, HIDDEN, LAYERS, Q_HEADS, KV_HEADS, HEAD_DIM, MLP = 256, 256, 2, 8, 2, 64, 512
PAGE, EPS = 16, 1e-6


def make_params(seed=0):
    """All of the model's tensors in one list, the way a plan takes them."""
    g = torch.Generator("cuda").manual_seed(seed)

    def weight(*shape):
        return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()

    p = {"embed": weight(VOCAB, HIDDEN)}
    for i in range(LAYERS):
        p |= {f"{i}.norm1": torch.ones(HIDDEN, device="cuda", dtype=torch.bfloat16),
              f"{i}.qkv": weight((Q_HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN),
              f"{i}.q_norm": torch.ones(HEAD_DIM, device="cuda", dtype=torch.bfloat16),
              f"{i}.k_norm": torch.ones(HEAD_DIM, device="cuda", dtype=torch.bfloat16),
              f"{i}.out": weight(HIDDEN, Q_HEADS * HEAD_DIM),
              f"{i}.norm2": torch.ones(HIDDEN, device="cuda", dtype=torch.bfloat16),
              f"{i}.up": weight(MLP, HIDDEN), f"{i}.down": weight(HIDDEN, MLP)}
    return p


def rope_table(rows):
    half = HEAD_DIM // 2
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * \
        1e4 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def norm(x, weight):
    x = x.float()
    return (x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * weight.float()).bfloat16()


class Rollout:
    """Caches, page table and buffers for `sequences` sequences of up to `longest` tokens,
    made once and used for every member."""

    def __init__(self, sequences, longest, dtype="bf16"):
        width = -(-longest // PAGE)
        pages = sequences * width
        self.sequences, self.width = sequences, width
        # any order of pages will do: a program's allocator hands them out as they come free
        self.table = torch.randperm(pages, device="cuda").to(torch.int32).view(sequences, width)
        self.seq_len = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.rope = rope_table(longest)
        shape = (pages, KV_HEADS, PAGE, HEAD_DIM)
        self.caches = []
        for _ in range(LAYERS):
            if dtype == "bf16":
                k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                self.caches.append(ro.es_cache_create(k, v))
            else:
                k, v = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
                ks, vs = (torch.zeros(shape[:3], device="cuda") for _ in range(2))
                self.caches.append(ro.es_cache_create(k, v, ks, vs))
        self.workspace = torch.zeros(ro.es_attention_workspace(self.caches[0], Q_HEADS), dtype=torch.uint8, device="cuda")
        self.step = ro.Batch(self.table, self.seq_len)  # one new token each

    def forward(self, params, tokens, batch):
        """Logits of the new tokens [tokens, VOCAB]; their keys and values go to the caches."""
        x = params["embed"][tokens]
        for i, cache in enumerate(self.caches):
            qkv = norm(x, params[f"{i}.norm1"]) @ params[f"{i}.qkv"].T
            q = torch.empty(len(tokens), Q_HEADS, HEAD_DIM, dtype=torch.bfloat16, device="cuda")
            ro.es_cache_append(cache, batch, qkv, q, params[f"{i}.q_norm"], params[f"{i}.k_norm"], self.rope, eps=EPS)
            out = torch.empty_like(q)
            ro.es_attention(cache, batch, q, out, self.workspace, scale=HEAD_DIM ** -0.5)
            x = x + out.view(len(tokens), -1) @ params[f"{i}.out"].T
            h = torch.nn.functional.silu(norm(x, params[f"{i}.norm2"]) @ params[f"{i}.up"].T)
            x = x + h @ params[f"{i}.down"].T
        return x @ params["embed"].T

    def run(self, params, prompts, new_tokens):
        """Greedy continuations [sequences, new_tokens] of prompts [sequences, length]."""
        b, n = prompts.shape
        self.seq_len.fill_(n)
        start = torch.arange(0, b * n + 1, n, dtype=torch.int32, device="cuda")
        prompt = ro.Batch(self.table, self.seq_len, start, b * n, n)
        logits = self.forward(params, prompts.reshape(-1), prompt).view(b, n, -1)[:, -1]
        written = [logits.argmax(-1)]
        for _ in range(new_tokens - 1):
            self.seq_len += 1
            written.append(self.forward(params, written[-1], self.step).argmax(-1))
        return torch.stack(written, 1)

    def cached(self, layer):
        """The keys and values that a layer's cache holds, all sequences end to end."""
        lengths = self.seq_len.cpu().tolist()
        start = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
        batch = ro.Batch(self.table, self.seq_len, start, sum(lengths), max(lengths))
        k, v = (torch.empty(sum(lengths), KV_HEADS, HEAD_DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ro.es_cache_read(self.caches[layer], batch, k, v)
        return k, v


def generations(count=3, members=24, sequences=32, prompt=24, new_tokens=12, sigma=0.01, alpha=0.02, dtype="bf16", seed=0):
    """Mean reward of each generation."""
    params = make_params(seed)
    plan = es.plan_from_tensors(list(params.values()))
    g = torch.Generator("cuda").manual_seed(seed + 1)
    roll = Rollout(sequences, prompt + new_tokens, dtype)
    history = []
    for t in range(count):
        prompts = torch.randint(0, VOCAB, (sequences, prompt), generator=g, device="cuda")
        seeds = [1 + 1000 * t + i for i in range(members)]
        rewards = []
        for s in seeds:
            es.es_perturb(plan, s, sigma)
            written = roll.run(params, prompts, new_tokens)
            rewards.append((written % 2 == 0).float().mean().item())
            es.es_restore(plan, s, sigma)
        if ro.es_attention_gave_up(roll.workspace):
            raise RuntimeError("es_attention gave up a wait: this generation's rewards are not to be used")
        rhat = es.es_normalize_rewards(rewards)
        es.es_update(plan, seeds, es.es_update_coeffs(rhat, alpha, sigma))
        history.append(sum(rewards) / members)
    plan.close()
    return history, roll


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--generations", type=int, default=20)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    a = ap.parse_args()
    history, roll = generations(a.generations, dtype=a.cache)
    for t, r in enumerate(history):
        print(f"generation {t}: mean reward {r:.4f}")
    k, v = roll.cached(0)
    print(f"layer 0 holds {k.shape[0]} tokens; rms of keys {k.float().pow(2).mean().sqrt():.3f}, of values "
          f"{v.float().pow(2).mean().sqrt():.3f}")


if __name__ == "__main__":
    main()
