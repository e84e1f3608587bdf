"""An ES generation over low-rank adapters whose members are all rolled out in one batch.

A member's perturbation is of its copy of the adapters alone (es_perturb on that copy), so the
weights that they stand beside are shared: every step of the rollouts reads them once for the whole
population, with es_project. Each layer's feed-forward part is a layer of experts: es_route,
es_project_experts and es_combine. The reward is the share of written tokens with an even number; the
update goes to the adapters.

    python examples/es_members.py [--generations N] [--weights e4m3]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17310_gb300 import esopt as es  # noqa: E402
from paper_2608_17310_gb300 import project as pj  # noqa: E402
from paper_2608_17310_gb300 import rollout as ro  # noqa: E402

VOCAB, HIDDEN, LAYERS, Q_HEADS, KV_HEADS, HEAD_DIM = 256, 256, 2, 8, 2, 64
EXPERTS, TOP, INNER, RANK, PAGE, EPS = 8, 2, 128, 8, 16, 1e-6
QKV = (Q_HEADS + 2 * KV_HEADS) * HEAD_DIM


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + EPS)).bfloat16()


class Model:
    """Shared weights, and `members` copies of the adapters [members, ...] beside the qkv projections."""

    def __init__(self, members, dtype="bf16", seed=0):
        g = torch.Generator("cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()

        def shared(*shape):
            w = weight(*shape)
            if dtype == "bf16":
                return w, pj.es_weights_create(w)
            scale = w.float().abs().amax((-2, -1)) / 448
            codes = (w.float() / scale[..., None, None]).to(torch.float8_e4m3fn)
            return codes, pj.es_weights_create(codes, scale)

        self.embed = weight(VOCAB, HIDDEN)
        self.qkv, self.up, self.down = ([shared(*s) for _ in range(LAYERS)] for s in
                                        ((QKV, HIDDEN), (EXPERTS, 2 * INNER, HIDDEN), (EXPERTS, HIDDEN, INNER)))
        self.out, self.gate = ([weight(*s) for _ in range(LAYERS)] for s in ((HIDDEN, Q_HEADS * HEAD_DIM), (EXPERTS, HIDDEN)))
        # the adapters that the updates go to, and each member's copy of them
        self.a = [weight(RANK, HIDDEN) for _ in range(LAYERS)]
        self.b = [torch.zeros(QKV, RANK, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.member_a = [a.repeat(members, 1, 1) for a in self.a]
        self.member_b = [b.repeat(members, 1, 1) for b in self.b]
        self.adapters = [pj.es_adapters_create(a, b) for a, b in zip(self.member_a, self.member_b)]
        self.plan = es.plan_from_tensors(self.a + self.b)
        bases = [s.index_base for s in es.segments_from_tensors(self.a + self.b)]
        # a member's tensors have the global indices of those that are updated, so that a seed gives them one direction
        self.member_plans = [es.plan_from_tensors([t[m] for t in self.member_a + self.member_b], bases) for m in range(members)]

    def perturb(self, seeds, sigma):
        for copy, own in zip(self.member_a + self.member_b, self.a + self.b):
            copy.copy_(own.expand_as(copy))
        for plan, seed in zip(self.member_plans, seeds):
            es.es_perturb(plan, seed, sigma)


class Rollout:
    """Buffers of all members' sequences, `each` of them a member."""

    def __init__(self, members, each, longest):
        n = members * each
        width = -(-longest // PAGE)
        self.sequences = n
        self.table = torch.randperm(n * width, device="cuda").to(torch.int32).view(n, width)
        self.seq_len = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.member = torch.arange(n, device="cuda", dtype=torch.int32) // each
        shape = (n * width, KV_HEADS, PAGE, HEAD_DIM)
        self.caches = [ro.es_cache_create(*(torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
                       for _ in range(LAYERS)]
        half = HEAD_DIM // 2
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * \
            1e4 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        self.rope = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        self.attention_space = torch.zeros(ro.es_attention_workspace(self.caches[0], Q_HEADS), dtype=torch.uint8, device="cuda")
        self.spaces = {}

    def space(self, kind, size):
        if kind not in self.spaces or self.spaces[kind].numel() < size:
            self.spaces[kind] = torch.zeros(size, dtype=torch.uint8, device="cuda")
        return self.spaces[kind]

    def experts(self, model, i, x):
        """The layer of experts of tokens x, added to them."""
        n = len(x)
        new = lambda *s, dtype: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        chosen, places, weights = new(n, TOP, dtype=torch.int32), new(n, TOP, dtype=torch.int32), new(n, TOP, dtype=torch.float32)
        start, rows = new(EXPERTS + 1, dtype=torch.int32), new(n * TOP, dtype=torch.int32)
        h, z, out = new(n * TOP, INNER, dtype=torch.bfloat16), new(n * TOP, HIDDEN, dtype=torch.bfloat16), torch.empty_like(x)
        y = norm(x)
        pj.es_route((y @ model.gate[i].T).float(), chosen, weights, start, rows, places,
                    self.space("route", pj.es_route_workspace(n, EXPERTS, TOP)))
        pj.es_project_experts(model.up[i][1], y, h, start, self.space("up", pj.es_project_workspace(model.up[i][1], n * TOP)),
                              rows=rows, gated=True)
        pj.es_project_experts(model.down[i][1], h, z, start, self.space("down", pj.es_project_workspace(model.down[i][1], n * TOP)))
        pj.es_combine(z, places, weights, out, add=x)
        return out

    def forward(self, model, tokens, batch, start):
        """Logits of the new tokens [tokens, VOCAB] of all members."""
        x = model.embed[tokens]
        n = len(x)
        for i, cache in enumerate(self.caches):
            qkv = torch.empty(n, QKV, dtype=torch.bfloat16, device="cuda")
            handle = model.qkv[i][1]
            pj.es_project(handle, norm(x), qkv, self.space("qkv", pj.es_project_workspace(handle, n, model.adapters[i])),
                          adapters=model.adapters[i], adapter=self.member, start=start)
            q = torch.empty(n, Q_HEADS, HEAD_DIM, dtype=torch.bfloat16, device="cuda")
            ro.es_cache_append(cache, batch, qkv, q, rope=self.rope, eps=EPS)
            out = torch.empty_like(q)
            ro.es_attention(cache, batch, q, out, self.attention_space, scale=HEAD_DIM ** -0.5)
            x = x + out.view(n, -1) @ model.out[i].T
            x = self.experts(model, i, x)
        return norm(x) @ model.embed.T

    def run(self, model, prompts, new_tokens):
        """Greedy continuations [sequences, new_tokens] of prompts [sequences, length]."""
        b, n = prompts.shape
        self.seq_len.fill_(n)
        start = torch.arange(0, b * n + 1, n, dtype=torch.int32, device="cuda")
        prompt = ro.Batch(self.table, self.seq_len, start, b * n, n)
        logits = self.forward(model, prompts.reshape(-1), prompt, start).view(b, n, -1)[:, -1]
        written = [logits.argmax(-1)]
        step = ro.Batch(self.table, self.seq_len)
        for _ in range(new_tokens - 1):
            self.seq_len += 1
            written.append(self.forward(model, written[-1], step, None).argmax(-1))
        if ro.es_attention_gave_up(self.attention_space) or \
                any(pj.es_project_gave_up(s) for k, s in self.spaces.items() if k != "route"):
            raise RuntimeError("a kernel gave up a wait: this rollout is not to be used")
        return torch.stack(written, 1)


def generations(count=3, members=16, each=8, prompt=24, new_tokens=12, sigma=0.05, alpha=0.05, dtype="bf16", seed=0):
    """Mean reward of each generation."""
    model, roll = Model(members, dtype, seed), Rollout(members, each, prompt + new_tokens)
    g = torch.Generator("cuda").manual_seed(seed + 1)
    history = []
    for t in range(count):
        prompts = torch.randint(0, VOCAB, (each, prompt), generator=g, device="cuda").repeat(members, 1)
        seeds = [1 + 1000 * t + i for i in range(members)]
        model.perturb(seeds, sigma)
        written = roll.run(model, prompts, new_tokens)
        rewards = (written % 2 == 0).float().mean(1).view(members, each).mean(1).tolist()
        rhat = es.es_normalize_rewards(rewards)
        es.es_update(model.plan, seeds, es.es_update_coeffs(rhat, alpha, sigma))
        history.append(sum(rewards) / members)
    return history, model, roll


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--generations", type=int, default=20)
    ap.add_argument("--weights", choices=("bf16", "e4m3"), default="bf16")
    a = ap.parse_args()
    for t, r in enumerate(generations(a.generations, dtype=a.weights)[0]):
        print(f"generation {t}: mean reward {r:.4f}")


if __name__ == "__main__":
    main()
