"""The rollout operators' definitions in 64 bits on the CPU, token by token, and the
tolerances of their tests. They share no code with the operators.

Tolerances, from the roundings that each operator makes:
  append     bf16 numbers are 2^-7 of their power of two apart, so a bf16 result is off by
             2^-8 of its size, plus 2^-20 of the vector's size for the fp32 arithmetic before
             it; an E4M3 code by half a step of the grid (2^-4 of its power of two, 2^-10
             below 2^-6), plus 2^-15 of 448 for that arithmetic; a scale by 2^-20 of it.
  read       nothing for bf16; one bf16 rounding (2^-8) for codes.
  attention  with A = sum p |v|, the largest that an output's parts add up to: 2^-8 A for
             exp(x) rounded to bf16, 2^-8 A for the result's rounding, 2^-12 A for the scores
             (an fp32 score of size up to 100 is off by 1e-4 at most, which is the relative
             error of exp), with A and the result in exact arithmetic. lse: 1e-4, the
             scores' error."""
import math

import torch


def places(pages, page_size, seq_len, new):
    """(sequence, position, page, slot) of each new token; None where it has no place."""
    out = []
    for b, n in enumerate(new):
        for i in range(n):
            p = seq_len[b] - n + i
            ok = 0 <= p < len(pages[b]) * page_size
            out.append((b, p, pages[b][p // page_size], p % page_size) if ok else None)
    return out


def append(qkv, q_heads, kv_heads, d, q_weight, k_weight, eps, rope, positions, interleaved):
    """q, k, v of every token as float64 [tokens, heads, d] before any rounding."""
    x = qkv.double().reshape(qkv.shape[0], q_heads + 2 * kv_heads, d).clone()
    q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]

    def head(y, w):
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        y = y.clone()
        if rope is None:
            return y
        half = rope.shape[1]
        for t in range(y.shape[0]):
            p = positions[t]
            if p is None or not 0 <= p < rope.shape[0]:
                y[t] = float("nan")
                continue
            c, s = rope[p, :, 0].double(), rope[p, :, 1].double()
            a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else \
                (slice(0, half), slice(half, 2 * half))
            ya, yb = y[t][:, a].clone(), y[t][:, b].clone()
            y[t][:, a], y[t][:, b] = ya * c - yb * s, yb * c + ya * s
        return y

    return head(q, q_weight), head(k, k_weight), v


def attention(q, k, v, seq_len, new, scale, softcap=0.0, slopes=None, window=0, first=None, last=None,
              absent=None):
    """out, A, lse in float64. k[b], v[b]: the sequence's vectors [len, kv_heads, d]; absent[b]:
    positions that hold no token."""
    tokens, heads, d = q.shape
    out = torch.zeros(tokens, heads, d, dtype=torch.float64)
    size = torch.zeros_like(out)
    lse = torch.full((tokens, heads), -math.inf, dtype=torch.float64)
    t = 0
    for b, n in enumerate(new):
        kv = k[b].shape[1]
        for i in range(n):
            p = seq_len[b] - n + i
            lo = 0 if first is None else max(0, int(first[t]))
            hi = p + 1 if last is None else int(last[t])
            if window:
                lo = max(lo, p - window + 1)
            hi = min(hi, seq_len[b])
            at = [j for j in range(lo, hi) if absent is None or j not in absent[b]]
            if p >= 0 and at:
                for h in range(heads):
                    g = h // (heads // kv)
                    x = (k[b][at, g].double() @ q[t, h].double()) * scale
                    if softcap:
                        x = softcap * torch.tanh(x / softcap)
                    if slopes is not None:
                        x = x - float(slopes[h]) * (p - torch.tensor(at, dtype=torch.float64)).abs()
                    lse[t, h] = torch.logsumexp(x, 0)
                    w = torch.softmax(x, 0)
                    out[t, h] = w @ v[b][at, g].double()
                    size[t, h] = w @ v[b][at, g].double().abs()
            t += 1
    return out, size, lse


def e4m3(codes):
    return codes.view(torch.uint8).view(torch.float8_e4m3fn).double()


def half_step(c):
    """Half the spacing of the E4M3 grid at |c|."""
    e = torch.floor(torch.log2(c.abs().clamp(2.0 ** -6, 448)))
    return 2.0 ** (e - 4)
