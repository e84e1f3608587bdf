"""The definitions of the products whose rows choose their weights, in 64 bits on the CPU, and the
tolerances of their tests. They share no code with the operators.

Tolerances, from the roundings that each operator makes:
  products   a sum of n products in fp32, in any order and with terms cut instead of rounded, is off by
             n 2^-23 of the sum of its terms' sizes; bf16 results by 2^-8 of their size, and 2^-134 (half
             the smallest bf16).
  project    also 2^-16 of each element of h = scale A x, which is kept as two bf16 numbers, through |B|.
  gated      silu has slopes within (-0.1, 1.1); exp and the division are off by 2^-20 of silu.
  route      a weight: exp, the sum of `experts` of them and the division, 2^-20 + experts 2^-23 of it.
  combine    as products, `top` + 1 terms."""
import math

import torch


def total(w, x, rows=None):
    """W x and the sums of its terms' sizes, [rows, out]."""
    w, x = w.double(), x.double()
    return x @ w.T, x.abs() @ w.abs().T


def bf16_off(y):
    return 2.0 ** -8 * y.abs() + 2.0 ** -134


def project(x, w, a=None, b=None, scale=None, member=None):
    """y and its tolerance. member: the adapter of each row, or -1."""
    y, size = total(w, x)
    off = (x.shape[1] + 8) * 2.0 ** -23 * size
    for i, m in enumerate(member or []):
        if m < 0:
            continue
        s = 1.0 if scale is None else float(scale[m])
        h, h_size = total(a[m], x[i:i + 1])
        h, h_size = s * h[0], abs(s) * h_size[0]
        h_off = 2.0 ** -16 * h.abs() + 2.0 ** -134 + (x.shape[1] + 8) * 2.0 ** -23 * h_size
        bm = b[m].double()
        y[i] += bm @ h
        off[i] += bm.abs() @ h_off + (len(h) + 8) * 2.0 ** -23 * (bm.abs() @ h.abs() + size[i])
    return y, off + bf16_off(y)


def experts(x, w, start, rows=None, gated=False):
    """y and its tolerance for the slots up to start[-1]; x of absent rows counts as zero."""
    out = w.shape[1] // 2 if gated else w.shape[1]
    y = torch.zeros(start[-1], out, dtype=torch.float64)
    off = torch.zeros_like(y)
    for g in range(w.shape[0]):
        lo, hi = start[g], start[g + 1]
        if hi <= lo:
            continue
        if rows is None:
            v = x[lo:hi]
        else:
            v = torch.zeros(hi - lo, x.shape[1], dtype=torch.float64)
            for i, r in enumerate(rows[lo:hi]):
                if 0 <= r < x.shape[0]:
                    v[i] = x[r].double()
        z, size = total(w[g], v)
        d = (x.shape[1] + 8) * 2.0 ** -23 * size
        if gated:
            p, q, dp, dq = z[:, :out], z[:, out:], d[:, :out], d[:, out:]
            s = p / (1 + torch.exp(-p))
            z = s * q
            d = 1.1 * dp * (q.abs() + dq) + s.abs() * dq + 2.0 ** -20 * z.abs()
        y[lo:hi], off[lo:hi] = z, d + bf16_off(z)
    return y, off


def route(scores, top, normalise):
    """chosen, weights, start, rows, places; token by token."""
    tokens, count = scores.shape
    chosen, weights, members = [], [], [[] for _ in range(count)]
    largest = torch.finfo(torch.float32).max
    for t, row in enumerate(scores.double().tolist()):
        row = [-math.inf if math.isnan(v) else min(v, largest) for v in row]
        best = [e for e in sorted(range(count), key=lambda e: (-row[e], e))[:top] if row[e] > -math.inf]
        p = [math.exp(v - row[best[0]]) if v > -math.inf else 0.0 for v in row] if best else []
        all_p = sum(p[e] for e in best) if normalise else sum(p)
        chosen.append(best + [-1] * (top - len(best)))
        weights.append([p[e] / all_p for e in best] + [0.0] * (top - len(best)))
        for j, e in enumerate(best):
            members[e].append((t, j))
    start, rows, places = [0], [], [[-1] * top for _ in range(tokens)]
    for pairs in members:
        for t, j in pairs:
            places[t][j] = len(rows)
            rows.append(t)
        start.append(len(rows))
    return chosen, weights, start, rows, places


def combine(y, places, weights, add=None):
    out = torch.zeros(len(places), y.shape[1], dtype=torch.float64)
    size = torch.zeros_like(out)
    for t, row in enumerate(places):
        for j, p in enumerate(row):
            if 0 <= p < y.shape[0]:
                out[t] += float(weights[t, j]) * y[p].double()
                size[t] += abs(float(weights[t, j])) * y[p].double().abs()
    if add is not None:
        out += add.double()
        size += add.double().abs()
    return out, (len(places[0]) + 1) * 2.0 ** -23 * size + bf16_off(out)
