"""The operators of products whose rows choose their weights, whose speed is measured: a
projection that all requests share with a low-rank adapter of each request beside it, and
the layer of experts (tokens to experts, products grouped by expert, back to tokens).

A case is one call of one operator ("op"):

  project   es_project: y = W x, plus B (A x) with the adapter of the row's request
  experts   es_project_experts: rows sorted by expert, each expert's times its own matrix,
            the rows gathered from the tokens and the product gated, or neither
  route     es_route: the largest gating scores of each token, and the rows of each expert
  combine   es_combine: the weighted sum of a token's rows, beside what is added to it

Row counts follow from the case alone; the seed gives values, orders and scores.
"""
import math
import random

import torch

own = False


# --- the cases ---------------------------------------------------------------------

def listed():
    return [
        # one sequence's next token, the query, key and value projection of the 4B-shaped set: latency of one call
        {"name": "project_token", "op": "project", "requests": 1, "rows_lo": 1, "rows_hi": 1, "adapters": 16,
         "rank": 16, "in": 2560, "out": 6144, "dtype": "bf16", "bare": 0},
        # a decode step of a whole population at once, each member with its adapter; the 27B-shaped set
        {"name": "project_step", "op": "project", "requests": 192, "rows_lo": 1, "rows_hi": 1, "adapters": 30,
         "rank": 16, "in": 5120, "out": 7168, "dtype": "bf16", "bare": 0},
        # a smaller step through FP8 weights, some requests without an adapter; down projection of the 4B-shaped set
        {"name": "project_step_e4m3", "op": "project", "requests": 45, "rows_lo": 1, "rows_hi": 1, "adapters": 16,
         "rank": 8, "in": 9728, "out": 2560, "dtype": "e4m3", "bare": 7},
        # the ragged prompts of 30 members at once, up projection of the 27B-shaped set
        {"name": "project_prompts", "op": "project", "requests": 30, "rows_lo": 211, "rows_hi": 701, "adapters": 30,
         "rank": 32, "in": 5120, "out": 17408, "dtype": "bf16", "bare": 0},
        # one token through its experts: latency
        {"name": "experts_token", "op": "experts", "tokens": 1, "top": 4, "experts": 32, "in": 2560, "out": 1280,
         "dtype": "bf16", "gathered": True, "gated": True},
        # a decode step of a population, gate and up products of many small experts
        {"name": "experts_step", "op": "experts", "tokens": 96, "top": 6, "experts": 64, "in": 2560, "out": 1280,
         "dtype": "bf16", "gathered": True, "gated": True},
        # the down product of a step through FP8 experts
        {"name": "experts_down_e4m3", "op": "experts", "tokens": 200, "top": 4, "experts": 48, "in": 1280, "out": 2560,
         "dtype": "e4m3", "gathered": False, "gated": False},
        # a long prompt's gate and up products, a quarter of the 4B-shaped set's feed-forward width an expert
        {"name": "experts_prompt", "op": "experts", "tokens": 8191, "top": 4, "experts": 32, "in": 2560, "out": 2432,
         "dtype": "bf16", "gathered": True, "gated": True},
        # a decode step's tokens to their experts
        {"name": "route_step", "op": "route", "tokens": 96, "top": 6, "experts": 64, "dtype": "bf16", "padded": 5,
         "normalise": True},
        # a long prompt's tokens to many experts
        {"name": "route_prompt", "op": "route", "tokens": 16383, "top": 8, "experts": 128, "dtype": "f32", "padded": 0,
         "normalise": True},
        # a decode step's rows back to their tokens
        {"name": "combine_step", "op": "combine", "tokens": 96, "top": 6, "out": 2560, "padded": 5, "add": True},
        # a long prompt's rows back to their tokens, hidden size of the 27B-shaped set
        {"name": "combine_prompt", "op": "combine", "tokens": 8191, "top": 4, "out": 5120, "padded": 0, "add": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, one row to some thousands, both weight types, sizes of the 4B- and 27B-shaped sets
    and odd ones, ranks of 8 to 64, requests of one row, of few and of many, experts from 4 to 128."""
    op = rng.choice(["project", "project", "project", "experts", "experts", "experts", "route", "combine"])
    c = {"op": op}
    if op == "project":
        c["requests"] = _log_uniform(rng, 1, 256)
        hi = rng.choice([1, 1, _log_uniform(rng, 2, 40), _log_uniform(rng, 20, 4000)])
        hi = max(1, min(hi, 12000 // c["requests"]))
        c["rows_lo"], c["rows_hi"] = max(1, int(hi * rng.uniform(0.2, 1.0))), hi
        c["adapters"] = _log_uniform(rng, 1, 64)
        c["rank"] = rng.choice([8, 16, 16, 32, 40, 64])
        c["in"], c["out"] = rng.choice([(2560, 6144), (4096, 2560), (2560, 9728), (9728, 2560), (5120, 7168),
                                        (5120, 5120), (17408, 5120), (1264, 1000), (720, 2072)])
        c["dtype"] = rng.choice(["bf16", "bf16", "e4m3"])
        c["bare"] = rng.choice([0, 0, 5, 9])
        return c
    c["tokens"] = _log_uniform(rng, 1, 7000)
    c["experts"] = rng.choice([4, 8, 16, 32, 60, 64, 128])
    c["top"] = rng.choice([k for k in (1, 2, 4, 6, 8) if k <= c["experts"] // 2])
    if op == "experts":
        c["top"] = min(c["top"], 4)
        c["gated"] = rng.random() < 0.5
        c["gathered"] = c["gated"] or rng.random() < 0.3
        c["in"], c["out"] = rng.choice([(2560, 1280), (1280, 2560), (2560, 2432), (2432, 2560), (1264, 728), (880, 1016)])
        c["dtype"] = rng.choice(["bf16", "bf16", "e4m3"])
        return c
    c["padded"] = rng.choice([0, 0, c["tokens"] // 7])
    if op == "route":
        c["dtype"] = rng.choice(["bf16", "f32"])
        c["normalise"] = rng.random() < 0.7
        return c
    del c["experts"]
    c["out"] = rng.choice([2560, 4096, 5120, 1000])
    c["add"] = rng.random() < 0.5
    return c


def _rows(c):
    """Rows of each request, an even, unordered spread over the case's range."""
    lo, hi = c["rows_lo"], c["rows_hi"]
    return [hi - int((hi - lo + 1) * ((i * 0.6180339887) % 1.0)) for i in range(c["requests"])]


def _adapters(c):
    """Adapter of each request: members in turn, every bare-th request without one (-1)."""
    return [-1 if c["bare"] and i % c["bare"] == c["bare"] - 1 else i * c["adapters"] // c["requests"] if
            c["requests"] >= c["adapters"] else i * 7 % c["adapters"] for i in range(c["requests"])]


def _loads(c):
    """Rows of each expert: uneven, some with none, tokens * top in all, none above the tokens."""
    n, e, left = c["tokens"], c["experts"], c["tokens"] * c["top"]
    share = [0.0 if i % 11 == 7 else 0.3 + (i * 0.7548776662) % 1.0 for i in range(e)]
    loads = [min(n, int(left * s / sum(share))) for s in share]
    left -= sum(loads)
    i = 0
    while left > 0:
        if share[i % e] and loads[i % e] < n:
            loads[i % e] += 1
            left -= 1
        i += 5 if e % 5 else 7
    return loads


def _bounds(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


# --- inputs ------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)
    dev, bf = torch.device("cuda"), torch.bfloat16
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=g, device=dev, dtype=dtype)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"case": c}

    def matrices(*shape):
        """Weights N(0, 0.02^2): bf16, or E4M3 numbers with max|w| / 448 of each matrix as its scale."""
        w = normal(*shape, dtype=bf).mul_(0.02)
        if c["dtype"] == "bf16":
            return w, None
        scale = w.float().abs().amax((-2, -1)) / 448
        return (w / scale[..., None, None]).to(torch.float8_e4m3fn), scale

    def hidden(rows):
        """Rows as they come out of a norm: channels of different size."""
        return (normal(rows, c["in"]) * torch.exp(0.4 * normal(c["in"]))).to(bf)

    if c["op"] == "project":
        rows = _rows(c)
        s["bounds"], s["members"] = _bounds(rows), _adapters(c)
        s["start"], s["adapter"] = ints(s["bounds"]), ints(s["members"])
        n = s["bounds"][-1]
        s["w"], s["w_scale"] = matrices(1, c["out"], c["in"])
        s["a"] = (normal(c["adapters"], c["rank"], c["in"]) * c["in"] ** -0.5).to(bf)
        s["b"] = (normal(c["adapters"], c["out"], c["rank"]) * 0.1).to(bf)
        s["scale"] = 0.5 + torch.rand(c["adapters"], generator=g, device=dev)
        s["x"] = hidden(n)
        s["y"] = torch.empty(n, c["out"], dtype=bf, device=dev)
    elif c["op"] == "experts":
        loads = _loads(c)
        s["bounds"] = _bounds(loads)
        s["start"] = ints(s["bounds"])
        slots = s["bounds"][-1]
        s["w"], s["w_scale"] = matrices(c["experts"], c["out"] * (2 if c["gated"] else 1), c["in"])
        s["x"] = hidden(c["tokens"] if c["gathered"] else slots)
        s["rows"] = None
        if c["gathered"]:
            order = torch.rand(c["experts"], c["tokens"], generator=g, device=dev).argsort(-1)
            s["rows"] = torch.cat([order[e, :k].sort()[0] for e, k in enumerate(loads)]).to(torch.int32)
        s["y"] = torch.empty(slots, c["out"], dtype=bf, device=dev)
    elif c["op"] == "route":
        x = 1.5 * normal(c["tokens"], c["experts"]) + 0.7 * normal(c["experts"])
        if c["padded"]:
            x[-c["padded"]:] = -math.inf
        s["scores"] = x.to(bf) if c["dtype"] == "bf16" else x
        n, k = c["tokens"], c["top"]
        s["chosen"], s["places"] = (torch.empty(n, k, dtype=torch.int32, device=dev) for _ in range(2))
        s["weights"] = torch.empty(n, k, device=dev)
        s["start"] = torch.empty(c["experts"] + 1, dtype=torch.int32, device=dev)
        s["rows"] = torch.full((n * k,), -1, dtype=torch.int32, device=dev)
    else:
        n, k = c["tokens"] - c["padded"], c["top"]
        s["y"] = normal(n * k, c["out"], dtype=bf)
        s["places"] = torch.full((c["tokens"], k), -1, dtype=torch.int32, device=dev)
        s["places"][:n] = torch.randperm(n * k, generator=g, device=dev).to(torch.int32).view(n, k)
        s["weights"] = torch.softmax(1.5 * normal(c["tokens"], k), -1)
        s["add"] = normal(c["tokens"], c["out"], dtype=bf) if c["add"] else None
        s["out"] = torch.empty(c["tokens"], c["out"], dtype=bf, device=dev)
    if own:
        from paper_2608_17310_gb300 import project as pj
        if "w" in s:
            s["handle"] = pj.es_weights_create(s["w"], s["w_scale"])
        if c["op"] == "project":
            s["handles"] = pj.es_adapters_create(s["a"], s["b"], s["scale"])
            need = pj.es_project_workspace(s["handle"], len(s["x"]), s["handles"])
        elif c["op"] == "experts":
            need = pj.es_project_workspace(s["handle"], len(s["y"]))
        elif c["op"] == "route":
            need = pj.es_route_workspace(c["tokens"], c["experts"], c["top"])
        else:
            need = 0
        s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=dev)
    return s


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        return _own(s, op)
    return {"project": _plain_project, "experts": _plain_experts, "route": _plain_route, "combine": _plain_combine}[op](s)


def _own(s, op):
    from paper_2608_17310_gb300 import project as pj
    c = s["case"]
    if op == "project":
        pj.es_project(s["handle"], s["x"], s["y"], s["workspace"], adapters=s["handles"], adapter=s["adapter"],
                      start=s["start"])
        return s["y"]
    if op == "experts":
        pj.es_project_experts(s["handle"], s["x"], s["y"], s["start"], s["workspace"], rows=s["rows"], gated=c["gated"])
        return s["y"]
    if op == "route":
        pj.es_route(s["scores"], s["chosen"], s["weights"], s["start"], s["rows"], s["places"], s["workspace"],
                    normalise=c["normalise"])
        return _routed(s)
    pj.es_combine(s["y"], s["places"], s["weights"], s["out"], add=s["add"])
    return s["out"]


def _routed(s):
    return {k: s[k] for k in ("chosen", "weights", "start", "rows", "places")}


# --- the plain forms ---------------------------------------------------------------

def _matrix(s, g):
    w = s["w"][g].float()
    return w if s["w_scale"] is None else w * s["w_scale"][g]


def _plain_project(s):
    c = s["case"]
    x = s["x"].float()
    y = x @ _matrix(s, 0).T
    if c["rows_hi"] == 1:
        m = s["adapter"].clamp_min(0).long()
        h = (s["a"][m].float() @ x[:, :, None]) * s["scale"][m][:, None, None]
        y += torch.where(s["adapter"][:, None] >= 0, (s["b"][m].float() @ h)[..., 0], torch.zeros_like(y))
    else:
        for lo, hi, m in zip(s["bounds"], s["bounds"][1:], s["members"]):
            if m >= 0:
                h = (x[lo:hi] @ s["a"][m].float().T) * s["scale"][m]
                y[lo:hi] += h @ s["b"][m].float().T
    return y.to(torch.bfloat16)


def _plain_experts(s):
    c = s["case"]
    x = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
    y = torch.empty_like(s["y"])
    for e, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if hi == lo:
            continue
        z = x[lo:hi].float() @ _matrix(s, e).T
        if c["gated"]:
            gate, up = z[:, :c["out"]], z[:, c["out"]:]
            z = gate / (1 + torch.exp(-gate)) * up
        y[lo:hi] = z.to(torch.bfloat16)
    return y


def _plain_route(s):
    c = s["case"]
    n, k, e = c["tokens"], c["top"], c["experts"]
    x = s["scores"].float()
    value, index = x.sort(dim=-1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k]
    there = value > -math.inf
    top = torch.where(there[:, :1], value[:, :1], torch.zeros_like(value[:, :1]))
    p = torch.exp(value - top)
    total = p.sum(-1, keepdim=True) if c["normalise"] else torch.exp(x - top).sum(-1, keepdim=True)
    s["weights"].copy_(torch.where(there, p / total, torch.zeros_like(p)))
    s["chosen"].copy_(torch.where(there, index, -1))
    key = torch.where(there, index, e).reshape(-1)
    order = key.argsort(stable=True)
    at = torch.arange(n * k, device=x.device)
    s["start"].copy_((key[None] < torch.arange(e + 1, device=x.device)[:, None]).sum(-1))
    place = torch.empty_like(at)
    place[order] = at
    s["places"].copy_(torch.where(there, place.view(n, k), -1))
    s["rows"].copy_(torch.where(at < s["start"][e], order // k, s["rows"]))
    return _routed(s)


def _plain_combine(s):
    there = (s["places"] >= 0)[..., None]
    rows = s["y"][s["places"].clamp_min(0).long()].float()
    out = torch.where(there, rows * s["weights"][..., None], torch.zeros_like(rows)).sum(1)
    if s["add"] is not None:
        out += s["add"].float()
    return out.to(torch.bfloat16)


# --- what a pass cannot do without -------------------------------------------------

def work(case):
    c = case
    if c["op"] == "project":
        rows, used = _rows(c), _adapters(c)
        n, m = sum(rows), len({a for a in used if a >= 0})
        adapted = sum(r for r, a in zip(rows, used) if a >= 0)
        size = 2 if c["dtype"] == "bf16" else 1
        return {"bytes": c["in"] * c["out"] * size + 2 * n * (c["in"] + c["out"]) + 2 * m * c["rank"] * (c["in"] + c["out"]),
                "flops": 2 * n * c["in"] * c["out"] + 2 * adapted * c["rank"] * (c["in"] + c["out"])}
    if c["op"] == "experts":
        loads = _loads(c)
        slots, used = sum(loads), sum(k > 0 for k in loads)
        size = 2 if c["dtype"] == "bf16" else 1
        wide = c["out"] * (2 if c["gated"] else 1)
        read = min(c["tokens"], slots) * 2 * c["in"] + 4 * slots if c["gathered"] else 2 * slots * c["in"]
        return {"bytes": used * wide * c["in"] * size + read + 2 * slots * c["out"], "flops": 2 * slots * c["in"] * wide}
    if c["op"] == "route":
        n, k = c["tokens"], c["top"]
        return {"bytes": n * c["experts"] * (2 if c["dtype"] == "bf16" else 4) + 16 * n * k + 4 * (c["experts"] + 1),
                "flops": 4 * n * c["experts"]}
    n, k = c["tokens"], c["top"]
    return {"bytes": 2 * (n - c["padded"]) * k * c["out"] + 8 * n * k + 2 * n * c["out"] * (2 if c["add"] else 1),
            "flops": 2 * (n - c["padded"]) * k * c["out"]}


# --- the definitions in 64 bits ----------------------------------------------------

def exact(case, seed):
    """From the definitions: rows by the adapter or expert that they meet, tokens one by one in the router."""
    c, s = case, prepare(case, seed)
    if c["op"] == "route":
        return _exact_route(c, s)
    if c["op"] == "combine":
        y = torch.cat([s["y"].double(), torch.zeros(1, c["out"], dtype=torch.float64, device="cuda")])
        out = torch.zeros(c["tokens"], c["out"], dtype=torch.float64, device="cuda")
        for j in range(c["top"]):
            out += y[s["places"][:, j].long()] * s["weights"][:, j, None].double()  # -1: the row of zeros behind the last
        return out if s["add"] is None else out + s["add"].double()
    out = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")

    def weight(g):
        return s["w"][g].double() * (1.0 if s["w_scale"] is None else s["w_scale"][g].double())

    if c["op"] == "project":
        x = s["x"].double()
        out = torch.nn.functional.linear(x, weight(0))
        at = torch.repeat_interleave(s["adapter"].long(), (s["start"][1:] - s["start"][:-1]).long())
        for m in range(c["adapters"]):
            mine = torch.nonzero(at == m)[:, 0]
            if len(mine):
                delta = s["b"][m].double() @ s["a"][m].double() if len(mine) > c["in"] else None
                inner = x[mine] @ delta.T if delta is not None else (x[mine] @ s["a"][m].double().T) @ s["b"][m].double().T
                out[mine] += s["scale"][m].double() * inner
        return out
    x = s["x"].double()
    of = torch.repeat_interleave(torch.arange(c["experts"], device="cuda"), (s["start"][1:] - s["start"][:-1]).long())
    for e in range(c["experts"]):
        slots = torch.nonzero(of == e)[:, 0]
        if not len(slots):
            continue
        v = x[slots if s["rows"] is None else s["rows"][slots].long()]
        z = torch.einsum("ik,ok->io", v, weight(e))
        out[slots] = z if not c["gated"] else torch.nn.functional.silu(z[:, :c["out"]]) * z[:, c["out"]:]
    return out


def _exact_route(c, s):
    scores = s["scores"].double().cpu().tolist()
    n, k, e = c["tokens"], c["top"], c["experts"]
    chosen, weights, members = [], [], [[] for _ in range(e)]
    for t, row in enumerate(scores):
        best = [i for i in sorted(range(e), key=lambda i: (-row[i], i))[:k] if row[i] > -math.inf]
        exps = [math.exp(row[i] - row[best[0]]) for i in best]
        total = sum(exps) if c["normalise"] else sum(math.exp(v - row[best[0]]) for v in row) if best else 1.0
        chosen.append(best + [-1] * (k - len(best)))
        weights.append([v / total for v in exps] + [0.0] * (k - len(best)))
        for j, i in enumerate(best):
            members[i].append((t, j))
    start, rows, places = [0], [], [[-1] * k for _ in range(n)]
    for pairs in members:
        for t, j in pairs:
            places[t][j] = len(rows)
            rows.append(t)
        start.append(len(rows))
    rows += [-1] * (n * k - len(rows))
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"chosen": whole(chosen), "weights": torch.tensor(weights, dtype=torch.float64, device="cuda"),
            "start": whole(start), "rows": whole(rows), "places": whole(places)}


if __name__ == "__main__":
    for a_case in listed() + [draw(random.Random(i)) for i in range(12)]:
        a_work = work(a_case)
        print("%-20s %10.3f MB %12.3f GFLOP" % (a_case.get("name", "drawn " + a_case["op"]), a_work["bytes"] / 1e6, a_work["flops"] / 1e9))
