"""The rollout operators whose speed is measured: a paged key/value cache that is
appended to (head norms, rotation, quantisation), read back, and attended over.

Between es_perturb and es_restore a program rolls the perturbed model out: it
feeds prompts, decodes single tokens, and feeds the turns in between. A case is one
call of one operator ("op") over a batch of sequences:

  append     es_cache_append: norms of the query and key heads, rotation, keys and
             values written to the cache in its own type
  read       es_cache_read: cached keys and values back as bf16 rows
  attention  es_attention: queries of the new tokens over the cached ones

Sequence lengths follow from the case alone; the seed gives values and page order.
"""
import math
import random

import torch

own = False

EPS = 1e-6


# --- the cases ---------------------------------------------------------------------

def listed():
    return [
        # one new token of one sequence, heads of the 4B-shaped set: latency of one call
        {"name": "append_token", "op": "append", "sequences": 1, "new_lo": 1, "new_hi": 1,
         "len_lo": 60, "len_hi": 60, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "dtype": "bf16", "rotary": 128},
        # a decode step of a population's rollouts over an FP8 cache, heads of the 27B-shaped set
        {"name": "append_step_e4m3", "op": "append", "sequences": 192, "new_lo": 1, "new_hi": 1,
         "len_lo": 3, "len_hi": 61, "q_heads": 40, "kv_heads": 8, "head_dim": 128, "page": 32,
         "dtype": "e4m3", "rotary": 128},
        # ragged prompts written to an FP8 cache, a quarter of each head rotated
        {"name": "append_prompts_e4m3", "op": "append", "sequences": 5, "new_lo": 1021,
         "new_hi": 5003, "len_lo": 5003, "len_hi": 5003, "q_heads": 32, "kv_heads": 8,
         "head_dim": 128, "page": 64, "dtype": "e4m3", "rotary": 32},
        # one long prompt, heads of the 27B-shaped set, bf16 cache
        {"name": "append_prompt", "op": "append", "sequences": 1, "new_lo": 16383, "new_hi": 16383,
         "len_lo": 16383, "len_hi": 16383, "q_heads": 40, "kv_heads": 8, "head_dim": 128,
         "page": 128, "dtype": "bf16", "rotary": 128},
        # the last turn of a few sequences read back for inspection
        {"name": "read_turn", "op": "read", "sequences": 3, "new_lo": 17, "new_hi": 90,
         "len_lo": 300, "len_hi": 900, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16,
         "dtype": "e4m3"},
        # whole sequences read back out of an FP8 cache
        {"name": "read_long_e4m3", "op": "read", "sequences": 6, "new_lo": 20000, "new_hi": 45000,
         "len_lo": 45000, "len_hi": 45000, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "dtype": "e4m3"},
        # one sequence's next token over a short cache: latency
        {"name": "decode_one", "op": "attention", "sequences": 1, "new_lo": 1, "new_hi": 1,
         "len_lo": 777, "len_hi": 777, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "dtype": "bf16", "cap": 0.0, "slopes": False, "window": 0, "mask": "none", "lse": False},
        # a decode step of many rollouts of very different lengths, heads of the 27B-shaped set
        {"name": "decode_step", "op": "attention", "sequences": 96, "new_lo": 1, "new_hi": 1,
         "len_lo": 200, "len_hi": 9000, "q_heads": 40, "kv_heads": 8, "head_dim": 128, "page": 64,
         "dtype": "bf16", "cap": 0.0, "slopes": False, "window": 0, "mask": "none", "lse": False},
        # few sequences with very long FP8 caches: the work is split along the cache
        {"name": "decode_long_e4m3", "op": "attention", "sequences": 3, "new_lo": 1, "new_hi": 1,
         "len_lo": 90000, "len_hi": 131071, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 128, "dtype": "e4m3", "cap": 0.0, "slopes": False, "window": 0, "mask": "none",
         "lse": True},
        # an agent's turn: some tokens of an observation each, over longer FP8 caches, capped scores
        {"name": "turn_capped_e4m3", "op": "attention", "sequences": 12, "new_lo": 9, "new_hi": 130,
         "len_lo": 2500, "len_hi": 8100, "q_heads": 40, "kv_heads": 8, "head_dim": 128, "page": 32,
         "dtype": "e4m3", "cap": 50.0, "slopes": False, "window": 0, "mask": "none", "lse": False},
        # packed documents with a bidirectional prefix each, a bias by distance, narrow heads
        {"name": "documents_biased", "op": "attention", "sequences": 3, "new_lo": 901, "new_hi": 4001,
         "len_lo": 4001, "len_hi": 4001, "q_heads": 16, "kv_heads": 4, "head_dim": 64, "page": 16,
         "dtype": "bf16", "cap": 0.0, "slopes": True, "window": 0, "mask": "documents", "lse": True},
        # a long prompt, heads of the 4B-shaped set
        {"name": "prompt", "op": "attention", "sequences": 1, "new_lo": 8191, "new_hi": 8191,
         "len_lo": 8191, "len_hi": 8191, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "dtype": "bf16", "cap": 0.0, "slopes": False, "window": 0, "mask": "none", "lse": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, 1 to some hundred sequences, new tokens from one to
    thousands, caches of up to 131,072 tokens, odd lengths among them, every page size,
    head layout and cache type."""
    op = rng.choice(["append", "append", "read", "attention", "attention", "attention"])
    heads = rng.choice([(32, 8, 128), (40, 8, 128), (16, 4, 64), (8, 8, 128), (24, 2, 64)])
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2],
         "page": rng.choice([16, 32, 64, 128]), "dtype": rng.choice(["bf16", "e4m3"])}
    if op == "attention":
        shape = rng.choice(["decode", "decode", "turn", "prompt"])
        if shape == "decode":
            c["sequences"] = _log_uniform(rng, 1, 256)
            new = 1
            longest = _log_uniform(rng, 30, min(131072, 900_000 // c["sequences"]))
        elif shape == "turn":
            c["sequences"] = _log_uniform(rng, 1, 24)
            new = _log_uniform(rng, 2, 200)
            longest = new + _log_uniform(rng, 30, 90_000 // c["sequences"])
        else:
            c["sequences"] = rng.choice([1, 1, 2, 3])
            new = _log_uniform(rng, 200, 8000 // c["sequences"])
            longest = new + rng.choice([0, 0, rng.randrange(1, 500)])
        c["new_lo"], c["new_hi"] = max(1, int(new * rng.uniform(0.3, 1.0))), new
        c["len_lo"] = max(new, int(longest * rng.uniform(0.2, 1.0)))
        c["len_hi"] = longest
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["slopes"] = rng.random() < 0.25
        c["window"] = rng.choice([0, 0, 0, _log_uniform(rng, 16, 4096)])
        c["mask"] = rng.choice(["none", "documents"]) if shape == "prompt" else "none"
        c["lse"] = rng.random() < 0.5
        return c
    c["sequences"] = _log_uniform(rng, 1, 192)
    new = _log_uniform(rng, 1, 16000 // c["sequences"])
    c["new_lo"], c["new_hi"] = max(1, int(new * rng.uniform(0.3, 1.0))), new
    c["len_lo"], c["len_hi"] = new, new + rng.randrange(0, 60)
    if op == "append":
        c["rotary"] = rng.choice([c["head_dim"], c["head_dim"], 32])
    return c


def _spread(lo, hi, n, step):
    """n whole numbers from lo to hi in an even, unordered spread."""
    return [hi - int((hi - lo + 1) * ((i * step) % 1.0)) if hi > lo else hi for i in range(n)]


def _lengths(c):
    """New tokens and cached tokens (the new ones included) of each sequence."""
    new = _spread(c["new_lo"], c["new_hi"], c["sequences"], 0.6180339887)
    total = _spread(c["len_lo"], c["len_hi"], c["sequences"], 0.7548776662)
    return new, [max(n, t) for n, t in zip(new, total)]


def _intervals(c):
    """(first, last) visible position of each new token where the case packs documents of
    about 700 tokens with a prefix of 37 that sees itself whole; else None."""
    if c["op"] != "attention" or c["mask"] != "documents":
        return None
    first, last = [], []
    for n, t in zip(*_lengths(c)):
        for p in range(t - n, t):
            begin = p // 701 * 701
            first.append(begin)
            last.append(min(t, max(p + 1, begin + 37)))
    return first, last


# --- inputs ------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)
    dev, bf = torch.device("cuda"), torch.bfloat16
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=g, device=dev, dtype=dtype)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    new, total = _lengths(c)
    page, hq, hkv, d = c["page"], c["q_heads"], c["kv_heads"], c["head_dim"]
    width = max(-(-t // page) for t in total)
    pages = sum(-(-t // page) for t in total)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.zeros(c["sequences"], width, dtype=torch.int32, device=dev)
    at = torch.arange(width, device=dev)[None, :] < ints([-(-t // page) for t in total])[:, None]
    table[at] = order
    s = {"case": c, "table": table, "seq_len": ints(total), "start": ints(start), "tokens": start[-1],
         "max_new": max(new), "max_len": max(total)}
    if c["op"] == "append":
        k = torch.zeros(pages, hkv, page, d, dtype=bf, device=dev)
        v = torch.zeros_like(k)
        # projections as they leave a layer: channels of different size, no row alike
        gain = torch.exp(0.5 * normal(hq + 2 * hkv, d))
        s["qkv"] = (normal(start[-1], hq + 2 * hkv, d) * gain).to(bf)
        s["q_weight"] = (1 + 0.2 * normal(d)).to(bf)
        s["k_weight"] = (1 + 0.2 * normal(d)).to(bf)
        half = c["rotary"] // 2
        angle = torch.arange(max(total), device=dev, dtype=torch.float64)[:, None] * \
            1e6 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        s["q_out"] = torch.empty(start[-1], hq, d, dtype=bf, device=dev)
    else:
        k = normal(pages, hkv, page, d, dtype=bf)
        v = normal(pages, hkv, page, d, dtype=bf) + 0.3 * normal(hkv, 1, d, dtype=bf)
    s["k"], s["v"] = k, v
    if c["dtype"] == "e4m3":
        s["k"], s["k_scale"] = _quantised(k.float())
        s["v"], s["v_scale"] = _quantised(v.float())
    if c["op"] == "read":
        s["k_out"] = torch.empty(start[-1], hkv, d, dtype=bf, device=dev)
        s["v_out"] = torch.empty_like(s["k_out"])
    if c["op"] == "attention":
        s["q"] = (1.5 * normal(start[-1], hq, d)).to(bf)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(start[-1], hq, device=dev) if c["lse"] else None
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device=dev) / hq) if c["slopes"] else None
        between = _intervals(c)
        s["first"], s["last"] = (None, None) if between is None else map(ints, between)
    if own:
        from paper_2608_17310_gb300 import rollout as ro
        s["cache"] = ro.es_cache_create(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"))
        s["batch"] = ro.Batch(table, s["seq_len"], s["start"], s["tokens"], s["max_new"])
        if c["op"] == "attention":
            s["workspace"] = torch.zeros(ro.es_attention_workspace(s["cache"], hq),
                                         dtype=torch.uint8, device=dev)
    return s


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        return _own(s, op)
    return _plain_append(s) if op == "append" else _plain_read(s) if op == "read" else _plain_attention(s)


def _own(s, op):
    from paper_2608_17310_gb300 import rollout as ro
    c = s["case"]
    if op == "append":
        ro.es_cache_append(s["cache"], s["batch"], s["qkv"], s["q_out"], s["q_weight"], s["k_weight"],
                           s["rope"], eps=EPS)
        return _appended(s, s["q_out"])
    if op == "read":
        ro.es_cache_read(s["cache"], s["batch"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    ro.es_attention(s["cache"], s["batch"], s["q"], s["out"], s["workspace"],
                    scale=c["head_dim"] ** -0.5, lse=s["lse"], softcap=c["cap"], slopes=s["slopes"],
                    window=c["window"], first=s["first"], last=s["last"])
    return {"out": s["out"], "lse": s["lse"]}


def _appended(s, q):
    """The queries and the whole cache; codes as the E4M3 numbers they are, with their scales."""
    out = {"q": q, "k": s["k"], "v": s["v"]}
    if "k_scale" in s:
        out["k_scale"], out["v_scale"] = s["k_scale"], s["v_scale"]
    return out


# --- the plain forms ---------------------------------------------------------------

def _quantised(x):
    """E4M3 numbers and one scale for each last-axis vector: max|x| / 448."""
    scale = (x.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
    return (x / scale[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn), scale


def _places(s):
    """Sequence and position of each new token, and the page and slot that hold it."""
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["start"][1:].long(), t, right=True)
    pos = s["seq_len"][seq].long() - s["start"][seq + 1].long() + t
    page = s["case"]["page"]
    return seq, pos, s["table"][seq, pos // page].long(), pos % page


def _plain_append(s):
    c = s["case"]
    hq, hkv = c["q_heads"], c["kv_heads"]
    _, pos, page, slot = _places(s)
    x = s["qkv"].float()
    turn = s["rope"][pos][:, None]

    def normed(x, w):
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        half = c["rotary"] // 2
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        cos, sin = turn[..., 0], turn[..., 1]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)

    q = normed(x[:, :hq], s["q_weight"]).to(torch.bfloat16)
    k, v = normed(x[:, hq:hq + hkv], s["k_weight"]), x[:, hq + hkv:]
    if c["dtype"] == "e4m3":
        k, ks = _quantised(k)
        v, vs = _quantised(v)
        s["k"].view(torch.uint8)[page, :, slot] = k.view(torch.uint8)
        s["v"].view(torch.uint8)[page, :, slot] = v.view(torch.uint8)
        s["k_scale"][page, :, slot] = ks
        s["v_scale"][page, :, slot] = vs
    else:
        s["k"][page, :, slot] = k.to(torch.bfloat16)
        s["v"][page, :, slot] = v.to(torch.bfloat16)
    return _appended(s, q)


def _plain_read(s):
    _, _, page, slot = _places(s)

    def rows(x, scale):
        if scale is None:
            return x[page, :, slot]
        x = x.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
        return (x * scale[page, :, slot][..., None]).to(torch.bfloat16)

    return {"k": rows(s["k"], s.get("k_scale")), "v": rows(s["v"], s.get("v_scale"))}


def _dense(s, x, scale):
    """Cached vectors in sequence order, 32 bits: [sequences, kv_heads, max_len, head_dim]."""
    c, table = s["case"], s["table"].long()
    y = x.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() if scale is not None else x[table].float()
    if scale is not None:
        y = y * scale[table][..., None]
    return y.transpose(1, 2).reshape(c["sequences"], c["kv_heads"], -1, c["head_dim"])[:, :, :s["max_len"]]


def _plain_attention(s):
    c = s["case"]
    b, hkv, d, m = c["sequences"], c["kv_heads"], c["head_dim"], s["max_new"]
    group = c["q_heads"] // hkv
    dev = s["q"].device
    start, length = s["start"].long(), s["seq_len"].long()
    count = start[1:] - start[:-1]
    i = torch.arange(m, device=dev)
    token = (start[:-1, None] + i).clamp_max(s["tokens"] - 1)              # [b, m], padded
    pos = (length - count)[:, None] + i
    q = s["q"][token].float().view(b, m, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * m, d)
    k, v = _dense(s, s["k"], s.get("k_scale")), _dense(s, s["v"], s.get("v_scale"))
    x = (q @ k.transpose(2, 3)).mul_(d ** -0.5)
    if c["cap"]:
        x = torch.tanh(x.div_(c["cap"])).mul_(c["cap"])
    x = x.view(b, hkv, group, m, s["max_len"])
    j = torch.arange(s["max_len"], device=dev)
    if s["slopes"] is not None:
        away = (pos[:, :, None] - j).abs().float()                         # [b, m, len]
        x = x - s["slopes"].view(1, hkv, group, 1, 1) * away[:, None, None]
    first = s["first"][token] if s["first"] is not None else torch.zeros_like(pos)
    last = s["last"][token] if s["last"] is not None else pos + 1
    if c["window"]:
        first = torch.maximum(first, pos - c["window"] + 1)
    last = torch.minimum(last, length[:, None])
    seen = (j >= first[:, :, None]) & (j < last[:, :, None])
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x.view(b, hkv, group * m, -1) @ v).view(b, hkv, group, m, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = (top + total.log())[..., 0]
    t = torch.arange(s["tokens"], device=dev)
    seq = torch.searchsorted(start[1:], t, right=True)
    row = t - start[seq]
    out = out[seq, :, :, row].reshape(s["tokens"], hkv * group, d).to(torch.bfloat16)
    return {"out": out, "lse": lse[seq, :, :, row].reshape(s["tokens"], hkv * group) if s["lse"] is not None else None}


# --- what a pass cannot do without -------------------------------------------------

def _vector_bytes(c):
    """Bytes of one cached vector of one head."""
    return c["head_dim"] + 4 if c["dtype"] == "e4m3" else 2 * c["head_dim"]


def work(case):
    c = case
    new, total = _lengths(c)
    t, hq, hkv, d = sum(new), c["q_heads"], c["kv_heads"], c["head_dim"]
    cached = 2 * hkv * _vector_bytes(c)
    if c["op"] == "append":
        rows = len({p for n, l in zip(new, total) for p in range(l - n, l)})
        return {"bytes": t * ((hq + 2 * hkv) * d * 2 + hq * d * 2 + cached) + rows * c["rotary"] * 4,
                "flops": t * (hq + hkv) * (4 * d + 3 * c["rotary"])}
    if c["op"] == "read":
        return {"bytes": t * (cached + 2 * hkv * d * 2), "flops": 0}
    between, pairs, seen, at = _intervals(c), 0, 0, 0
    for n, l in zip(new, total):
        lo_all, hi_all = l, 0
        for p in range(l - n, l):
            lo, hi = (0, p + 1) if between is None else (between[0][at], between[1][at])
            if c["window"]:
                lo = max(lo, p - c["window"] + 1)
            pairs += max(0, hi - lo)
            lo_all, hi_all, at = min(lo_all, lo), max(hi_all, hi), at + 1
        seen += max(0, hi_all - lo_all)
    return {"bytes": t * hq * (4 * d + (4 if c["lse"] else 0)) + seen * cached, "flops": 4 * d * hq * pairs}


# --- the definitions in 64 bits ----------------------------------------------------

def exact(case, seed):
    """Token by token and head by head from the definitions; cached codes are given as the
    unrounded numbers that they stand nearest to."""
    c, s = case, prepare(case, seed)
    new, total = _lengths(c)
    table = s["table"].cpu().tolist()
    hq, hkv, d, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    bounds = s["start"].cpu().tolist()
    spots = [(b, p) for b, (n, l) in enumerate(zip(new, total)) for p in range(l - n, l)]
    if c["op"] == "append":
        x = s["qkv"].double()
        pg = torch.tensor([table[b][p // page] for b, p in spots], device="cuda")
        sl = torch.tensor([p % page for b, p in spots], device="cuda")
        z = torch.view_as_complex(s["rope"].double())[torch.tensor([p for b, p in spots], device="cuda")]
        half = c["rotary"] // 2

        def head(x, w):
            y = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + EPS) * w.double()
            w = torch.complex(y[..., :half], y[..., half:2 * half]) * z[:, None]
            y[..., :half], y[..., half:2 * half] = w.real, w.imag
            return y

        k, v = head(x[:, hq:hq + hkv], s["k_weight"]), x[:, hq + hkv:]
        out = {"q": head(x[:, :hq], s["q_weight"])}
        for name, y in (("k", k), ("v", v)):
            whole = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
            if c["dtype"] == "e4m3":
                scale = s[name + "_scale"].double()
                mine = y.abs().amax(-1) / 448
                scale[pg, :, sl] = mine
                out[name + "_scale"] = scale
                y = y / mine[..., None]
            whole[pg, :, sl] = y
            out[name] = whole
        return out

    def sequence(b, name, lo, hi):
        """Positions lo .. hi - 1 of sequence b: [hi - lo, kv_heads, head_dim]."""
        ids = torch.tensor(table[b][lo // page:-(-hi // page)], device="cuda")
        y = s[name][ids].double() if c["dtype"] == "bf16" else s[name].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double()
        if c["dtype"] == "e4m3":
            y = y * s[name + "_scale"][ids].double()[..., None]
        return y.transpose(1, 2).reshape(-1, hkv, d)[lo % page:lo % page + hi - lo]

    if c["op"] == "read":
        return {n: torch.cat([sequence(b, n, l - k, l) for b, (k, l) in enumerate(zip(new, total))]) for n in ("k", "v")}
    out = torch.zeros(s["tokens"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["tokens"], hq, dtype=torch.float64, device="cuda")
    for b, (n, l) in enumerate(zip(new, total)):
        at = slice(bounds[b], bounds[b + 1])
        p = torch.arange(l - n, l, device="cuda")[:, None]
        j = torch.arange(l, device="cuda")[None]
        hide = (j > p) if s["last"] is None else (j >= s["last"][at, None])
        if s["first"] is not None:
            hide = hide | (j < s["first"][at, None])
        if c["window"]:
            hide = hide | (p - j >= c["window"])
        ks, vs = sequence(b, "k", 0, l), sequence(b, "v", 0, l)
        for h in range(hq):
            g = h * hkv // hq
            x = s["q"][at, h].double() @ ks[:, g].T / math.sqrt(d)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (p - j).abs()
            x = x.masked_fill(hide, -math.inf)
            lse[at, h] = torch.logsumexp(x, -1)
            out[at, h] = torch.softmax(x, -1) @ vs[:, g]
    return {"out": out, "lse": lse if c["lse"] else None}


if __name__ == "__main__":
    for a_case in listed() + [draw(random.Random(i)) for i in range(6)]:
        a_work = work(a_case)
        print("%-24s %10.3f MB %12.3f GFLOP" % (a_case.get("name", "drawn"), a_work["bytes"] / 1e6, a_work["flops"] / 1e9))
