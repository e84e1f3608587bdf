"""The rollout operators against their definitions in 64 bits: a paged cache appended to,
read back and attended over. Tolerances and their reasons: rollout_reference.py."""
import math

import numpy as np
import pytest
import torch

import rollout_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ro(es):
    from paper_2608_17310_gb300 import rollout
    return rollout


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Setup:
    """A cache of random contents with shuffled pages, and the batch of its new tokens."""

    def __init__(self, ro, seq_len, new, kv_heads=2, d=128, page=16, dtype="bf16", seed=0, spare=3,
                 interleave=False, gap=0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.ro, self.seq_len, self.new = g, ro, list(seq_len), list(new)
        self.page, self.kv_heads, self.d, self.dtype = page, kv_heads, d, dtype
        need = [max(1, -(-max(l, n) // page)) for l, n in zip(seq_len, new)]
        count = sum(need) + spare
        order = torch.randperm(count, generator=g).tolist()
        width = max(need) + 1
        self.pages, k = [], 0
        for n in need:
            self.pages.append(order[k:k + n] + [-1] * (width - n))
            k += n
        value = torch.randn(count, 2, kv_heads, page, d, generator=g)
        if dtype == "bf16":
            store = value.bfloat16()
            self.scale = None
        else:
            self.scale = (value.abs().amax(-1) / 448).contiguous()
            store = (value / self.scale[..., None]).to(torch.float8_e4m3fn)
        # k and v of a page beside one another (page_stride over a page), or apart
        if interleave:
            both = store.view(torch.uint8).cuda().view(store.dtype) if dtype != "bf16" else store.cuda()
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k = store[:, 0].contiguous().view(torch.uint8).cuda().view(store.dtype)
            self.v = store[:, 1].contiguous().view(torch.uint8).cuda().view(store.dtype)
        self.ks = self.vs = None
        if self.scale is not None:
            both = self.scale.cuda()
            self.ks, self.vs = (both[:, 0], both[:, 1]) if interleave else \
                (both[:, 0].contiguous(), both[:, 1].contiguous())
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
        self.tokens = self.start[-1]
        self.remake()

    def remake(self):
        ro = self.ro
        self.cache = ro.es_cache_create(self.k, self.v, self.ks, self.vs)
        self.batch = ro.Batch(i32(self.pages), i32(self.seq_len), i32(self.start), self.tokens,
                              max(1, max(self.new)))

    def dense(self):
        """Every sequence's vectors in float64, [len, kv_heads, d] each for k and v."""
        out = []
        for x, s in ((self.k, self.ks), (self.v, self.vs)):
            y = R.e4m3(x.contiguous().cpu()) * s.cpu().double()[..., None] if s is not None else x.cpu().double()
            seqs = []
            for b, l in enumerate(self.seq_len):
                rows = [y[max(0, self.pages[b][p // self.page]), :, p % self.page] for p in range(l)]
                seqs.append(torch.stack(rows) if rows else torch.zeros(0, self.kv_heads, self.d, dtype=torch.float64))
            out.append(seqs)
        return out

    def absent(self):
        return [{p for p in range(l) if self.pages[b][p // self.page] < 0} for b, l in enumerate(self.seq_len)]


def attend(s, q_heads, q=None, stream=None, **kw):
    if q is None:
        q = (1.5 * torch.randn(s.tokens, q_heads, s.d, generator=s.g)).bfloat16().cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full((s.tokens, q_heads), 7.0, device="cuda")
    ws = torch.zeros(s.ro.es_attention_workspace(s.cache, q_heads), dtype=torch.uint8, device="cuda")
    args = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in kw.items()}
    for _ in range(2):  # the second call finds the workspace as the first left it
        out.fill_(7.0)
        lse.fill_(7.0)
        s.ro.es_attention(s.cache, s.batch, q, out, ws, scale=s.d ** -0.5, lse=lse, stream=stream, **args)
        first = out.clone() if _ == 0 else first
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), out.view(torch.int16)), "two calls differ"
    assert not ws[:4352].any(), "counters or the flag of a given-up wait are left"
    return q, out, lse


def assert_attention(s, q, out, lse, absent=None, **kw):
    k, v = s.dense()
    kw = {k: (v.cpu() if torch.is_tensor(v) else v) for k, v in kw.items()}
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, s.d ** -0.5, absent=absent, **kw)
    err = (out.cpu().double() - want).abs()
    bound = (2.0 ** -7 + 2.0 ** -12) * size
    assert (err <= bound).all(), f"off by {(err / bound.clamp_min(1e-30)).max():.3g} of the bound"
    hit = want_lse > -math.inf
    assert torch.equal(hit, lse.cpu() > -math.inf)
    assert ((lse.cpu().double() - want_lse)[hit].abs() <= 1e-4).all()


def check(s, q_heads, absent=None, **kw):
    q, out, lse = attend(s, q_heads, **kw)
    assert_attention(s, q, out, lse, absent, **kw)


DTYPES = ["bf16", "e4m3"]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,kv_heads", [(1, 3), (4, 2), (5, 1), (16, 1)])
def test_decode_matches_definition(ro, dtype, d, group, kv_heads):
    lens = [1, 2, 63, 64, 65, 128, 130, 257, 0, 400]
    s = Setup(ro, lens, [1 if l else 0 for l in lens], kv_heads, d, 32, dtype)
    check(s, group * kv_heads)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode_of_a_long_cache(ro, dtype, page):
    # one sequence over many blocks, whose parts are joined
    s = Setup(ro, [5003], [1], 2, 128, page, dtype, seed=page)
    check(s, 8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[2, 3, 1], [17, 0, 5], [33, 130, 64], [129, 1, 40]])
def test_several_new_tokens(ro, dtype, d, new):
    lens = [n + extra if n else 9 for n, extra in zip(new, (0, 61, 200))]
    check(Setup(ro, lens, new, 2, d, 16, dtype, seed=sum(new)), 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 3, 33]])
@pytest.mark.parametrize("kw", [{"softcap": 5.0}, {"slopes": True}, {"window": 7}, {"window": 100},
                                {"softcap": 30.0, "slopes": True, "window": 50}],
                         ids=["cap", "slopes", "window7", "window100", "all"])
def test_scores_and_window(ro, dtype, new, kw):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = 2.0 ** -torch.arange(1, 9, dtype=torch.float32)
    check(Setup(ro, [200, 90, 333], new, 2, 128, 32, dtype, seed=5), 8, **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [50, 1, 129, 66]])
def test_intervals_and_empty_rows(ro, dtype, new):
    # random intervals, among them empty, reversed, negative and past the end
    s = Setup(ro, [150, 1, 260, 66], new, 2, 128, 16, dtype, seed=9)
    rng = np.random.default_rng(3)
    first = torch.tensor(rng.integers(-20, 270, s.tokens), dtype=torch.int32)
    last = torch.tensor(rng.integers(-20, 400, s.tokens), dtype=torch.int32)
    first[0], last[0] = 40, 40
    check(s, 4, first=first, last=last)
    check(s, 4, first=first)
    check(s, 4, last=last, window=30)
    first[:] = 1000  # nothing is seen at all
    q, out, lse = attend(s, 4, first=first)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [3, 2], [90, 64]])
def test_what_is_not_seen_does_not_reach(ro, dtype, new):
    # NaN and infinities in every slot that holds no token, before a window, and in the
    # keys and values of tokens that only later tokens see
    s = Setup(ro, [150, 75], new, 2, 128, 32, dtype, seed=4)
    used = {(s.pages[b][p // s.page], p % s.page): (b, p) for b, l in enumerate(s.seq_len) for p in range(l)}
    # the last token of each sequence poisons itself alone (causal), its first ones are before `first`
    poisoned_last = max(new) > 1
    bad = [float("nan"), float("inf"), -float("inf")]

    def poison(page, slot, n):
        if dtype == "bf16":
            s.k[page, :, slot] = bad[n % 3]
            s.v[page, :, slot, n % s.d] = bad[n % 3]
        else:
            s.k.view(torch.uint8)[page, :, slot] = 0x7F
            s.v.view(torch.uint8)[page, :, slot, n % s.d] = 0xFF
            if n % 2:
                s.vs[page, :, slot] = bad[n % 3]
                s.ks[page, :, slot] = bad[n % 3]

    clean = s.dense()
    n = 0
    for page in range(s.k.shape[0]):
        for slot in range(s.page):
            b, p = used.get((page, slot), (None, None))
            last_token = poisoned_last and b is not None and p == s.seq_len[b] - 1
            if b is None or p < 11 or last_token:
                poison(page, slot, n)
                n += 1
    first = torch.full((s.tokens,), 11, dtype=torch.int32)
    q, out, lse = attend(s, 8, first=first)
    s.dense = lambda: clean
    ends = [e - 1 for e in s.start[1:]]
    rows = [t for t in range(s.tokens) if not (poisoned_last and t in ends)]
    k, v = clean
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, s.d ** -0.5, first=first)
    err = (out.cpu().double() - want).abs()[rows]
    assert (err <= ((2.0 ** -7 + 2.0 ** -12) * size)[rows]).all()
    assert ((lse.cpu().double() - want_lse)[rows].abs() <= 1e-4).all()
    if poisoned_last:
        assert torch.isnan(out[ends].float()).all()


@pytest.mark.parametrize("new", [[1, 1], [65, 80]])
def test_a_poisoned_value_reaches_those_that_see_it(ro, new):
    s = Setup(ro, [150, 90], new, 2, 128, 32, "bf16", seed=6)
    at = s.seq_len[0] - new[0]  # the first new token's value: all new tokens see it
    s.v[s.pages[0][at // 32], 1, at % 32, 5] = float("inf")
    q, out, lse = attend(s, 8)
    k, v = s.dense()
    seen = out[:new[0], 4:, 5].float()
    assert (seen == math.inf).all()
    other = out.clone()
    other[:new[0], 4:, 5] = 0
    assert torch.isfinite(other.float()).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 70, 3]])
def test_pages_that_do_not_exist_hold_no_tokens(ro, dtype, new):
    s = Setup(ro, [100, 200, 60], new, 2, 128, 16, dtype, seed=8)
    s.pages[0][2] = -1
    s.pages[1][0] = 10 ** 9
    s.pages[1][12] = -(2 ** 31)
    s.pages[2][:] = [-1] * len(s.pages[2])
    for row in s.pages:
        for i, p in enumerate(row):
            row[i] = p if p < s.k.shape[0] else -7 if p != 10 ** 9 else p
    s.batch = ro.Batch(i32(s.pages), i32(s.seq_len), i32(s.start), s.tokens, max(new))
    for row in s.pages:
        row[:] = [p if 0 <= p < s.k.shape[0] else -1 for p in row]
    check(s, 4, absent=s.absent())


@pytest.mark.parametrize("dtype", DTYPES)
def test_lengths_and_starts_out_of_range(ro, dtype):
    # a length over the table counts as the table's reach, a negative one as none, and a
    # sequence shorter than its new tokens has no place for the first of them
    s = Setup(ro, [64, 10, 5], [1, 3, 4], 2, 128, 16, dtype)
    s.seq_len = [len(s.pages[0]) * 16, 10, 2]
    s.batch = ro.Batch(i32(s.pages), i32([10 ** 9, 10, 2]), i32(s.start), s.tokens, 4)
    check(s, 4, absent=s.absent())
    s.batch = ro.Batch(i32(s.pages), i32([-5, -1, -2 ** 31]), i32(s.start), s.tokens, 4)
    q, out, lse = attend(s, 4)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [5, 77]])
def test_strides(ro, dtype, new):
    s = Setup(ro, [99, 180], new, 2, 64, 16, dtype, interleave=True)
    wide = torch.randn(s.tokens, 8 * 64 + 24, generator=s.g).bfloat16().cuda()
    q = wide[:, 8:8 + 512].view(s.tokens, 8, 64) if s.tokens == 1 else wide[:, 8:520].unflatten(1, (8, 64))
    out_wide = torch.full((s.tokens, 600), 3.0, dtype=torch.bfloat16, device="cuda")
    out = out_wide[:, 16:528].unflatten(1, (8, 64))
    lse = torch.empty(s.tokens, 8, device="cuda")
    ws = torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")
    ro.es_attention(s.cache, s.batch, q, out, ws, scale=0.125, lse=lse)
    assert_attention(s, q, out, lse)
    assert (out_wide[:, :16] == 3).all() and (out_wide[:, 528:] == 3).all()


def test_one_new_token_each_without_start(ro):
    s = Setup(ro, [30, 77, 5], [1, 1, 1], 2, 128, 16, "bf16")
    q, out, lse = attend(s, 4)
    s.batch = ro.Batch(i32(s.pages), i32(s.seq_len))
    _, out2, lse2 = attend(s, 4, q=q)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_large_scores_and_lengths_of_very_different_size(ro):
    # scores of +-60 and more: the running maximum moves through the tiles
    s = Setup(ro, [3000, 10, 700], [1, 1, 40], 1, 128, 64, "bf16", seed=2)
    q = (12 * torch.randn(s.tokens, 4, 128, generator=s.g)).bfloat16().cuda()
    q, out, lse = attend(s, 4, q=q)
    k, v = s.dense()
    want, size, want_lse = R.attention(q.cpu(), k, v, s.seq_len, s.new, s.d ** -0.5)
    assert ((out.cpu().double() - want).abs() <= (2.0 ** -7 + 2.0 ** -11) * size).all()
    assert ((lse.cpu().double() - want_lse).abs() <= 2e-4).all()


def test_offsets_past_32_bits(ro):
    # pages that lie over 2^32 elements into the cache: the buffer is never filled as a whole
    free, _ = torch.cuda.mem_get_info()
    pages = 2 ** 32 // (2 * 64 * 128) + 40
    if free < 3 * pages * 2 * 64 * 128 * 2:
        pytest.fail("not enough free device memory")
    k = torch.empty(pages, 2, 64, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache = ro.es_cache_create(k, v)
    table = [[pages - 1 - i for i in range(4)], [0, pages - 9, 1, pages - 8]]
    for new in ([200, 190], [1, 1]):
        batch = ro.Batch(i32(table), i32([200, 190]), i32([0, new[0], sum(new)]), sum(new), max(new))
        g = torch.Generator().manual_seed(1)
        if new[0] > 1:
            qkv = torch.randn(sum(new), 8, 128, generator=g).bfloat16().cuda()
            q = torch.empty(sum(new), 4, 128, dtype=torch.bfloat16, device="cuda")
            ro.es_cache_append(cache, batch, qkv, q)
            k_out, v_out = torch.empty(2, sum(new), 2, 128, dtype=torch.bfloat16, device="cuda")
            ro.es_cache_read(cache, batch, k_out, v_out)
            assert torch.equal(q, qkv[:, :4]) and torch.equal(k_out, qkv[:, 4:6]) and torch.equal(v_out, qkv[:, 6:])
        x = torch.randn(sum(new), 4, 128, generator=g).bfloat16().cuda()
        out = torch.empty_like(x)
        ws = torch.zeros(ro.es_attention_workspace(cache, 4), dtype=torch.uint8, device="cuda")
        ro.es_attention(cache, batch, x, out, ws, scale=0.1)
        ks, vs = qkv[:, 4:6].cpu(), qkv[:, 6:].cpu()
        want, size, _ = R.attention(x.cpu(), [ks[:200], ks[200:]], [vs[:200], vs[200:]], [200, 190], new, 0.1)
        assert ((out.cpu().double() - want).abs() <= (2.0 ** -7 + 2.0 ** -12) * size).all()


def test_two_streams_with_a_workspace_each(ro):
    torch.cuda.synchronize()
    sets = [Setup(ro, [900, 300], n, 2, 128, 32, "bf16", seed=i) for i, n in enumerate(([1, 1], [80, 9]))]
    one = [attend(s, 8) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for s, st, (q, _, _) in zip(sets, streams, one):
        with torch.cuda.stream(st):
            ws = torch.zeros(ro.es_attention_workspace(s.cache, 8), dtype=torch.uint8, device="cuda")
            outs = [torch.empty_like(q) for _ in range(20)]
            got.append((outs, ws))
    torch.cuda.synchronize()
    for i in range(20):
        for s, st, (q, _, _), (outs, ws) in zip(sets, streams, one, got):
            ro.es_attention(s.cache, s.batch, q, outs[i], ws, scale=s.d ** -0.5, stream=st)
    torch.cuda.synchronize()
    for (_, out, _), (outs, _) in zip(one, got):
        assert all(torch.equal(out, o) for o in outs)


def test_graph_reads_lengths_when_it_runs(ro):
    s = Setup(ro, [40, 40], [1, 1], 2, 128, 16, "e4m3")
    q, out, lse = attend(s, 4)
    lens = i32([40, 40])
    s.batch = ro.Batch(i32(s.pages), lens, i32(s.start), 2, 1)
    ws = torch.zeros(ro.es_attention_workspace(s.cache, 4), dtype=torch.uint8, device="cuda")
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ro.es_attention(s.cache, s.batch, q, got, ws, scale=s.d ** -0.5, lse=got_lse)
    for new_lens in ([40, 40], [17, 33], [1, 40]):
        lens.copy_(i32(new_lens))
        graph.replay()
        torch.cuda.synchronize()
        s.seq_len = new_lens
        assert_attention(s, q, got, got_lse)


# --- append and read ------------------------------------------------------------------

def append_case(ro, dtype, d, rotary, interleaved=False, weights=True, positions=None, new=(5, 0, 19, 1),
                lens=(5, 3, 40, 33), q_heads=6, kv_heads=2, eps=1e-6, wide=0, x=None, in_place=False, page=16):
    s = Setup(ro, lens, new, kv_heads, d, page, dtype, interleave=wide > 0)
    heads = q_heads + 2 * kv_heads
    if x is None:
        x = torch.randn(s.tokens, heads * d, generator=s.g) * torch.exp(torch.randn(heads * d, generator=s.g))
    store = torch.zeros(s.tokens, heads * d + wide, dtype=torch.bfloat16)
    store[:, :heads * d] = x.bfloat16()
    store = store.cuda()
    qkv = store[:, :heads * d].unflatten(1, (heads, d))
    host = qkv.cpu().clone()
    qw = (1 + 0.3 * torch.randn(d, generator=s.g)).bfloat16().cuda() if weights else None
    kw = (1 + 0.3 * torch.randn(d, generator=s.g)).bfloat16().cuda() if weights else None
    rope = None
    if rotary:
        ang = torch.rand(50, rotary // 2, generator=s.g, dtype=torch.float64) * 100
        rope = torch.stack([ang.cos(), ang.sin()], -1).float().cuda()
    q = qkv[:, :q_heads] if in_place else torch.full((s.tokens, q_heads, d), 9.0, dtype=torch.bfloat16, device="cuda")
    pos = None if positions is None else i32(positions)
    before = [t.clone() for t in (s.k.view(torch.uint8), s.v.view(torch.uint8))] if dtype == "e4m3" else [s.k.clone(), s.v.clone()]
    ro.es_cache_append(s.cache, s.batch, qkv, q, qw, kw, rope, eps=eps, positions=pos, interleaved=interleaved)
    torch.cuda.synchronize()
    spots = R.places(s.pages, s.page, s.seq_len, s.new)
    turns = positions if positions is not None else [sp and sp[1] for sp in spots]
    wq, wk, wv = R.append(host, q_heads, kv_heads, d, qw.cpu() if weights else None, kw.cpu() if weights else None,
                          eps, None if rope is None else rope.cpu(), turns, interleaved)
    return s, q, (wq, wk, wv), spots, before


def assert_appended(s, q, want, spots, before):
    wq, wk, wv = want

    def near(got, want):
        size = want.abs().amax(-1, keepdim=True)
        nan = torch.isnan(want)
        assert torch.equal(nan, torch.isnan(got))
        ok = (got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size
        assert (ok | nan | (got == want)).all()  # an infinity is itself

    near(q.cpu().double(), wq)
    touched = set()
    for t, sp in enumerate(spots):
        if sp is None or sp[2] < 0:
            continue
        _, _, page, slot = sp
        touched.add((page, slot))
        for store, scale, w in ((s.k, s.ks, wk[t]), (s.v, s.vs, wv[t])):
            if scale is None:
                near(store[page, :, slot].cpu().double(), w)
            else:
                got = R.e4m3(store.view(torch.uint8)[page, :, slot].cpu())
                sc = scale[page, :, slot].cpu().double()
                fin = torch.where(torch.isfinite(w), w.abs(), torch.zeros_like(w)).amax(-1) / 448
                fin = fin.clamp_min(2.0 ** -126)
                assert ((sc - fin).abs() <= 2.0 ** -20 * fin).all()
                y = (w / fin[:, None]).clamp(-448, 448)
                nan = torch.isnan(w)
                assert torch.equal(nan, torch.isnan(got))
                assert (((got - y).abs() <= R.half_step(y) + 448 * 2.0 ** -15) | nan).all()
    for store, old in zip((s.k, s.v), before):
        now = store.view(torch.uint8) if s.dtype == "e4m3" else store
        for page in range(store.shape[0]):
            for slot in range(s.page):
                if (page, slot) not in touched:
                    assert torch.equal(now[page, :, slot], old[page, :, slot])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,rotary,interleaved", [(128, 128, False), (128, 32, False), (128, 48, True), (128, 0, False),
                                                  (64, 64, False), (64, 16, True), (64, 32, False), (128, 128, True)])
def test_append_matches_definition(ro, dtype, d, rotary, interleaved):
    assert_appended(*append_case(ro, dtype, d, rotary, interleaved))


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_options(ro, dtype):
    assert_appended(*append_case(ro, dtype, 128, 64, weights=False))
    assert_appended(*append_case(ro, dtype, 128, 64, positions=[(7 * i) % 50 for i in range(25)]))
    assert_appended(*append_case(ro, dtype, 64, 64, wide=40, page=128))
    assert_appended(*append_case(ro, dtype, 128, 128, in_place=True))
    assert_appended(*append_case(ro, dtype, 128, 128, eps=0.5, q_heads=16, kv_heads=1))


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_outside_the_tables(ro, dtype):
    # positions without a rope row: NaN queries and keys; more new tokens than the sequence
    # is long: no place for the first
    assert_appended(*append_case(ro, dtype, 128, 128, positions=[49, 50, -1, 2 ** 31 - 1, 0] * 5))
    s, q, want, spots, before = append_case(ro, dtype, 128, 128, new=(4, 3), lens=(2, 3))
    assert spots[0] is None and spots[1] is None
    assert_appended(s, q, want, spots, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_of_unusual_values(ro, dtype):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(25, 10 * 128, generator=g)
    x[0] = 0
    x[1, 128:256] = 1e-38          # the norm's eps decides
    x[2, 1024:] *= 1e30
    x[3, 9 * 128 + 3] = float("inf")
    x[4, 8 * 128 + 5] = float("nan")
    x[5, 8 * 128:] = 1e-39         # below the smallest scale times a code
    x[6, 8 * 128:] *= 1e-36
    assert_appended(*append_case(ro, dtype, 128, 0, x=x, eps=1e-6))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_read_returns_what_the_cache_holds(ro, dtype, d):
    s = Setup(ro, [70, 5, 33, 1], [70, 0, 20, 1], 3, d, 16, dtype)
    s.pages[2][1] = -1
    s.remake()
    k, v = (torch.full((s.tokens, 3, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ro.es_cache_read(s.cache, s.batch, k, v)
    only = torch.empty_like(v)
    ro.es_cache_read(s.cache, s.batch, None, only)
    assert torch.equal(only, v)
    dk, dv = s.dense()
    for t, (b, p, page, slot) in enumerate(R.places(s.pages, 16, s.seq_len, s.new)):
        for got, want in ((k, dk), (v, dv)):
            w = want[b][p] if page >= 0 else torch.zeros(3, d, dtype=torch.float64)
            assert ((got[t].cpu().double() - w).abs() <= (2.0 ** -8 * w.abs() if dtype == "e4m3" else 0)).all()


# --- refusals -----------------------------------------------------------------------------

def status(es, call, *args, **kw):
    with pytest.raises(es.EsError) as e:
        call(*args, **kw)
    return e.value.status


def test_refusals(es, ro):
    s = Setup(ro, [20, 20], [2, 3], 2, 128, 16, "bf16")
    q = torch.zeros(5, 4, 128, dtype=torch.bfloat16, device="cuda")
    out, ws = torch.zeros_like(q), torch.zeros(ro.es_attention_workspace(s.cache, 4), dtype=torch.uint8, device="cuda")
    good = dict(scale=1.0)
    ro.es_attention(s.cache, s.batch, q, out, ws, **good)
    bad = es.ES_ERR_INVALID_ARG
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws, scale=float("nan")) == es.ES_ERR_NONFINITE
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws, scale=1.0, softcap=float("inf")) == es.ES_ERR_NONFINITE
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws, scale=1.0, softcap=-1.0) == bad
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws, scale=1.0, window=-1) == bad
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws, scale=1.0, softcap=1e-35) == bad
    assert status(es, ro.es_attention, s.cache, s.batch, q, out, ws[:-1], scale=1.0) == bad
    q3 = torch.zeros(5, 3, 128, dtype=torch.bfloat16, device="cuda")  # 3 query heads of 2 key heads
    assert status(es, ro.es_attention, s.cache, s.batch, q3, torch.zeros_like(q3), ws, **good) == bad
    q34 = torch.zeros(5, 34, 128, dtype=torch.bfloat16, device="cuda")  # 17 per key head
    assert status(es, ro.es_attention, s.cache, s.batch, q34, torch.zeros_like(q34), ws, **good) == bad
    assert ro.es_attention_workspace(s.cache, 3) == 0 and ro.es_attention_workspace(s.cache, 34) == 0
    odd = torch.zeros(5 * 516, dtype=torch.bfloat16, device="cuda").view(5, 516)[:, :512]
    assert status(es, ro.es_attention, s.cache, s.batch, odd, out, ws, **good) == es.ES_ERR_ALIGNMENT
    off = torch.zeros(5 * 512 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(5, 512)
    assert status(es, ro.es_attention, s.cache, s.batch, off, out, ws, **good) == es.ES_ERR_ALIGNMENT
    host = torch.zeros(5, 4, 128, dtype=torch.bfloat16).pin_memory()
    with pytest.raises(ValueError):
        ro.es_attention(s.cache, s.batch, host, out, ws, **good)
    with pytest.raises(ValueError):
        ro.es_attention(s.cache, s.batch, q.float(), out, ws, **good)
    with pytest.raises(ValueError):
        ro.es_attention(s.cache, s.batch, q, out[:4], ws, **good)
    with pytest.raises(ValueError):
        ro.es_attention(s.cache, s.batch, q, out, ws, first=i32([0]), **good)
    for kw in (dict(max_new=0), dict(max_new=6), dict(tokens=-1)):
        a = dict(tokens=5, max_new=3) | kw
        b = ro.Batch(i32(s.pages), i32(s.seq_len), i32(s.start), a["tokens"], a["max_new"])
        x = torch.zeros(max(0, a["tokens"]), 4, 128, dtype=torch.bfloat16, device="cuda")
        if a["tokens"] < 0:
            assert status(es, ro.es_cache_read, s.cache, b) == bad
        else:
            assert status(es, ro.es_attention, s.cache, b, x, torch.zeros_like(x), ws, **good) == bad
    none = ro.Batch(i32(s.pages), i32(s.seq_len), i32([0, 0, 0]), 0, 1)
    ro.es_attention(s.cache, none, q[:0], out[:0], ws, **good)  # no tokens: nothing to do
    # append
    qkv = torch.zeros(5, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert status(es, ro.es_cache_append, s.cache, s.batch, qkv, q, eps=float("nan")) == es.ES_ERR_NONFINITE
    assert status(es, ro.es_cache_append, s.cache, s.batch, qkv, q, eps=-1.0) == bad
    assert status(es, ro.es_cache_append, s.cache, s.batch, qkv, q, rope=torch.zeros(9, 4, 2, device="cuda")) == bad
    assert status(es, ro.es_cache_append, s.cache, s.batch, qkv, q, rope=torch.zeros(9, 72, 2, device="cuda")) == bad
    with pytest.raises(ValueError):
        ro.es_cache_append(s.cache, s.batch, qkv[:, :7], q)


def test_cache_refusals(es, ro):
    bad = es.ES_ERR_INVALID_ARG
    page = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
    for shape in ((2, 2, 16, 96), (2, 2, 24, 128), (2, 2, 8, 128), (2, 2, 256, 128), (0, 2, 16, 128), (2, 1025, 16, 64)):
        assert status(es, ro.es_cache_create, page(*shape), page(*shape)) == bad
    x = page(2, 2, 16, 128)
    scale = torch.ones(2, 2, 16, device="cuda")
    assert status(es, ro.es_cache_create, x, x.clone(), scale, scale) == bad
    c = page(2, 2, 16, 128, dtype=torch.uint8)
    assert status(es, ro.es_cache_create, c, c.clone()) == bad
    off = torch.zeros(2 * 2 * 16 * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 2, 16, 128)
    assert status(es, ro.es_cache_create, off, x) == es.ES_ERR_ALIGNMENT
    with pytest.raises(ValueError):
        ro.es_cache_create(x, x[:1])
    with pytest.raises(ValueError):
        ro.es_cache_create(x.float(), x.float())
    with pytest.raises(ValueError):
        ro.es_cache_create(x.cpu(), x.cpu())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kw", [{}, {"softcap": 20.0}], ids=["plain", "cap"])
@pytest.mark.parametrize("shape", ["tiles", "units"])
def test_prompts_of_many_tiles(ro, dtype, kw, shape):
    if shape == "tiles":
        # blocks walk many tiles and units, most of them seen whole; units are shared by blocks
        s = Setup(ro, [3000, 700, 1500], [900, 700, 70], 2, 128, 64, dtype, seed=12)
        heads = 8
    else:
        # blocks walk many units, of one and of two tiles of rows in all orders
        new = [64, 20, 20, 20, 20, 20, 20, 40, 9] * 14
        s = Setup(ro, [n + 3 * i for i, n in enumerate(new)], new, 8, 64, 32, dtype, seed=12)
        heads = 32
    q, out, lse = attend(s, heads, **kw)
    k, v = s.dense()
    t = 0
    for b, n in enumerate(s.new):
        p = torch.arange(s.seq_len[b] - n, s.seq_len[b])[:, None]
        hide = torch.arange(s.seq_len[b])[None] > p
        for h in range(heads):
            x = (q[t:t + n, h].cpu().double() @ k[b][:, h // 4].T) * s.d ** -0.5
            if "softcap" in kw:
                x = kw["softcap"] * torch.tanh(x / kw["softcap"])
            x = x.masked_fill(hide, -math.inf)
            w = torch.softmax(x, -1)
            err = (out[t:t + n, h].cpu().double() - w @ v[b][:, h // 4]).abs()
            assert (err <= (2.0 ** -7 + 2.0 ** -12) * (w @ v[b][:, h // 4].abs())).all()
            assert ((lse[t:t + n, h].cpu().double() - torch.logsumexp(x, -1)).abs() <= 1e-4).all()
        t += n


@pytest.mark.parametrize("new", [1, 40])
def test_every_e4m3_code_counts_as_its_number(ro, new):
    # one key holds every code as its value (two heads of 128), and is all that is seen
    s = Setup(ro, [64], [new], 2, 128, 16, "e4m3")
    codes = torch.arange(256, dtype=torch.uint8).view(2, 128).cuda()
    page, slot = s.pages[0][0], 5
    s.v.view(torch.uint8)[page, :, slot] = codes
    s.vs[page, :, slot] = torch.tensor([1.0, 0.5], device="cuda")
    first = torch.full((new,), 5, dtype=torch.int32)
    q, out, lse = attend(s, 4, first=first, last=first + 1)
    want = (R.e4m3(codes.cpu()) * torch.tensor([[1.0], [0.5]])).repeat_interleave(2, 0)
    got = out.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want).expand_as(got))
    keep = ~torch.isnan(want)
    assert (got[:, keep] == want[keep]).all()
