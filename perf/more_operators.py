"""The operators of serving a network of AAP layers a token at a time, and what their performance is
measured on: the calls that a user makes of them, through paper_2410_05911_gb300.aecct.

Three operators, each direction a "kind" of case:

  append  kv_append: the keys and values of new tokens into a paged cache, quantised by eq. Quant as they are
          written: int8 codes with one scale for each token and head.  A 16-bit cache takes them as they are.
  read    kv_read: those of whole sequences back from the cache, one row for each token.
  attend  paged_attention: one new token of each sequence over its cached keys and values.
  sample  sample: the next token from a row of logits, by temperature, top-k, top-p and min-p, from given
          random numbers.

Sequences run from no token at all to a million; heads from the decoder's width of 16 to 256, odd ones
among them; pages from 8 tokens to 256; batches from one request to 512.
"""
import math

import torch

own = False

DTYPES = dict(fp32=torch.float32, bf16=torch.bfloat16, fp16=torch.float16, int8=torch.int8)
SIZE = dict(fp32=4, bf16=2, fp16=2, int8=1)
ALPHA_MIN = 2.0 ** -100  # the least absmax a row is scaled by


def listed():
    return [
        # one new token of one request: latency
        dict(name="append_token", kind="append", batch=1, length=700, new=1, heads=8, dim=128, page=64, dtype="bf16", cache="int8"),
        # prompts that arrive together, some 16,000 tokens of different lengths
        dict(name="append_prompts", kind="append", batch=8, length=4000, new=4000, heads=8, dim=128, page=64, dtype="bf16", cache="int8"),
        # the tail of 37 prompts of a model in 32 bits, heads of an odd width, pages of 24 tokens
        dict(name="append_odd", kind="append", batch=37, length=2500, new=333, heads=12, dim=100, page=24, dtype="fp32", cache="int8"),
        # whole sequences read back: a prefix that is attended to by many tokens at once, or moved
        dict(name="read_sequences", kind="read", batch=32, length=4000, heads=8, dim=128, page=64, dtype="bf16", cache="int8"),
        # the same from a cache in 16 bits, with pages of 8 tokens and heads that no vector load divides
        dict(name="read_odd", kind="read", batch=13, length=3001, heads=5, dim=77, page=8, dtype="fp16", cache="fp16"),
        # one request early in its answer: latency
        dict(name="attend_token", kind="attend", batch=1, length=500, heads=8, group=4, dim=128, page=64, dtype="bf16", cache="int8", window=0),
        # a serving batch, contexts of up to 8,000 tokens
        dict(name="attend_batch", kind="attend", batch=64, length=8000, heads=8, group=4, dim=128, page=64, dtype="bf16", cache="int8", window=0),
        # a single request over a very long context
        dict(name="attend_long", kind="attend", batch=1, length=1000003, heads=8, group=8, dim=128, page=256, dtype="bf16", cache="int8", window=0),
        # many short sequences through the decoder's own heads (d = 128 in 8 of them), in its own type
        dict(name="attend_words", kind="attend", batch=512, length=180, heads=8, group=1, dim=16, page=16, dtype="fp32", cache="int8", window=0),
        # a cache in 16 bits, heads of 80, pages of 24, a sliding window over most of the sequences
        dict(name="attend_odd", kind="attend", batch=29, length=9001, heads=12, group=3, dim=80, page=24, dtype="fp16", cache="fp16", window=4099),
        # the next token of one request, every filter on: latency
        dict(name="sample_token", kind="sample", batch=1, vocab=50021, dtype="fp32", t=0.8, k=50, p=0.95, min_p=0.02, each=False),
        # a serving batch whose requests have their own settings
        dict(name="sample_batch", kind="sample", batch=128, vocab=131072, dtype="bf16", t=0.9, k=0, p=0.9, min_p=0.0, each=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("append", "read", "attend", "sample"), (0.22, 0.15, 0.4, 0.23))[0]
    dtype = rng.choice(("bf16", "bf16", "fp32", "fp16"))
    if kind == "sample":
        vocab = _log_int(rng, 100, 300000)
        batch = _log_int(rng, 1, max(1, min(512, 16 * 10 ** 6 // vocab)))
        return dict(kind=kind, batch=batch, vocab=vocab, dtype=dtype, t=round(rng.choice((rng.uniform(0.2, 1.6), rng.uniform(0.6, 1.0))), 3),
                    k=rng.choice((0, 0, 1, _log_int(rng, 2, vocab))), p=rng.choice((1.0, 0.9, round(rng.uniform(0.05, 0.999), 3))),
                    min_p=rng.choice((0.0, 0.0, round(rng.uniform(0.001, 0.3), 4))), each=rng.random() < 0.4)
    heads = rng.choice((1, 2, 4, 8, 8, 16, rng.randint(1, 40)))
    dim = rng.choice((16, 32, 64, 128, 128, 256, rng.randint(8, 256), 8 * rng.randint(3, 31)))
    page = rng.choice((8, 16, 16, 32, 64, 128, 256, rng.randint(8, 100)))
    cache = "int8" if dtype == "fp32" else rng.choice(("int8", "int8", dtype))
    group = rng.choice((1, 2, 4, 7, 8, 16))
    most = (2000 if kind == "attend" else 200) * 10 ** 6 // (2 * heads * dim * SIZE[cache])  # tokens
    if kind == "attend":
        most = min(most, 8 * 10 ** 9 // (heads * dim * group))
    batch = _log_int(rng, 1, max(1, min(512, most // 64)))
    length = _log_int(rng, 1, max(2, min(10 ** 6, most // batch)))
    case = dict(kind=kind, batch=batch, length=length, heads=heads, dim=dim, page=page, dtype=dtype, cache=cache)
    if kind == "append":
        return dict(case, new=rng.choice((1, 1, length, _log_int(rng, 1, length))))
    if kind == "attend":
        return dict(case, group=group, window=rng.choice((0, 0, 0, _log_int(rng, 1, length))))
    return case


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _lengths(case, g):
    """One sequence of the case's length and others shorter than that; one in sixteen of a large batch is a free place, without
    a token.  Their order is the inputs' own, their sum the case's."""
    b, most = case["batch"], case["length"]
    n = ((0.1 + 0.9 * (torch.arange(b) + 1) / b) * most).round().long().clamp(1, most)
    if b >= 16:
        n[torch.arange(b) % 16 == 5] = 0
    return n[torch.randperm(b, generator=g)].tolist()


def _cache(case, pages):
    """An empty cache: k and v [pages, heads, page, dim], and for int8 codes a scale for each row of them."""
    shape, dtype = (pages, case["heads"], case["page"], case["dim"]), DTYPES[case["cache"]]
    if own:
        from paper_2410_05911_gb300 import aecct

        c = aecct.kv_cache(*shape, dtype=dtype)
        for t in c:
            if t is not None:
                t.zero_()
        return c
    scales = [torch.zeros(shape[:3], device="cuda") if case["cache"] == "int8" else None for _ in range(2)]
    return tuple(torch.zeros(shape, device="cuda", dtype=dtype) for _ in range(2)) + tuple(scales)


def _fill(t, g):
    """Keys or values of a model, as a cache holds them: codes of every size, or numbers of about unit size."""
    if t.dtype == torch.int8:
        for part in t.split(max(1, (1 << 28) // max(1, t[0].numel()))):
            part.copy_(torch.empty(part.shape, device="cuda", dtype=torch.float16).normal_(0, 42, generator=g).clamp_(-127, 127).round_())
    elif t.dtype == torch.float32:
        t.copy_(torch.exp(0.4 * torch.randn(t.shape, device="cuda", generator=g)) * 0.02)
    else:
        t.copy_(torch.empty(t.shape, device="cuda", dtype=t.dtype).normal_(generator=g))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    kind, st, dtype = case["kind"], dict(case=case), DTYPES[case["dtype"]]
    if kind == "sample":
        b, v = case["batch"], case["vocab"]
        x = torch.empty((b, v), device="cuda").normal_(generator=g)
        x *= 1.0 + 2.5 * torch.rand((b, 1), device="cuda", generator=g)  # sure and unsure rows
        x[:, torch.randint(0, v, (max(1, v // 50),), device="cuda", generator=g)] = -math.inf  # words that are not allowed
        x[:, 0] = 0.0
        st["logits"], st["u"] = x.to(dtype), torch.rand((b,), device="cuda", generator=g)
        st["t"], st["k"], st["p"], st["min_p"] = case["t"], case["k"], case["p"], case["min_p"]
        if case["each"]:  # settings of each request's own, one in eight of them greedy, one in eight without a filter
            r = torch.rand((b,), device="cuda", generator=g)
            st["t"] = torch.where(r < 0.125, 0.0, case["t"] * (0.8 + 0.4 * r)).float()
            st["k"] = torch.where(r > 0.6, max(case["k"], 20), case["k"]).int()
            st["p"] = torch.where(r > 0.875, 1.0, case["p"] - 0.04 * r).float()
            st["min_p"] = torch.where(r > 0.75, 0.01, case["min_p"]).float()
        return st
    lens = _lengths(case, host)
    page, heads, dim = case["page"], case["heads"], case["dim"]
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 1, generator=host)  # pages are handed out as they come free
    table = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n], at = order[at:at + n], at + n
    st["lens"], st["table"], st["lengths"] = lens, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    st["cache"] = _cache(case, sum(need) + 1)
    if kind == "append":
        new = [min(n, case["new"]) for n in lens]
        rows = [0]
        for n in new:
            rows.append(rows[-1] + n)
        st["new"], st["one"] = new, case["new"] == 1 and min(new) == 1
        st["rows"] = torch.tensor(rows, dtype=torch.int32).cuda()
        fused = torch.empty((rows[-1], 6 * heads * dim), device="cuda").normal_(generator=g)  # (a row of the product that makes queries, keys and values)
        fused *= torch.exp(0.5 * torch.randn((rows[-1], 1), device="cuda", generator=g))
        fused = fused.to(dtype)
        st["k_new"], st["v_new"] = (fused[:, i * heads * dim:(i + 1) * heads * dim].view(-1, heads, dim) for i in (4, 5))
        return st
    for t in st["cache"]:
        if t is not None:
            _fill(t, g)
    if kind == "read":
        rows = [0]
        for n in lens:
            rows.append(rows[-1] + n)
        st["total"], st["rows"] = rows[-1], torch.tensor(rows, dtype=torch.int32).cuda()
        return st
    q = torch.empty((len(lens), heads * case["group"], dim), device="cuda").normal_(generator=g)
    q *= 0.5 + 2.5 * torch.rand((1, heads * case["group"], 1), device="cuda", generator=g)  # flat heads and sharp ones
    st["q"] = q.to(dtype)
    st["firsts"] = [max(0, n - case["window"]) if case["window"] else 0 for n in lens]
    st["first"] = torch.tensor(st["firsts"], dtype=torch.int32).cuda() if case["window"] else None
    return st


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return (_own if own else _plain)[kind](st)


def _named(cache):
    return {n: t for n, t in zip(("k", "v", "k_scale", "v_scale"), cache) if t is not None}


def _places(st, n):
    """Where the cache holds the last tokens of each sequence that the n rows stand for: a page and a place in it, for each row."""
    page = st["case"]["page"]
    seq = torch.repeat_interleave(torch.arange(len(st["lens"]), device="cuda"), st["rows"].diff(), output_size=n)
    at = torch.arange(n, device="cuda") - st["rows"][seq + 1] + st["lengths"][seq]
    return st["table"][seq, at // page].long(), at % page


def _append(st):
    cache = st["cache"]
    slot, off = _places(st, st["k_new"].shape[0])
    for x, t, s in ((st["k_new"], cache[0], cache[2]), (st["v_new"], cache[1], cache[3])):
        if s is None:
            t[slot, :, off] = x.to(t.dtype)
            continue
        x = x.float()
        alpha = x.abs().amax(2).clamp_min(ALPHA_MIN)
        t[slot, :, off] = torch.round(x * torch.div(torch.full_like(alpha, 127.0), alpha)[:, :, None]).to(torch.int8)
        s[slot, :, off] = alpha / 127.0
    return _named(cache)


def _values(t, s, at):
    x = t[at].float()
    return x if s is None else x * s[at][..., None]


def _read(st):
    cache, dtype = st["cache"], DTYPES[st["case"]["dtype"]]
    slot, off = _places(st, st["total"])
    at = (slot, slice(None), off)
    return dict(k=_values(cache[0], cache[2], at).to(dtype), v=_values(cache[1], cache[3], at).to(dtype))


def _attend(st):
    case, cache = st["case"], st["cache"]
    pages, b, heads = st["table"].clamp_min(0).long(), case["batch"], case["heads"]

    def every(t, s):  # [batch, heads, positions, dim]
        x = _values(t, s, pages)
        return x.transpose(1, 2).reshape(b, heads, -1, case["dim"])

    q = st["q"].float().view(b, heads, -1, case["dim"])
    s = (q @ every(cache[0], cache[2]).transpose(2, 3)) * (case["dim"] ** -0.5)
    at = torch.arange(s.shape[3], device="cuda")[None]
    seen = at < st["lengths"][:, None]
    if st["first"] is not None:
        seen &= at >= st["first"][:, None]
    s = torch.where(seen[:, None, None], s, -math.inf)
    e = torch.exp(s - s.amax(3, keepdim=True).clamp_min(-1e30))
    o = (e @ every(cache[1], cache[3])) / e.sum(3, keepdim=True).clamp_min(1e-30)
    return dict(out=o.reshape(st["q"].shape).to(st["q"].dtype))


def _column(v, like):
    """A setting for every row, or one for each, as a column."""
    return v.double()[:, None] if isinstance(v, torch.Tensor) else torch.full((1, 1), float(v), dtype=torch.float64, device=like.device)


def _sample(st):
    x = st["logits"].double()
    t, k, p, min_p = (_column(st[n], x) for n in ("t", "k", "p", "min_p"))
    p, min_p = p.float().double(), min_p.float().double()  # (a call takes settings in 32 bits)
    t = t.float().double()
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(t > 0, t, 1.0))
    w = torch.where(torch.isfinite(x), w.clamp_min(1e-300), 0.0)
    rank = torch.arange(x.shape[1], device="cuda")[None]
    keep = (rank < k) | (k <= 0)
    wk = torch.where(keep, w, 0.0)
    upto = torch.cumsum(wk, 1)
    keep = keep & ((upto - wk < p * upto[:, -1:]) | (p >= 1) | (rank == 0)) & (w >= min_p)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    upto = torch.cumsum(kept, 1)
    picked = ((upto > st["u"].double()[:, None] * upto[:, -1:]) & (kept > 0)).int().argmax(1)
    return dict(tokens=torch.where(t[:, 0] > 0, picked, order[:, 0]))


def _own_append(st):
    from paper_2410_05911_gb300 import aecct

    aecct.kv_append(st["k_new"], st["v_new"], st["cache"], st["table"], st["lengths"], rows=None if st["one"] else st["rows"])
    return _named(st["cache"])


def _own_read(st):
    from paper_2410_05911_gb300 import aecct

    k, v = aecct.kv_read(st["cache"], st["table"], st["lengths"], st["rows"], st["total"], dtype=DTYPES[st["case"]["dtype"]])
    return dict(k=k, v=v)


def _own_attend(st):
    from paper_2410_05911_gb300 import aecct

    out, _ = aecct.paged_attention(st["q"], st["cache"], st["table"], st["lengths"], first=st["first"])
    return dict(out=out)


def _own_sample(st):
    from paper_2410_05911_gb300 import aecct

    return dict(tokens=aecct.sample(st["logits"], st["u"], temperature=st["t"], top_k=st["k"], top_p=st["p"], min_p=st["min_p"]))


_plain = dict(append=_append, read=_read, attend=_attend, sample=_sample)
_own = dict(append=_own_append, read=_own_read, attend=_own_attend, sample=_own_sample)


# ------------------------------------------------------------------------------------------
# the work of a pass
# ------------------------------------------------------------------------------------------
def work(case):
    kind, s = case["kind"], SIZE[case["dtype"]]
    if kind == "sample":
        n = float(case["batch"]) * case["vocab"]
        return dict(bytes=n * s + 12.0 * case["batch"], flops=4.0 * n)
    mean = (0.1 * case["batch"] + 0.45 * (case["batch"] + 1)) * (15 / 16 if case["batch"] >= 16 else 1)  # sequences of the largest length
    tokens = mean * case["length"]
    row = 2.0 * case["heads"] * (case["dim"] * SIZE[case["cache"]] + (4 if case["cache"] == "int8" else 0))  # a token in the cache
    if kind == "append":
        tokens = min(tokens, float(case["batch"]) * case["new"])
    if kind in ("append", "read"):
        values = 2.0 * tokens * case["heads"] * case["dim"]
        return dict(bytes=tokens * row + values * s + 8.0 * case["batch"], flops=2 * values)
    if case["window"]:
        tokens = min(tokens, float(case["batch"]) * case["window"])
    q = float(case["batch"]) * case["heads"] * case["group"] * case["dim"]
    return dict(bytes=tokens * row + 2 * q * s, flops=4.0 * tokens * case["heads"] * case["group"] * case["dim"])


# ------------------------------------------------------------------------------------------
# the same values in 64 bits
# ------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "sample":
        return None  # (tokens are whole numbers)
    st = prepare(case, seed)
    page = case["page"]
    names = ("k", "v", "k_scale", "v_scale")
    cache = dict(zip(names, st["cache"]))
    if case["kind"] == "append":
        wide = {n: t.double() for n, t in cache.items() if t is not None and t.dtype != torch.int8}
        at = 0
        for b, (n, new) in enumerate(zip(st["lens"], st["new"])):
            positions = torch.arange(n - new, n, device="cuda")
            where = (st["table"][b].long()[positions // page], slice(None), positions % page)
            for name in ("k", "v"):
                x = st[name + "_new"][at:at + new].double()
                if case["cache"] == "int8":
                    wide[name + "_scale"][where] = torch.linalg.vector_norm(x, ord=math.inf, dim=2).clamp_min(ALPHA_MIN) / 127
                else:
                    wide[name][where] = x
            at += new
        return {n: wide.get(n) for n in names if cache[n] is not None}

    def rows(name, b, positions):
        at = (st["table"][b].long()[positions // page], slice(None), positions % page)
        x = cache[name][at].double()
        return x if cache[name + "_scale"] is None else torch.einsum("nhd,nh->nhd", x, cache[name + "_scale"][at].double())

    if case["kind"] == "read":
        every = [torch.arange(n, device="cuda") for n in st["lens"]]
        return {name: torch.cat([rows(name, b, p) for b, p in enumerate(every)]) for name in ("k", "v")}
    if sum(st["lens"]) * case["heads"] * case["dim"] * case["group"] > 10 ** 10 or max(st["lens"]) * case["heads"] * case["dim"] > 2 * 10 ** 9:
        return None
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["lens"]):
        if n:
            positions = torch.arange(st["firsts"][b], n, device="cuda")
            q = st["q"][b].double().unflatten(0, (case["heads"], case["group"]))
            p = torch.softmax(torch.einsum("hgd,nhd->hgn", q, rows("k", b, positions)) / math.sqrt(case["dim"]), dim=2)
            out[b] = torch.einsum("hgn,nhd->hgd", p, rows("v", b, positions)).flatten(0, 1)
    return dict(out=out)
