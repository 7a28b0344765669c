"""paged_attention on the GPU against its formula in 64 bits, on the same codes and scales.

Tolerances, from the operations.  A score is a sum of d products, whose additions on the tensor cores cut off up to 2^-23 of what
is there, and a few products rounded to 2^-24: off by at most e = (d + 8) 2^-23 A, A the largest scale sum_i |q_i k_ji| of the
head (a float32 q is cut into two pieces of 11 bits, 2^-22 of it, inside of that).  A weight is then off by a factor of 1 + e, and
by its own rounding w: 2^-22 for exp2, and to the type that the tensor cores take: 2^-11 for bfloat16 queries on codes (one
piece in half), 2^-16 for a cache in bfloat16 (two pieces), else 2^-22 (two pieces in half).  Weights change the output both in the sum and
under the quotient: (2 e + 2 w) sum_j p_j |v_j|; its additions in 32 bits, one for 16 keys and some for the parts, add
(n / 16 + 64) 2^-23 of it; the result is rounded once.
Weights in half end at its smallest step, 2^-24: one that is less than 2^-29 of the largest, which is 2^14 to 2^15, is off by half
a step, 2^-25, and not by a part of itself.  In units of the largest weight with its row's scale, max_j p_j vs_j, that is 2^-39 at most (vs = 1 for
rows without a scale), and over the keys 2^-39 max_j (p_j vs_j) sum_j |c_jd|, c the codes (or a half cache's values)."""
import math

import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}
F16, BF16, F32, I8 = torch.float16, torch.bfloat16, torch.float32, torch.int8


def make(lens, heads, group, dim, page, dtype, cache_dtype, seed=0, spread=1.0, first=None):
    """A cache whose unused rows, pages and scales are NaN or large, and queries.  `spread` is the size of the queries."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-max(0, n) // page) for n in lens]
    total = sum(need) + 2
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(lens), max(need + [1])), 10 ** 6, dtype=torch.int32)
    cache = A.kv_cache(total, heads, page, dim, dtype=cache_dtype)
    used = torch.zeros((total, page), dtype=torch.bool)
    at = 0
    for b, n in enumerate(need):
        table[b, :n], at = order[at:at + n].int(), at + n
        for i in range(n):
            used[table[b, i], :max(0, min(page, lens[b] - i * page))] = True
    used = used.cuda()[:, None]
    for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        if cache_dtype is I8:
            x.copy_(torch.randint(-127, 128, x.shape, device="cuda", generator=g))
            s.copy_(torch.exp(torch.randn(s.shape, device="cuda", generator=g)) / 64)
            s.copy_(torch.where(used, s, float("nan")))
            x.copy_(torch.where(used[..., None], x, 127))
        else:
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
            x.copy_(torch.where(used[..., None], x, float("nan")))
    q = (torch.randn((len(lens), heads * group, dim), device="cuda", generator=g) * spread).to(dtype)
    return q, cache, table.cuda(), torch.tensor(lens, **I32), first


def reference(q, cache, table, lengths, first=None, scale=None):
    """Output and lse in 64 bits, and what the tolerances take: the largest absolute score, the weighted sum of |v|, the steps of small weights."""
    pages, heads, page, dim = cache.k.shape
    batch, hq = q.shape[:2]
    scale = dim ** -0.5 if scale is None else scale
    out = torch.zeros((batch, hq, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((batch, hq), -math.inf, dtype=torch.float64, device="cuda")
    big, mass, step = torch.zeros((batch, hq, 1), dtype=torch.float64, device="cuda"), torch.zeros_like(out), torch.zeros_like(out)
    for b in range(batch):
        n = min(max(0, int(lengths[b])), table.shape[1] * page)
        at = torch.arange(min(n, max(0, int(first[b]))) if first is not None else 0, n, device="cuda")
        on = table[b].long()[at // page]
        fine = (on >= 0) & (on < pages)
        at, on = at[fine], on[fine]
        if not len(at):
            continue
        k, v = (x[on, :, at % page].double() * (1.0 if s is None else s[on, :, at % page].double()[..., None])
                for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        k, v = (t.transpose(0, 1).repeat_interleave(hq // heads, 0) for t in (k, v))  # [hq, n, dim]
        qb = q[b].double()[:, None]
        s = (qb * k).sum(2) * scale
        big[b] = ((qb * k).abs().sum(2) * abs(scale)).amax(1, keepdim=True)
        lse[b] = torch.logsumexp(s, 1)
        p = torch.softmax(s, 1)[:, None]
        out[b], mass[b] = (p @ v)[:, 0], (p @ v.abs())[:, 0]
        vs = torch.ones_like(p) if cache.v_scale is None else cache.v_scale[on, :, at % page].double().t().repeat_interleave(hq // heads, 0)[:, None]
        step[b] = 2.0 ** -39 * (p * vs).amax(2) * (v.abs() / vs[:, 0, :, None]).sum(1)
    return out, lse, big, mass, step


def with_room(table, page, tokens=40000):
    """The same table with columns of no page for `tokens` more tokens: calls whose sequences may be long deal out their tiles, others take
    a cluster to each sequence."""
    return torch.cat([table, torch.full((table.shape[0], -(-tokens // page)), -1, **I32)], 1)


def check(q, cache, table, lengths, first=None, scale=None, **kw):
    """Both ways, the second's result."""
    page = cache.k.shape[2]
    if q.shape[0] <= 300 and not int((lengths > table.shape[1] * page).sum()):
        check_one(q, cache, with_room(table, page), lengths, first, scale, **kw)
    return check_one(q, cache, table, lengths, first, scale, **kw)


def check_one(q, cache, table, lengths, first=None, scale=None, **kw):
    out, lse = A.paged_attention(q, cache, table, lengths, first=first, scale=scale, want_lse=True, **kw)
    want, wl, big, mass, step = reference(q, cache, table, lengths, first, scale)
    assert out.dtype == q.dtype and out.shape == q.shape and lse.shape == q.shape[:2] and lse.dtype == F32
    n, dim = max(1, int(lengths.max())), q.shape[2]
    e = (dim + 8) * 2.0 ** -23 * big
    w = 2.0 ** -11 if q.dtype is BF16 and cache.k.dtype is I8 else 2.0 ** -16 if cache.k.dtype is BF16 else 2.0 ** -22
    tol = (2 * e + 2 * (w + 2.0 ** -22) + (n / 16 + 64) * 2.0 ** -23) * mass + HALF[q.dtype] * want.abs() + TINY[q.dtype]
    if cache.k.dtype is not BF16:
        tol = tol + step
    off = (out.double() - want).abs()
    assert (off <= tol).all(), (off / tol).max().item()
    empty = wl == -math.inf
    assert (lse[empty] == -math.inf).all() and not out[empty].any()
    tl = e[..., 0] + (n / 16 + 64) * 2.0 ** -23 + 2.0 ** -21 * wl.abs()
    assert ((lse.double() - wl).abs()[~empty] <= tl[~empty]).all()
    return out


KINDS = [(BF16, I8), (F16, I8), (F32, I8), (F16, F16), (BF16, BF16)]


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("dim", [1, 8, 16, 24, 32, 33, 64, 77, 80, 96, 128, 130, 192, 256])
def test_dims(dim, dtype, cache):
    check(*make([45, 1, 130, 0, 16], 3, 2, dim, 16, dtype, cache, seed=dim))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 40])
def test_groups(group, dtype, cache):
    check(*make([100, 37], 2, group, 64, 16, dtype, cache, seed=group))
    check(*make([100, 37], 1, group, 128, 16, dtype, cache, seed=group))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("page", [1, 3, 8, 16, 24, 31, 32, 33, 64, 100, 256])
def test_pages(page, dtype, cache):
    check(*make([200, 31, 32, 33, 1, 15], 2, 4, 128, page, dtype, cache, seed=page))


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_every_length(dtype, cache):
    check(*make(list(range(0, 131)), 1, 4, 64, 16, dtype, cache))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("batch,length", [(1, 1), (1, 5000), (1, 40000), (3, 9000), (600, 40), (2000, 3)])
def test_splits(batch, length, dtype, cache):
    """Few long sequences, which many CTAs share, to many short ones, of which a warp takes several."""
    lens = [max(0, length - (b * 7) % max(1, length)) for b in range(batch)]
    check(*make(lens, 2, 4, 32, 64, dtype, cache, seed=batch))


def test_one_long_sequence_among_many():
    lens = [3] * 300 + [30000] + [0] * 40 + [17] * 100
    check(*make(lens, 2, 4, 64, 32, BF16, I8))
    check(*make(lens[::-1], 1, 8, 128, 32, F32, I8))


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_first_positions(dtype, cache):
    lens = [100, 100, 100, 64, 64, 5, 0, 1000]
    q, c, table, lengths, _ = make(lens, 2, 4, 128, 16, dtype, cache)
    for first in ([0, 1, 99, 63, 64, 100, 0, 937], [-5, 33, 16, 17, 2 ** 31 - 1, 4, 3, 0]):
        check(q, c, table, lengths, first=torch.tensor(first, **I32))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0])
def test_flat_and_sharp_rows(spread, dtype, cache):
    check(*make([700, 90], 2, 4, 64, 16, dtype, cache, spread=spread))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sizes_of_queries_and_scales_far_from_one(dtype):
    for size in (1e-30, 1e30):
        q, c, table, lengths, _ = make([300, 40], 2, 4, 64, 16, dtype, I8)
        q = (q.float() * size).to(dtype)
        c.k_scale.mul_(1 / size)
        check(q, c, table, lengths)


def test_values_scales_that_differ_by_far():
    """Rows of zeros (their scale is 2^-100 / 127), and a row 2^40 times larger than all others that no query attends to."""
    q, c, table, lengths, _ = make([300], 1, 4, 64, 16, F32, I8)
    on = table[0].long()
    c.v_scale[on[3]] = 2.0 ** -100 / 127
    c.v[on[3]] = 0
    c.k[on[5], 0, 7], c.k_scale[on[5], 0, 7] = 1, 1.0
    q[:] = -20.0
    c.k[on[5], 0, 7] = 100  # a score of -16,000
    c.v_scale[on[5], 0, 7] = 2.0 ** 40
    check(q, c, table, lengths)


def test_scale_and_strides():
    q, c, table, lengths, _ = make([90, 40, 33], 2, 3, 40, 16, BF16, I8)
    for scale in (0.3, 0.0, -0.1, 2.0):
        check(q, c, table, lengths, scale=scale)
    wide = torch.zeros((3, 5, 6, 43), device="cuda", dtype=BF16)
    wide[:, 2, :, 3:] = q
    assert torch.equal(check(wide[:, 2, :, 3:], c, table, lengths), check(q, c, table, lengths))
    turned = q.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    assert turned.stride(2) != 1
    check(turned, c, table, lengths)
    check(q[:1].expand(3, 6, 40), c, table, lengths)
    t = torch.full((3, 11), -7, **I32)
    t[:, 4:4 + table.shape[1]] = table
    check(q, c, t[:, 4:], lengths)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_pages_that_are_none(dtype, cache):
    q, c, table, lengths, _ = make([200, 200, 40], 2, 4, 64, 16, dtype, cache)
    table[0, 3], table[0, 7], table[1, :], table[2, 2] = -1, 2 ** 31 - 1, -1, c.k.shape[0]
    check(q, c, table, lengths)


def test_lengths_past_the_table_and_negative():
    q, c, table, lengths, _ = make([64, 64, 30], 2, 4, 64, 16, BF16, I8)
    check(q, c, table, torch.tensor([2 ** 31 - 1, 65, -3], **I32))


def test_sequences_that_share_pages():
    q, c, table, lengths, _ = make([100, 100], 2, 4, 64, 16, BF16, I8)
    table[1] = table[0]
    q[1] = q[0]
    out = check(q, c, table, lengths)
    off = (out[0].double() - out[1].double()).abs()
    assert (off <= 2.0 ** -7 * out[0].double().abs() + 1e-3).all()


def test_rows_that_are_not_numbers_stay_in_their_sequence():
    q, c, table, lengths, _ = make([100, 100, 100], 2, 4, 64, 16, F16, F16)
    c.k[table[1, 2].long(), 1, 3, 5] = float("nan")
    out, lse = A.paged_attention(q, c, table, lengths, want_lse=True)
    assert out[1, 4:].isnan().all() and lse[1, 4:].isnan().all()
    assert out[0].isfinite().all() and out[2].isfinite().all() and out[1, :4].isfinite().all()


def test_a_cache_past_32_bits():
    """Rows that lie more than 2^32 bytes from the start of the cache."""
    pages, heads, page, dim = 70000, 4, 64, 256  # 4.6e9 bytes
    c = A.kv_cache(pages, heads, page, dim)
    last = pages - 3
    for t in (c.k, c.v):
        t[last:] = torch.randint(-127, 128, (3, heads, page, dim), device="cuda", dtype=torch.int8)
    for s in (c.k_scale, c.v_scale):
        s[last:] = torch.rand((3, heads, page), device="cuda") * 0.01 + 0.01
    table, lengths = torch.tensor([[last, last + 2, last + 1]], **I32), torch.tensor([190], **I32)
    q = torch.randn((1, 8, dim), device="cuda")
    check(q, c, table, lengths)
    A.kv_append(q[:, :heads], q[:, heads:], c, table, lengths)
    k, v = A.kv_read(c, table, lengths, None, 1)
    assert ((k - q[:, :heads]).abs() <= q.abs().amax() / 127).all() and ((v - q[:, heads:]).abs() <= q.abs().amax() / 127).all()
    check(q, c, table, lengths)


def test_same_bits_on_every_run_on_another_stream_and_in_graphs():
    q, c, table, lengths, _ = make([3000, 1, 700, 20], 2, 4, 128, 32, BF16, I8)
    out, lse = A.paged_attention(q, c, table, lengths, want_lse=True)
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    torch.cuda._sleep(50_000_000)
    late.copy_(q)
    again = A.paged_attention(late, c, table, lengths, want_lse=True, stream=side)
    side.synchronize()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    graphs, outs = [], []
    pool = torch.cuda.graph_pool_handle()
    for _ in range(2):  # two graphs that share a pool, and so their workspaces
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(A.paged_attention(late, c, table, lengths)[0])
        graphs.append(g)
    for n in ([3000, 1, 700, 20], [5, 0, 699, 19]):  # the lengths change between replays
        lengths.copy_(torch.tensor(n, **I32))
        for g, o in zip(graphs, outs):
            g.replay()
            assert torch.equal(o, A.paged_attention(q, c, table, lengths)[0])
    check(q, c, table, lengths)


def test_two_calls_at_once():
    a = make([2000, 300], 2, 4, 128, 16, BF16, I8, seed=1)[:4]
    b = make([1500, 9], 4, 2, 64, 16, F32, I8, seed=2)[:4]
    want = [A.paged_attention(*x)[0] for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[A.paged_attention(*x, stream=s)[0] for _ in range(20)] for x, s in zip((a, b), streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for outs, w in zip(got, want) for o in outs)


def test_nothing_to_do():
    q, c, table, lengths, _ = make([8], 2, 4, 64, 16, BF16, I8)
    out, lse = A.paged_attention(q[:0], c, table[:0], lengths[:0], want_lse=True)
    assert out.shape == (0, 8, 64) and lse.shape == (0, 8)
    out, lse = A.paged_attention(q, c, table[:, :0], lengths, want_lse=True)
    assert not out.any() and (lse == -math.inf).all()
    out, lse = A.paged_attention(q, A.kv_cache(0, 2, 16, 64), table, lengths)
    assert not out.any() and lse is None


def test_refusals():
    q, c, table, lengths, _ = make([8], 2, 4, 64, 16, BF16, I8)
    half = A.kv_cache(4, 2, 16, 64, dtype=F16)
    calls = [lambda: A.paged_attention(q[:, :3], c, table, lengths), lambda: A.paged_attention(q[..., :32], c, table, lengths),
             lambda: A.paged_attention(q, half, table, lengths), lambda: A.paged_attention(q.double(), c, table, lengths),
             lambda: A.paged_attention(q.expand(2, 8, 64), c, table, lengths), lambda: A.paged_attention(q[0], c, table, lengths),
             lambda: A.paged_attention(q, c, table, lengths, first=lengths.long()), lambda: A.paged_attention(q, c, table, lengths, first=table),
             lambda: A.paged_attention(q.requires_grad_(), c, table, lengths), lambda: A.paged_attention(q.cpu(), c, table, lengths),
             lambda: A.paged_attention(q, tuple(c[:2]), table, lengths)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    with torch.no_grad():
        for scale in (math.inf, math.nan, 1e39):
            with pytest.raises(A.AecctError):
                A.paged_attention(q, c, table, lengths, scale=scale)
