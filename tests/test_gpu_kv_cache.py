"""kv_append and kv_read on the GPU, bit for bit against eq. Quant in numpy's 32-bit arithmetic (each operation is rounded
once there and here: the quotient 127 / alpha, the product with it, the rounding to a whole number, alpha / 127)."""
import math

import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]
I32 = dict(dtype=torch.int32, device="cuda")


def quant(x):
    """Codes and scales of rows (the last dimension) in float32."""
    x = x.float().cpu().numpy()
    alpha = np.maximum(np.abs(x).max(-1), np.float32(2.0 ** -100)).astype(np.float32)
    codes = np.rint(x * (np.float32(127) / alpha)[..., None]).astype(np.int8)
    return codes, alpha / np.float32(127)


def pages_for(lens, page, spare=3, seed=0):
    """A table with pages in no order, its unused entries of no page, and the number of pages."""
    need = [-(-n // page) for n in lens]
    order = np.random.default_rng(seed).permutation(sum(need) + spare)
    table = np.full((len(lens), max(need + [1])), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n], at = order[at:at + n], at + n
    return torch.tensor(table).cuda(), sum(need) + spare


def marked(pages, heads, page, dim, dtype):
    """A cache full of a mark."""
    c = A.kv_cache(pages, heads, page, dim, dtype=dtype)
    for t in c:
        if t is not None:
            t.fill_(77)
    return c


def tokens(n, heads, dim, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, heads * dim * 3 + pad), device="cuda", generator=g) * torch.exp(torch.randn((n, 1), device="cuda", generator=g))
    x[torch.rand((n,), device="cuda", generator=g) < 0.1] = 0.0
    x = x.to(dtype)
    return x[:, :heads * dim].view(n, heads, dim), x[:, 2 * heads * dim:3 * heads * dim].view(n, heads, dim)


def check(lens, new, heads, dim, page, dtype, cache_dtype, pad=0, rows=True):
    table, pages = pages_for(lens, page)
    cache = marked(pages, heads, page, dim, cache_dtype)
    at = np.concatenate([[0], np.cumsum(new)])
    k, v = tokens(int(at[-1]), heads, dim, dtype, sum(lens) + dim, pad)
    lengths = torch.tensor(lens, **I32)
    where = torch.tensor(at, **I32) if rows else None
    A.kv_append(k, v, cache, table, lengths, rows=where)
    t = table.cpu().numpy()
    for x, c, s in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want = np.full(c.shape, 77, np.float32)
        ws = np.full(c.shape[:3], 77, np.float32)
        codes, scale = quant(x) if s is not None else (x.float().cpu().numpy(), None)
        for b in range(len(lens)):
            for i in range(new[b]):
                p, r = lens[b] - new[b] + i, at[b] + i
                if p < 0:
                    continue
                want[t[b, p // page], :, p % page] = codes[r]
                if s is not None:
                    ws[t[b, p // page], :, p % page] = scale[r]
        assert np.array_equal(c.float().cpu().numpy(), want)
        if s is not None:
            assert np.array_equal(s.cpu().numpy(), ws)
    for out_dtype in DTYPES:  # and back
        back = A.kv_read(cache, table, lengths, where, int(at[-1]), dtype=out_dtype)
        for x, got in zip((k, v), back):
            if cache_dtype is torch.int8:
                codes, scale = quant(x)
                want = torch.tensor(codes.astype(np.float32) * scale[..., None])
            else:
                want = x.float().cpu()
            want = want.to(out_dtype)
            for b in range(len(lens)):
                drop = max(0, new[b] - lens[b])
                want[at[b]:at[b] + drop] = 0
            assert got.dtype == out_dtype and torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,heads,page", [(1, 1, 1), (7, 3, 5), (16, 8, 16), (64, 2, 24), (77, 5, 8), (100, 12, 7), (128, 8, 64), (250, 1, 3), (256, 2, 256)])
def test_sizes(dim, heads, page, dtype):
    check([9, 0, 300, 1, 65], [9, 0, 131, 1, 64], heads, dim, page, dtype, torch.int8, pad=dim % 3)
    if dtype is not torch.float32:
        check([9, 0, 300, 1, 65], [9, 0, 131, 1, 64], heads, dim, page, dtype, dtype, pad=dim % 2)


@pytest.mark.parametrize("batch", [1, 2, 33, 300])
def test_one_new_token_each(batch):
    lens = [1 + (b * 37) % 90 for b in range(batch)]
    check(lens, [1] * batch, 8, 128, 16, torch.bfloat16, torch.int8, rows=False)
    check([0] + lens, [1] * (batch + 1), 2, 32, 16, torch.bfloat16, torch.int8, rows=False)  # (a free place: its token is not written)


def test_more_new_tokens_than_a_sequence_has():
    check([3, 5], [7, 5], 2, 16, 4, torch.float32, torch.int8)


def test_many_sequences_and_many_rows():
    lens = [(b * 13) % 41 for b in range(700)]
    check(lens, lens, 3, 40, 16, torch.float16, torch.int8)


def test_rows_of_no_sequence():
    table, pages = pages_for([8, 8], 4)
    cache = marked(pages, 2, 4, 16, torch.int8)
    k, v = tokens(20, 2, 16, torch.float32, 1)
    rows, lengths = torch.tensor([3, 6, 9], **I32), torch.tensor([8, 8], **I32)
    A.kv_append(k, v, cache, table, lengths, rows=rows)
    assert int((cache.k_scale != 77).sum()) == 6 * 2 and int((cache.v_scale != 77).sum()) == 6 * 2
    back, _ = A.kv_read(cache, table, lengths, rows, 20)
    assert not back[:3].any() and not back[9:].any() and back[3:9].abs().amax((1, 2)).gt(0).sum() >= 4


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "pages"])
def test_pages_that_are_none(bad):
    table, pages = pages_for([40], 8, spare=0)
    cache = marked(pages, 1, 8, 32, torch.int8)
    table[0, 2] = pages if bad == "pages" else bad
    k, v = tokens(40, 1, 32, torch.float32, 1)
    rows, lengths = torch.tensor([0, 40], **I32), torch.tensor([40], **I32)
    A.kv_append(k, v, cache, table, lengths, rows=rows)
    assert int((cache.k_scale != 77).sum()) == 32
    back, _ = A.kv_read(cache, table, lengths, rows, 40)
    assert not back[16:24].any()


def test_lengths_past_the_table():
    table, pages = pages_for([32], 8)
    cache = marked(pages, 1, 8, 32, torch.int8)
    k, v = tokens(10, 1, 32, torch.float32, 1)
    for n in (37, 2 ** 31 - 1, -5):
        lengths, rows = torch.tensor([n], **I32), torch.tensor([0, 10], **I32)
        A.kv_append(k, v, cache, table, lengths, rows=rows)
        back, _ = A.kv_read(cache, table, lengths, rows, 10)
        assert not back[5:].any()
    assert int((cache.k_scale != 77).sum()) == 5  # (positions 27 to 31 of the first call)


def test_rows_that_are_not_finite():
    table, pages = pages_for([3], 4)
    cache = marked(pages, 1, 4, 16, torch.int8)
    k = torch.ones((3, 1, 16), device="cuda")
    k[0, 0, 3], k[1, 0, 5] = float("nan"), float("inf")
    rows, lengths = torch.tensor([0, 3], **I32), torch.tensor([3], **I32)
    A.kv_append(k, k, cache, table, lengths, rows=rows)
    s = cache.k_scale[table[0, 0].long(), 0]
    assert not s[0].isfinite() and not s[1].isfinite() and s[2] == np.float32(1) / np.float32(127)


def test_strides_and_a_cache_of_the_users_own():
    table, pages = pages_for([50], 16)
    whole = torch.full((pages, 2, 16, 48), 5, device="cuda", dtype=torch.int8)  # rows of 20 in 48
    scales = torch.full((2, pages, 2, 16), 77.0, device="cuda")
    cache = A.KVCache(whole[..., :20], whole.clone()[..., :20], scales[0], scales[1])
    x = torch.randn((20, 2, 50), device="cuda").permute(2, 1, 0)  # [50, 2, 20], the elements of a row far apart
    y = torch.randn((50, 1, 20), device="cuda").expand(50, 2, 20)  # one row for both heads
    rows, lengths = torch.tensor([0, 50], **I32), torch.tensor([50], **I32)
    wide = torch.full((1, 9), -1, **I32)
    wide[:, 2:2 + table.shape[1]] = table
    A.kv_append(x, y, cache, wide[:, 2:], lengths, rows=rows)
    assert (whole[..., 20:] == 5).all()
    k, v = A.kv_read(cache, table, lengths, rows, 50)
    for got, src in ((k, x), (v, y)):
        codes, scale = quant(src)
        assert torch.equal(got.cpu(), torch.tensor(codes.astype(np.float32) * scale[..., None]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("dim,heads", [(8, 1), (16, 1), (48, 2), (77, 3), (128, 8)])
def test_nothing_is_read_past_the_last_token(dim, heads, off, dtype):
    """Rows that would lie 2^36 bytes and more after the last token's, where no memory is."""
    x = torch.randn(heads * dim + off, device="cuda").to(dtype)[off:].as_strided((1, heads, dim), (2 ** 35, dim, 1))
    table, pages = pages_for([3], 4)
    cache = marked(pages, heads, 4, dim, torch.int8)
    lengths = torch.tensor([3], **I32)
    A.kv_append(x, x, cache, table, lengths)
    A.kv_append(x, x, cache, table, lengths, rows=torch.tensor([0, 1], **I32))
    codes, scale = quant(x[0])
    for got in A.kv_read(cache, table, lengths, None, 1):
        assert torch.equal(got[0].cpu(), torch.tensor(codes.astype(np.float32) * scale[..., None]))


def test_on_another_stream_and_in_a_graph():
    lens = [40, 17]
    table, pages = pages_for(lens, 16)
    rows, lengths = torch.tensor([0, 40, 57], **I32), torch.tensor(lens, **I32)
    k, v = tokens(57, 2, 64, torch.bfloat16, 4)
    want = marked(pages, 2, 16, 64, torch.int8)
    A.kv_append(k, v, want, table, lengths, rows=rows)
    side = torch.cuda.Stream()
    cache = marked(pages, 2, 16, 64, torch.int8)
    late = torch.zeros_like(k)
    torch.cuda._sleep(50_000_000)
    late.copy_(k)
    A.kv_append(late, v, cache, table, lengths, rows=rows, stream=side)
    back = A.kv_read(cache, table, lengths, rows, 57, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(cache, want))
    again = A.kv_read(want, table, lengths, rows, 57)
    assert all(torch.equal(a, b) for a, b in zip(back, again))
    cache = marked(pages, 2, 16, 64, torch.int8)
    one = torch.tensor([3, 1], **I32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.kv_append(k[:2], v[:2], cache, table, one)
        out = A.kv_read(cache, table, one, None, 2)
    for n in ((40, 17), (1, 16), (0, 5)):  # the lengths change between replays
        one.copy_(torch.tensor(n, **I32))
        graph.replay()
        codes, scale = quant(k[:2])
        want = torch.tensor(codes.astype(np.float32) * scale[..., None])
        want[[i for i in range(2) if n[i] == 0]] = 0
        assert torch.equal(out[0].cpu(), want)


def test_refusals():
    table, pages = pages_for([8], 4)
    cache = marked(pages, 2, 4, 16, torch.int8)
    half = marked(pages, 2, 4, 16, torch.float16)
    k, v = tokens(1, 2, 16, torch.float32, 1)
    n = torch.tensor([8], **I32)
    calls = [lambda: A.kv_append(k, v[:, :1], cache, table, n), lambda: A.kv_append(k.double(), v.double(), cache, table, n),
             lambda: A.kv_append(k, v, half, table, n), lambda: A.kv_append(k.cpu(), v.cpu(), cache, table, n),
             lambda: A.kv_append(k, v, cache, table.long(), n), lambda: A.kv_append(k, v, cache, table, n.long()),
             lambda: A.kv_append(k, v, cache, table, n[:0]), lambda: A.kv_append(k, v, cache, table, n, rows=n),
             lambda: A.kv_append(k.expand(3, 2, 16), v.expand(3, 2, 16), cache, table, n), lambda: A.kv_append(k, v, list(cache), table, n),
             lambda: A.kv_append(k, v, cache._replace(k=cache.k[..., :15]), table, n), lambda: A.kv_append(k, v, cache._replace(k_scale=None), table, n),
             lambda: A.kv_append(k, v, cache._replace(k=cache.k.transpose(1, 2)), table, n), lambda: A.kv_append(k, v, half._replace(k_scale=cache.k_scale), table, n),
             lambda: A.kv_append(k.requires_grad_(), v, cache, table, n), lambda: A.kv_append(k[:, :, :8], v[:, :, :8], cache, table, n),
             lambda: A.kv_read(cache, table, n, None, 2), lambda: A.kv_read(cache, table, n, n, -1), lambda: A.kv_read(cache, table, n, None, 1, dtype=torch.int8),
             lambda: A.kv_cache(4, 2, 4, 257), lambda: A.kv_cache(4, 2, 4, 0), lambda: A.kv_cache(4, 2, -4, 16), lambda: A.kv_cache(4, 2, 4, 16, dtype=torch.float32)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    assert (cache.k == 77).all()


@pytest.mark.parametrize("dtype,size", [(torch.int8, 80), (torch.float16, 80), (torch.float16, 8)])
def test_memory_that_ends_with_the_last_row(dtype, size):
    """Rows `size` elements apart, of which the last has nothing behind it, and what is behind the others is no number or 100."""
    dim, page, heads = size - 3, 4, 2
    table, pages = pages_for([12, 8], page, spare=0)  # (every row of every page)
    n = torch.tensor([12, 8], **I32)
    rows = pages * heads * page

    def cut_short():
        flat = torch.full(((rows - 1) * size + dim,), 100 if dtype is torch.int8 else math.nan, device="cuda", dtype=dtype)
        return flat.as_strided((pages, heads, page, dim), (heads * page * size, page * size, size, 1))

    plain = A.kv_cache(pages, heads, page, dim, dtype=dtype)
    cache = plain._replace(k=cut_short(), v=cut_short())
    if dtype is torch.int8:
        cache = cache._replace(k_scale=torch.zeros_like(plain.k_scale), v_scale=torch.zeros_like(plain.v_scale))
    k, v = tokens(20, heads, dim, torch.float16, 3)
    first = torch.tensor([0, 12, 20], **I32)
    for c in (plain, cache):
        A.kv_append(k, v, c, table, n, rows=first)
    for out in (torch.float16, torch.float32):
        got, want = A.kv_read(cache, table, n, first, 20, dtype=out), A.kv_read(plain, table, n, first, 20, dtype=out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        if dtype is torch.float16:
            assert torch.equal(got[0].half(), k) and torch.equal(got[1].half(), v)


def test_scales_that_autograd_records_are_refused():
    table, pages = pages_for([8], 4)
    plain = marked(pages, 2, 4, 16, torch.int8)
    k, v = tokens(1, 2, 16, torch.float32, 1)
    n = torch.tensor([8], **I32)
    for name in ("k_scale", "v_scale"):
        cache = plain._replace(**{name: getattr(plain, name).clone().requires_grad_()})
        for call in (lambda: A.kv_append(k, v, cache, table, n), lambda: A.kv_read(cache, table, n, None, 1), lambda: A.paged_attention(k, cache, table, n)):
            with pytest.raises(ValueError):
                call()
        with torch.no_grad():
            A.kv_append(k, v, cache, table, n)
    half = marked(pages, 2, 4, 16, torch.float16)  # (has no scales)
    A.kv_append(k.half(), v.half(), half, table, n)


def test_nothing_to_do():
    table, pages = pages_for([8], 4)
    cache = marked(pages, 2, 4, 16, torch.int8)
    none = torch.zeros((0, 2, 16), device="cuda")
    A.kv_append(none, none, cache, table[:0], torch.zeros(0, **I32))
    A.kv_append(none, none, cache, table, torch.tensor([8], **I32), rows=torch.zeros(2, **I32))
    k, v = A.kv_read(cache, table, torch.tensor([8], **I32), torch.zeros(2, **I32), 0)
    assert k.shape == v.shape == (0, 2, 16) and (cache.k == 77).all()
    empty = A.kv_cache(0, 2, 4, 16)
    one = torch.ones((1, 2, 16), device="cuda")
    A.kv_append(one, one, empty, table, torch.tensor([8], **I32))
    assert not A.kv_read(empty, table, torch.tensor([8], **I32), None, 1)[0].any()
