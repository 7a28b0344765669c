"""paged_attention over batches of many sequences: more than 1,024 of them, whose tiles are found by whole CTAs, and many short ones, each of which
has a warp to itself; with places without a token, first positions and absent pages.  Tolerances as in test_gpu_paged_attention.py, the same
formula in 64 bits for many sequences at once."""
import math

import pytest

from paper_2410_05911_gb300 import aecct as A
from test_gpu_paged_attention import BF16, F16, F32, HALF, I8, I32, KINDS, TINY, make, with_room

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(q, cache, table, lengths, first=None):
    out, lse = A.paged_attention(q, cache, table, lengths, first=first, want_lse=True)
    pages, heads, page, dim = cache.k.shape
    batch, hq = q.shape[:2]
    scale, longest = dim ** -0.5, max(1, int(lengths.max()))
    w = 2.0 ** -11 if q.dtype is BF16 and cache.k.dtype is I8 else 2.0 ** -16 if cache.k.dtype is BF16 else 2.0 ** -22
    sums = (longest / 16 + 64) * 2.0 ** -23
    order = torch.argsort(lengths)
    some = 0
    for part in (*order[:-1].split(64), order[-1:]):  # (the longest by itself)
        if not len(part):
            continue
        n = max(1, int(lengths[part].max()))
        at = torch.arange(n, device="cuda")
        on = table[part].long()[:, at // page]
        seen = (at < lengths[part][:, None]) & (on >= 0) & (on < pages)
        if first is not None:
            seen &= at >= first[part][:, None]
        on = torch.where(seen, on, 0)

        def values(x, s):
            x = x[on, :, (at % page).expand_as(on)].double()  # [sequences, n, heads, dim]
            if s is not None:
                x = x * s[on, :, (at % page).expand_as(on)].double()[..., None]
            return torch.where(seen[..., None, None], x, 0.0)

        k, v = values(cache.k, cache.k_scale), values(cache.v, cache.v_scale)
        qs = q[part].double().unflatten(1, (heads, hq // heads))
        s = torch.einsum("bhgd,bnhd->bhgn", qs, k) * scale
        big = torch.einsum("bhgd,bnhd->bhgn", qs.abs(), k.abs()).amax(3, keepdim=True) * scale
        s = torch.where(seen[:, None, None], s, -math.inf)
        wl = torch.logsumexp(s, 3)
        p = torch.where(seen[:, None, None], torch.exp(s - torch.where(wl == -math.inf, 0.0, wl)[..., None]), 0.0)
        want, mass = torch.einsum("bhgn,bnhd->bhgd", p, v), torch.einsum("bhgn,bnhd->bhgd", p, v.abs())
        vs = torch.ones(seen.shape + (heads,), dtype=torch.float64, device="cuda") if cache.v_scale is None else cache.v_scale[on, :, (at % page).expand_as(on)].double()
        vs = torch.where(seen[..., None], vs, 1.0)
        step = 2.0 ** -39 * (p * vs.transpose(1, 2)[:, :, None]).amax(3, keepdim=True) * (v.abs() / vs[..., None]).sum(1)[:, :, None]
        e = (dim + 8) * 2.0 ** -23 * big
        tol = (2 * e + 2 * (w + 2.0 ** -22) + sums) * mass + HALF[q.dtype] * want.abs() + TINY[q.dtype]
        if cache.k.dtype is not BF16:
            tol = tol + step
        got, gl = out[part].double().unflatten(1, (heads, hq // heads)), lse[part].double().unflatten(1, (heads, hq // heads))
        off = (got - want).abs()
        assert (off <= tol).all(), (off / tol).max().item()
        empty = wl == -math.inf
        assert (gl[empty] == -math.inf).all() and not got[empty].any()
        tl = e[..., 0] + sums + 2.0 ** -21 * wl.abs()
        assert ((gl - wl).abs()[~empty] <= tl[~empty]).all()
        some += int((~empty).sum())
    assert some


def lens_of(batch, most, seed, empty=0.1):
    r = torch.Generator().manual_seed(seed)
    n = torch.randint(1, most + 1, (batch,), generator=r)
    return torch.where(torch.rand((batch,), generator=r) < empty, 0, n).tolist()


def firsts(lens, seed):
    """First positions of every kind: before the sequence, in it, at its end and past it."""
    r = torch.Generator().manual_seed(seed)
    f = (torch.rand((len(lens),), generator=r) * (torch.tensor(lens) + 8)).int() - 4
    return torch.where(torch.rand((len(lens),), generator=r) < 0.4, 0, f).int().cuda()


MANY = {
    "a run of one sequence to a lane": lens_of(1024, 60, 1),
    "one more than that": lens_of(1025, 60, 2),
    "short ones": lens_of(3000, 40, 3, empty=0.3),
    "empty runs about a long one": [0] * 900 + lens_of(50, 30, 4) + [9001] + [0] * 600 + lens_of(400, 90, 5) + [0] * 100,
    "the first alone": [700] + [0] * 2000,
    "the last alone": [0] * 2000 + [700],
    "two far apart": [0] * 5 + [333] + [0] * 1500 + [100] + [0] * 3,
}


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens", MANY.values(), ids=MANY.keys())
def test_more_than_a_thousand_sequences_dealt_out(lens, dtype, cache):
    q, c, table, lengths, _ = make(lens, 2, 4, 64, 16, dtype, cache, seed=len(lens))
    table = with_room(table, 16)
    check(q, c, table, lengths)
    check(q, c, table, lengths, first=firsts(lens, 6))


@pytest.mark.parametrize("dim,heads,group,dtype,cache", [(16, 3, 1, F32, I8), (128, 1, 17, BF16, I8), (256, 1, 3, F16, F16), (128, 2, 9, BF16, BF16)])
def test_more_than_a_thousand_sequences_of_other_heads(dim, heads, group, dtype, cache):
    lens = MANY["one more than that"] + [0] * 300 + [2000, 1, 0, 31]
    q, c, table, lengths, _ = make(lens, heads, group, dim, 8, dtype, cache, seed=dim)
    table[7, 1], table[500, 0], table[1325, 30] = -1, 2 ** 31 - 1, c.k.shape[0]
    check(q, c, with_room(table, 8), lengths, first=firsts(lens, 7))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("group", [1, 9, 16])
@pytest.mark.parametrize("dim", [16, 64, 77, 128, 256])
def test_a_warp_to_each_of_many_short_sequences(dim, group, dtype, cache):
    tile = 32 if (32 if dim <= 32 else 64 if dim <= 64 else 128 if dim <= 128 else 256) * (1 if cache is I8 else 2) <= 128 else 16
    lens = lens_of(200, 5 * tile, dim + group)
    lens[:3] = [0, 5 * tile, 1]
    q, c, table, lengths, _ = make(lens, 2, group, dim, 16, dtype, cache, seed=dim + group)
    table[1, 1], table[4, 0], table[9, :] = -1, 2 ** 31 - 1, c.k.shape[0]
    check(q, c, table, lengths)
    check(q, c, table, lengths, first=firsts(lens, 8))


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_a_warp_to_each_of_many_sequences_of_up_to_16_tiles(dtype, cache):
    tile = 32 if cache is I8 else 16
    lens = lens_of(1300, 15 * tile, 9)
    check(*make(lens, 2, 2, 128, 16, dtype, cache, seed=9)[:4], first=firsts(lens, 9))
