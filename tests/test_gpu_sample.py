"""sample on the GPU against its definition in 64 bits.  Tokens are equal, but where u lies next to the border between two.
A weight is off by less than 2^-28 of itself (its table, the series and the product are whole numbers of 2^-30) and by less than its unit,
2^-44; the sum of all is 1 at least, as the largest logit's is 1: borders between n tokens, as parts of the sum, are off by less than
2^-28 + n 2^-44."""
import math

import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def kept_weights(x, t, k, p, mp):
    """The weights of one row's tokens, those that do not stay with 0.  x in float64."""
    x = np.where(np.isnan(x), -np.inf, x)
    w = np.zeros(len(x))
    if not len(x) or x.max() == -np.inf:
        return w
    order = np.argsort(-x, kind="stable")
    if not t > 0:
        w[order[0]] = 1.0
        return w
    top = x[order[0]]
    with np.errstate(invalid="ignore", over="ignore"):
        each = np.where(x == top, 1.0, np.exp((x - top) / t))
    each[np.isnan(each)] = 0.0
    stay = [i for i in order if x[i] > -np.inf and (top < np.inf or x[i] == top)]
    if k > 0:
        stay = stay[:k]
    if p < 1:
        total, before, cut = math.fsum(each[stay]), 0.0, len(stay)
        for n, i in enumerate(stay):
            before += each[i]
            if before >= p * total * (1 - 1e-15):
                cut = n + 1
                break
        stay = stay[:cut]
    for i in stay:
        if x[i] == top or each[i] >= mp:
            w[i] = max(each[i], 1e-300)
    return w


def expected(x, u, t, k, p, mp):
    """(token, tokens that may be chosen as well)"""
    w = kept_weights(x, t, k, p, mp)
    if not w.any():
        return -1, {-1}
    upto = np.cumsum(w)
    pick = lambda v: int(np.argmax((upto > v * upto[-1]) & (w > 0)))  # noqa: E731
    last = int(np.nonzero(w)[0][-1])
    if not u > 0:
        return pick(0.0), {pick(0.0)}
    if u >= 1:
        return last, {last}
    near = 2.0 ** -28 + len(x) * 2.0 ** -44
    return pick(u), {pick(u), pick(max(0.0, u - near)), last if u + near >= 1 else pick(u + near)}


def column(v, n):
    return v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(n, v)


def check(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    got = A.sample(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    assert got.dtype == torch.int64 and got.shape == x.shape[:-1]
    rows = x.double().cpu().numpy().reshape(-1, x.shape[-1])
    n = len(rows)
    t, p, mp = (column(v, n).astype(np.float32).astype(np.float64) for v in (temperature, top_p, min_p))
    k = column(top_k, n)
    for r, token in enumerate(got.reshape(-1).tolist()):
        want, may = expected(rows[r], float(u.reshape(-1)[r]), t[r], int(k[r]), p[r], mp[r])
        assert token in may, (r, token, want)
    return got


def logits(rows, vocab, dtype, seed=0, size=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, vocab), device="cuda", generator=g) * size
    return x.to(dtype), torch.rand((rows,), device="cuda", generator=g)


SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=5), dict(top_k=40, temperature=1.5), dict(top_p=0.9),
            dict(top_p=0.3, temperature=0.5), dict(top_p=0.0), dict(min_p=0.05), dict(min_p=1.0), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.02),
            dict(top_k=10 ** 6, top_p=0.999), dict(temperature=100.0, top_p=0.5), dict(temperature=0.01, top_k=20)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 100, 1023, 1025, 5003])
@pytest.mark.parametrize("settings", SETTINGS)
def test_settings(settings, vocab, dtype):
    check(*logits(9, vocab, dtype, seed=vocab), **settings)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 50021), (2, 131072), (3, 2 ** 19), (300, 700)])
@pytest.mark.parametrize("settings", [dict(), dict(top_p=0.9), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.02), dict(top_k=3000), dict(temperature=50.0, top_p=0.6)])
def test_large(settings, rows, vocab, dtype):
    check(*logits(rows, vocab, dtype, seed=rows), **settings)


@pytest.mark.parametrize("settings", SETTINGS)
def test_equal_logits(settings):
    """Ties: the lower index first, at every cut."""
    g = torch.Generator(device="cuda").manual_seed(5)
    u = torch.rand((8,), device="cuda", generator=g)
    check(torch.zeros((8, 3001), device="cuda"), u, **settings)
    check(torch.randint(0, 3, (8, 3001), device="cuda", generator=g).float(), u, **settings)
    check(torch.randint(0, 40, (8, 70001), device="cuda", generator=g).bfloat16() / 4, u, **settings)
    x = torch.zeros((8, 999), device="cuda")
    x[:, ::2] = -0.0  # (equal to 0)
    check(x, u, **settings)


@pytest.mark.parametrize("settings", SETTINGS)
def test_logits_that_are_not_finite(settings):
    x, u = logits(10, 2001, torch.float32, seed=3)
    x[:, ::3] = -math.inf
    x[1, 5:300] = math.nan
    x[2] = -math.inf
    x[3] = math.nan
    x[4] = -math.inf
    x[4, 700] = -1e30
    x[5, [7, 99, 1500]] = math.inf
    x[6] = torch.finfo(torch.float32).min
    x[7] = torch.finfo(torch.float32).min
    x[7, 1234] = torch.finfo(torch.float32).max
    x[8, :1900] = -math.inf
    got = check(x, u, **settings)
    assert got[2] == got[3] == -1 and got[4] == 700


@pytest.mark.parametrize("settings", SETTINGS)
def test_numbers_at_the_ends(settings):
    x, _ = logits(8, 700, torch.float32, seed=4)
    u = torch.tensor([0.0, 1.0, -1.0, math.nan, 1 - 2.0 ** -24, 2.0 ** -24, 2.0, -0.0], device="cuda")
    check(x, u, **settings)


def test_settings_of_each_row():
    x, u = logits(64, 4001, torch.bfloat16, seed=6)
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda: torch.rand((64,), device="cuda", generator=g)  # noqa: E731
    t = torch.where(r() < 0.2, 0.0, 0.3 + r())
    t[3], t[4] = -1.0, math.nan
    k = torch.where(r() < 0.5, 0, 1 + (100 * r()).int()).int()
    k[5] = -3
    p = torch.where(r() < 0.5, 1.0, r())
    p[6], p[7] = 1.5, -0.5
    check(x, u, temperature=t, top_k=k, top_p=p, min_p=torch.where(r() < 0.5, 0.0, 0.2 * r()))
    check(x, u, temperature=t, top_p=0.8)


def test_shares():
    """200,000 numbers over four tokens: each is chosen as often as its weight says, within five standard deviations."""
    n = 200_000
    x = torch.tensor([0.1, 0.3, 0.6, 0.0], device="cuda").log().expand(n, 4).contiguous()
    got = A.sample(x, (torch.arange(n, device="cuda") + 0.5) / n)
    for token, share in enumerate((0.1, 0.3, 0.6, 0.0)):
        assert abs(int((got == token).sum()) - share * n) <= 2


def test_shapes_and_strides():
    x, u = logits(12, 999, torch.float16, seed=8)
    want = check(x, u, top_k=30)
    wide = torch.zeros((12, 2003), device="cuda", dtype=torch.float16)
    wide[:, 501:1500] = x
    assert torch.equal(check(wide[:, 501:1500], u, top_k=30), want)
    assert torch.equal(check(x.view(3, 4, 999), u.view(3, 4), top_k=30).view(-1), want)
    assert torch.equal(check(x.t().contiguous().t(), u, top_k=30), want)
    assert check(x[0], u[0], top_k=30) == want[0]
    assert torch.equal(check(x[:1].expand(12, 999), u, top_k=30)[:1], want[:1])
    assert torch.equal(check(x, u.repeat_interleave(2)[::2], top_k=30), want)
    assert A.sample(x[:0], u[:0]).shape == (0,)


def test_same_on_another_stream_and_in_a_graph():
    x, u = logits(16, 30011, torch.bfloat16, seed=9)
    want = A.sample(x, u, top_p=0.9)
    side = torch.cuda.Stream()
    late = torch.zeros_like(x)
    torch.cuda._sleep(50_000_000)
    late.copy_(x)
    again = A.sample(late, u, top_p=0.9, stream=side)
    side.synchronize()
    assert torch.equal(again, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = A.sample(late, u, top_p=0.9)
    for seed in (10, 11):
        y, v = logits(16, 30011, torch.bfloat16, seed=seed)
        late.copy_(y)
        u.copy_(v)
        graph.replay()
        assert torch.equal(out, A.sample(y, v, top_p=0.9))


def test_a_row_hangs_on_nothing_but_itself():
    x, u = logits(40, 20011, torch.float32, seed=12)
    want = A.sample(x, u, top_p=0.95, temperature=1.3)
    for b in (1, 2, 7):
        assert torch.equal(A.sample(x[:b], u[:b], top_p=0.95, temperature=1.3), want[:b])


def test_refusals():
    x, u = logits(4, 100, torch.float32)
    each = torch.ones((4,), device="cuda")
    calls = [lambda: A.sample(x.double(), u), lambda: A.sample(x.cpu(), u), lambda: A.sample(x, u[:3]), lambda: A.sample(x, u.double()),
             lambda: A.sample(x, u, temperature=each[:3]), lambda: A.sample(x, u, top_k=each), lambda: A.sample(x, u, top_p=each.double()),
             lambda: A.sample(x, u, top_k=-1), lambda: A.sample(x, u, top_k=1.5), lambda: A.sample(x.clone().requires_grad_(), u), lambda: A.sample(x, u.cpu())]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=-0.1), dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=math.inf)):
        with pytest.raises(A.AecctError):
            A.sample(x, u, **bad)
    with pytest.raises(A.AecctError):
        A.sample(x[:, :0], u)
    with pytest.raises(A.AecctError):
        A.sample(torch.zeros((1, 2 ** 19 + 1), device="cuda"), u[:1])


@pytest.mark.parametrize("vocab", [1000, 50021])
@pytest.mark.parametrize("near", [1, 3, 127, 128, 129, 300])
@pytest.mark.parametrize("p", [0.5, 0.95])
def test_a_cut_among_logits_close_to_each_other(p, near, vocab):
    """The mass is that of `near` logits 1e-6 apart, and the cut lies among them: 1e-5 at least from the next border, where 300 weights are off by
    300 2^-28 = 1.2e-6 together."""
    g = torch.Generator(device="cuda").manual_seed(near)
    x = torch.full((6, vocab), -20.0, device="cuda")
    for r in range(6):
        x[r, torch.randperm(vocab, device="cuda", generator=g)[:near]] = -1e-6 * torch.arange(near, device="cuda", dtype=torch.float32)
    x[3:] = (x[3:] * 1e4).round() / 1e4  # (ties, in the order of the row)
    u = torch.rand((6,), device="cuda", generator=g)
    check(x, u, top_p=p)
    check(x, u, top_p=p, top_k=near)
    check(x, u, top_p=p, min_p=0.5)
