"""sample on rows that are hard to weigh or to divide: against its definition in 64 bits, as in test_gpu_sample.py.  Borders between n tokens, as
parts of the sum, are off by less than near(n) = 2^-28 + n 2^-44 (a weight by 2^-28 of itself and 2^-44 of the largest)."""
import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def near(n):
    return 2.0 ** -28 + n * 2.0 ** -44


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n", [4001, 100_001])
def test_borders_between_small_logits_under_a_large_one(n, dtype):
    """Logits of 3 2^-24 in one half of the row and of minus that in the other, under one of 8: the differences are whole and equal in 24 bits, which
    moves the borders in the middle by 2^-23.4 of the sum."""
    x = torch.full((n,), 3 * 2.0 ** -24, device="cuda")
    x[n // 2:] *= -1
    x[50] = 8.0
    x = x.to(dtype)
    w = np.exp(x.double().cpu().numpy() - 8.0)
    upto = np.cumsum(w) / w.sum()
    borders = upto[n // 2 - 40:n // 2 + 40]
    u = (borders[:, None] + np.linspace(-1, 1, 9) * 2.0 ** -23).astype(np.float32).reshape(-1)
    far = np.abs(u.astype(np.float64) - np.repeat(borders, 9)) > near(n)
    assert 300 < far.sum()
    got = A.sample(x.expand(len(u), n), torch.tensor(u).cuda()).cpu().numpy()
    want = np.searchsorted(upto, u.astype(np.float64), side="right")
    assert (got == want)[far].all(), int((got != want)[far].sum())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab,many", [(4001, 3000), (50_021, 20_000), (2 ** 19, 2 ** 19)])
def test_many_logits_of_plus_infinity(vocab, many, dtype):
    """They share the row equally: what stays of them are the first, and u counts them."""
    g = torch.Generator(device="cuda").manual_seed(many)
    x = torch.randn((vocab,), device="cuda", generator=g)
    at = torch.randperm(vocab, device="cuda", generator=g)[:many].sort().values
    x[at] = float("inf")
    u = ((torch.arange(64, device="cuda", dtype=torch.float64) + 0.5) / 64).float()  # (whole sixty-fourths of a half: exact)
    rows = x.to(dtype).expand(64, vocab)
    for settings, stay in ((dict(), many), (dict(top_p=0.5), -(-many // 2)), (dict(top_k=7), 7), (dict(min_p=0.9), many), (dict(top_k=many - 1, top_p=0.25), -(-(many - 1) // 4)),
                           (dict(temperature=50.0), many), (dict(temperature=0.0), 1)):
        want = at[(u.double() * stay).long()]  # the lowest with (rank + 1) > u stay
        assert torch.equal(A.sample(rows, u, **settings), want), settings


def kept(x, t, k, p, mp):
    """The weights of a row's tokens in 64 bits, those that do not stay with 0 (test_gpu_sample.py's kept_weights without its loops)."""
    x = np.where(np.isnan(x), -np.inf, x)
    w = np.zeros(len(x))
    top = x.max()
    if top == -np.inf:
        return w
    order = np.argsort(-x, kind="stable")
    if not t > 0:
        w[order[0]] = 1.0
        return w
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        each = np.where(x == top, 1.0, np.exp((x - top) / t))
    stay = order[(x[order] > -np.inf) & ((top < np.inf) | (x[order] == top))]
    stay = stay[:k] if k > 0 else stay
    if p < 1:
        upto = np.cumsum(each[stay].astype(np.longdouble))
        stay = stay[:int(np.searchsorted(upto, p * upto[-1])) + 1]
    stay = stay[(x[stay] == top) | (each[stay] >= mp)]
    w[stay] = np.maximum(each[stay], 1e-300)
    return w


def tokens(x, u, t, k, p, mp):
    """The token that the definition takes, and those that it would take with u or p off by near(n)."""
    may = []
    for q in {p, p * (1 - near(len(x))), p * (1 + near(len(x)))}:
        w = kept(x, t, k, q, mp)
        if not w.any():
            return {-1}
        upto = np.cumsum(w)
        last = int(np.nonzero(w)[0][-1])
        pick = lambda v: int(np.argmax((upto > v * upto[-1]) & (w > 0))) if v < 1 else last  # noqa: B023, E731
        if not u > 0:
            may += [pick(0.0)]
        elif u >= 1:
            may += [last]
        else:
            may += [pick(u), pick(max(0.0, u - near(len(x)))), pick(u + near(len(x)))]
    return set(may)


NOT_FINITE = [dict(), dict(temperature=0.0), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.02), dict(top_p=0.9), dict(top_k=3000), dict(min_p=0.05),
              dict(temperature=50.0, top_p=0.6)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [4095, 4096, 4097, 8191, 16_384, 50_021, 131_072])
def test_logits_that_are_not_finite_in_rows_of_several_ctas(vocab, dtype):
    """What is a number lies in the parts of some CTAs of a row only, or nowhere."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    inf = float("inf")
    x = rand(11, vocab) * 3
    x[0, ::3] = -inf
    x[1] = -inf
    x[2] = float("nan")
    x[3, :vocab - vocab // 8] = -inf
    x[4, 11:] = -inf
    x[5] = -inf
    x[5, vocab // 2] = -6e4
    x[6, [vocab - 1, vocab - 2, vocab - vocab // 8]] = inf
    x[7, torch.rand((vocab,), device="cuda", generator=g) < 0.5] = float("nan")
    x[8], x[8, vocab // 2:vocab // 2 + vocab // 4] = -inf, 1.5
    x[9, :vocab // 2], x[9, vocab // 2:] = float("nan"), -inf
    x[10], x[10, 0] = -inf, inf
    x = x.to(dtype)
    rows = x.double().cpu().numpy()
    for i, settings in enumerate(NOT_FINITE):
        u = torch.rand((11,), device="cuda", generator=g)
        u[i] = (0.0, 1.0, 1 - 2.0 ** -24, -1.0, 2.0 ** -24, 2.0, 0.5)[i]
        got = A.sample(x, u, **settings).tolist()
        s = dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **settings)
        t, p, mp = (float(np.float32(s[n])) for n in ("temperature", "top_p", "min_p"))
        for r, token in enumerate(got):
            assert token in tokens(rows[r], float(u[r]), t, s["top_k"], p, mp), (r, settings, token)
        assert got[1] == got[2] == got[9] == -1 and got[5] == vocab // 2 and got[10] == 0


def test_the_largest_logits_stay_whatever_min_p_is():
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randint(0, 9, (8, 5000), device="cuda", generator=g).float()
    u = torch.rand((8,), device="cuda", generator=g)
    for kw in (dict(), dict(top_p=0.01), dict(top_k=300), dict(top_k=300, top_p=0.01)):
        want = A.sample(x, u, min_p=1.0, **kw)
        assert torch.equal(A.sample(x, u, min_p=1.5, **kw), want) and torch.equal(A.sample(x, u, min_p=3e38, **kw), want)
        assert (x[torch.arange(8), want] == 8).all()
