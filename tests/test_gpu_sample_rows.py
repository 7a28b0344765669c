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
