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
