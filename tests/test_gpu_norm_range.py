"""rms_quant_backward on rows far from unit size: r^3 of them is no 32-bit number, the gradient is.

Tolerances as in the tests of rows near unit size (u = 2^-24): each of the two terms within 64 u of its size, dgain within
(rows + 64) u of its terms' sizes, and one rounding to 16 bits."""
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
WIDTHS = [46, 128, 257, 1001, 4096, 8191, 16384, 32768]  # groups of lanes, rows in shared memory (odd ones too), rows in registers


def formula(dy, h, gain, eps):
    dy, h, gain = dy.double(), h.double(), gain.double()
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    t, u = dy * gain, h * r
    dx = r * (t - u * (t * u).mean(1, keepdim=True))
    size = r * (t.abs() + u.abs() * (t * u).abs().mean(1, keepdim=True))
    return dx, size, dy * u


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e16, 1e13, 1e-13, 1e-16])
@pytest.mark.parametrize("d", WIDTHS)
def test_large_and_small_rows(d, size, dtype):
    g = torch.Generator(device="cuda").manual_seed(d)
    rows = 37
    # (a term of its own along the row: without it the second term would be no more than rounding in a wide row)
    h = (torch.randn((rows, d), device="cuda", generator=g) * size).to(dtype)
    dy = (torch.randn((rows, d), device="cuda", generator=g) + 2 * h.float() / size).mul(0.1).to(dtype)
    gain = 1.0 + 0.3 * torch.randn((d,), device="cuda", generator=g)
    dx, dgain = A.rms_quant_backward(dy, h, gain, eps=0.0)
    want, terms, p = formula(dy, h, gain, 0.0)
    assert ((dx.double() - want).abs() <= 64 * U * terms + ROUND[dtype] * want.abs()).all()
    assert ((dgain.double() - p.sum(0)).abs() <= (rows + 64) * U * p.abs().sum(0)).all()


@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_zeros_and_a_tiny_eps(d):
    """dx is r dy gain there, r = 1 / sqrt(eps)."""
    dy = torch.randn((3, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(d))
    gain, eps = torch.full((d,), 1.5, device="cuda"), float(torch.tensor(1e-30))
    dx, dgain = A.rms_quant_backward(dy, torch.zeros_like(dy), gain, eps=eps)
    want = dy.double() * 1.5 * eps ** -0.5
    assert ((dx.double() - want).abs() <= 64 * U * want.abs()).all() and not dgain.any()
