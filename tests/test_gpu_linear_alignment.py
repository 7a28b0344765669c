"""aap_linear and aap_linear_backward on codes and gradients whose first row starts anywhere, at sizes of each way of
taking a product.  Tolerances are those of the tests of aligned rows."""
import pytest
from test_gpu_linear import DTYPES, check_backward, check_forward, make

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def shifted(t, at, pad=0):
    """t, `at` elements behind a 16-byte boundary and rows `pad` further apart; around it are numbers that would show."""
    rows, d = t.shape
    room = torch.full((at + rows * (d + pad) + 16,), 111 if t.dtype == torch.int8 else float("nan"), device="cuda", dtype=t.dtype)
    v = room[at:at + rows * (d + pad)].view(rows, d + pad)[:, :d]
    v.copy_(t)
    return v


@pytest.mark.parametrize("at,pad", [(1, 0), (3, 2), (4, 0), (15, 17)])
@pytest.mark.parametrize("M,K,N", [(1, 64, 40), (2, 4, 1), (4, 4096, 33), (5, 100, 70), (16, 512, 128), (70, 1028, 130), (300, 256, 300),
                                   (2300, 260, 1030), (2048, 100, 2500), (9800, 68, 300), (5000, 1100, 700)])
def test_forward(M, K, N, at, pad):
    c, s, p, w, b = make(M, K, N, 1)
    c = shifted(c, at, pad)
    check_forward(c, s, p, w, b, A.aap_linear(c, s, p, w, bias=b))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at,pad", [(1, 0), (3, 2), (8, 0), (5, 8)])
@pytest.mark.parametrize("M,K,N", [(1, 64, 40), (2, 4, 1), (33, 260, 1001), (70, 64, 96), (300, 520, 130), (1500, 2048, 1280), (2600, 1028, 264)])
def test_backward(M, K, N, at, pad, dtype):
    c, s, p, w, _ = make(M, K, N, 1)
    dy = (torch.randn((M, N), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 0.1).to(dtype)
    c, dy = shifted(c, at, pad), shifted(dy, at, pad)
    check_backward(dy, c, s, p, w, A.aap_linear_backward(dy, c, s, p, w, weight_dtype=dtype))
