"""What the weights' gradient of aap_linear keeps of its terms: a result in 16 bits is the sum's own rounding, and nothing
else that is as large.

Tolerances, from the operations.  Let w be the exact sum, s the sum of its terms' sizes and v what the kernel has before it
rounds to the gradient's type.  A term's factor dy scale is rounded to 32 bits and cut to 16: 2^-15 of it at most
(2^-24 + 2^-16).  The tensor cores lose up to 2^-23 at each of the M / 8 + 8 additions of 16 products of two pieces.  So
|v - w| <= a, a = (2^-15 + (M / 8 + 8) 2^-23) s.  The rounding of v is at most as far from v as that of w is: the
result is within |round(w) - w| + 2 a of w."""
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# single tiles (few tokens, few outputs, many of both), pairs from gradients laid out first
SHAPES = [(64, 64, 40), (65, 64, 40), (300, 1100, 777), (513, 132, 2048), (3000, 128, 130), (1500, 2048, 1280), (2600, 2500, 2100)]


def layer(M, K, N, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-128, 128, (M, K), device="cuda", generator=g, dtype=torch.int8)
    scale = torch.rand(M, device="cuda", generator=g) * 0.02 + 0.001
    packed = torch.randint(0, 256, (N * K // 4,), device="cuda", generator=g, dtype=torch.uint8) & 0x55
    return codes, scale, packed, torch.full((1,), 0.037, device="cuda"), g


def check(dy, codes, scale, dw):
    M = dy.shape[0]
    f, q = dy.double() * scale.double()[:, None], codes.double()
    w, s = f.T @ q, f.abs().T @ q.abs()
    own = (w.to(dw.dtype).double() - w).abs()
    assert ((dw.double() - w).abs() <= own + 2 * (2.0 ** -15 + (M / 8 + 8) * 2.0 ** -23) * s).all()


@pytest.mark.parametrize("weights", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_terms_keep_more_than_the_result(M, K, N, dtype, weights):
    codes, scale, packed, w_scale, g = layer(M, K, N, M)
    dy = ((torch.rand((M, N), device="cuda", generator=g) + 0.5) * 0.01).to(dtype)
    for c in (codes, codes.clamp(min=1)):  # sums of terms of both signs, and of one
        check(dy, c, scale, A.aap_linear_backward(dy, c, scale, packed, w_scale, weight_dtype=weights, want=(False, True, False))[1])


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_terms_alike(M, K, N):
    """Factors of 1 + 0.9 / 256: rounded to 8 bits they would all be 1, and the sum short by 2^-8 of itself."""
    _, _, packed, w_scale, _ = layer(M, K, N, 1)
    codes, scale = torch.ones((M, K), device="cuda", dtype=torch.int8), torch.full((M,), 1 + 0.9 / 256, device="cuda")
    dy = torch.ones((M, N), device="cuda", dtype=torch.bfloat16)
    check(dy, codes, scale, A.aap_linear_backward(dy, codes, scale, packed, w_scale, weight_dtype=torch.bfloat16)[1])
