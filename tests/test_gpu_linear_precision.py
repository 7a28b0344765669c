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

# single tiles (few tokens, few outputs, many of both), pairs from gradients laid out first, few of them in parts
SHAPES = [(64, 64, 40), (65, 64, 40), (300, 1100, 777), (513, 132, 2048), (3000, 128, 130), (1500, 2048, 1280), (2600, 2500, 2100),
          (14000, 388, 261)]


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


# The longest sums, of one sign: a part of at most 1,024 additions (8,192 for bfloat16) loses 2^-23 of itself at each, however
# long the whole is, and up to 64 parts are added with 2^-24 each.
LONG = {torch.float16: 2.0 ** -13 + 64 * 2.0 ** -24, torch.bfloat16: 2.0 ** -10 + 64 * 2.0 ** -24}


def check_long(got, w, factor):
    own = (w.to(got.dtype).double() - w).abs()
    assert ((got.double() - w).abs() <= own + 2 * (LONG[got.dtype] + factor) * w).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_sums_over_many_tokens(dtype):
    M, K, N = 262149, 1536, 1792
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = (torch.rand((M, N), device="cuda", generator=g) + 0.5).to(dtype)
    q = torch.randint(1, 128, (K,), device="cuda", generator=g, dtype=torch.int8)
    codes, scale = q.repeat(M, 1), torch.full((M,), 1.1e-3, device="cuda")
    packed, w_scale = torch.zeros(N * K // 4, device="cuda", dtype=torch.uint8), torch.ones(1, device="cuda")
    dw = A.aap_linear_backward(dy, codes, scale, packed, w_scale, weight_dtype=dtype, want=(False, True, False))[1]
    sums = sum(part.double().sum(0) for part in dy.split(1 << 14)) * scale[0].double()
    check_long(dw, sums[:, None] * q.double(), 2.0 ** -15)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_sums_over_many_outputs(dtype):
    M, K, N = 1536, 1792, 262144
    dy = (torch.rand((M, N), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) + 0.5).to(dtype)
    codes, scale = torch.zeros((M, K), device="cuda", dtype=torch.int8), torch.ones(M, device="cuda")
    packed, w_scale = torch.full((N * K // 4,), 0x55, device="cuda", dtype=torch.uint8), torch.full((1,), 0.037, device="cuda")
    dx = A.aap_linear_backward(dy, codes, scale, packed, w_scale, want=(True, False, False))[0]
    sums = torch.stack([row.double().sum() for row in dy]) * w_scale.double()
    check_long(dx, sums[:, None].expand(M, K), 0.0)
