"""The AAP linear layer's ways of splitting its products, at the sizes where one takes over from another: a few
tokens in integers, single tiles and pairs of them, parts of long 32-bit sums, operands laid out first."""
import pytest
import torch

from paper_2410_05911_gb300 import aecct

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -23


def generator(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def random_layer(M, K, N, gen, ldc=None, offset=0):
    """Codes of rows ldc apart, 2-bit weights of any fields (10 among them) `offset` bytes into an allocation."""
    ldc = K if ldc is None else ldc
    codes = torch.randint(-128, 128, (M, ldc), device="cuda", dtype=torch.int8, generator=gen)[:, :K]
    scale = torch.rand(M, device="cuda", generator=gen) * 0.02 + 0.001
    room = torch.randint(0, 256, (N * K // 4 + offset,), device="cuda", dtype=torch.uint8, generator=gen)
    packed = room[offset:]
    w_scale = torch.full((1,), 0.037, device="cuda")
    fields = torch.stack([(packed >> s) & 3 for s in (0, 2, 4, 6)], -1).reshape(N, K)
    t = (fields & 1).double() * (1 - (fields & 2).double())
    return codes, scale, packed, w_scale, t


def forward64(codes, scale, w_scale, t, bias):
    """The integer sum is exact in float64; the kernels' factor scale * w_scale is one float32 product."""
    y = (codes.double() @ t.T) * (scale * w_scale).double()[:, None]
    return y if bias is None else y + bias.double()


@pytest.mark.parametrize("K,N", [(4, 1), (36, 7), (128, 512), (1100, 77), (2048, 33), (4096, 130), (20480, 9), (65536, 5)])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 16, 17])
def test_few_tokens(M, K, N):
    """One rounding after an exact sum: within 2^-23 of the largest of its two terms and itself."""
    gen = generator(M * 7 + K)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen)
    bias = torch.randn(N, device="cuda", generator=gen)
    y = aecct.aap_linear(codes, scale, packed, w_scale, bias=bias)
    ref = forward64(codes, scale, w_scale, t, bias)
    assert ((y.double() - ref).abs() <= U32 * ref.abs()).all()


@pytest.mark.parametrize("M", [1, 3, 4])
@pytest.mark.parametrize("K,N,ldc,offset", [(256, 40, 272, 0), (256, 40, 257, 4), (64, 33, 64, 1), (100, 31, 103, 3), (4096, 18, 4099, 2)])
def test_few_tokens_of_any_alignment(M, K, N, ldc, offset):
    gen = generator(K + offset)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen, ldc, offset)
    y = aecct.aap_linear(codes, scale, packed, w_scale)
    ref = forward64(codes, scale, w_scale, t, None)
    assert ((y.double() - ref).abs() <= U32 * ref.abs()).all()


@pytest.mark.parametrize("M,K,N", [(2048, 100, 2500), (4096, 132, 1500), (2304, 64, 1024), (2300, 260, 1030)])
def test_forward_in_pairs(M, K, N):
    """Tiles of pairs, with codes laid out first (1,536 columns and more) and without."""
    gen = generator(M)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen, K + 3)
    bias = torch.randn(N, device="cuda", generator=gen)
    y = aecct.aap_linear(codes, scale, packed, w_scale, bias=bias)
    ref = forward64(codes, scale, w_scale, t, bias)
    assert ((y.double() - ref).abs() <= U32 * ref.abs()).all()


# Sums of 32-bit gradients: a part of at most 28 additions on the tensor cores, each of which loses up to 2^-23 of what is
# there, and a rounded addition a chunk and a split (at most 40 here, half as much each): 48 in all, where all terms have one
# sign.  dW's operand is rounded once more when it is scaled: 49.
LONG = 49 * U32
LONG_SHAPES = [
    (10240, 128, 1500),  # dX: more tiles than SMs, more than one chunk of 20 steps of 64
    (30000, 128, 512),   # dW: split among the SMs, more than one chunk each
    (1500, 2048, 1280),  # dW in pairs
    (1280, 2048, 1500),  # dX in pairs
    (64, 64, 2000), (2000, 64, 64),
]


@pytest.mark.parametrize("M,K,N", LONG_SHAPES)
@pytest.mark.parametrize("sign", ["one", "both"])
def test_long_sums_of_32_bit_gradients(M, K, N, sign):
    gen = generator(N)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen)
    dy = torch.rand((M, N), device="cuda", generator=gen) + 0.25
    if sign == "one":
        codes, packed = codes.abs().clamp(min=1), torch.full_like(packed, 0x55)
        t = torch.ones_like(t)
    else:
        dy = dy * torch.randn((M, N), device="cuda", generator=gen)
    dx, dw, db = aecct.aap_linear_backward(dy, codes, scale, packed, w_scale)
    d64, q64 = dy.double(), codes.double() * scale.double()[:, None]
    for got, ref, size in [(dx, d64 @ t * w_scale.double(), d64.abs() @ t.abs() * w_scale.double()),
                           (dw, d64.T @ q64, d64.abs().T @ q64.abs())]:
        assert ((got.double() - ref).abs() <= LONG * size).all()
    assert ((db.double() - d64.sum(0)).abs() <= 1e-5 * d64.abs().sum(0)).all()


@pytest.mark.parametrize("dtype,unit", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
@pytest.mark.parametrize("M,K,N,ld", [(33, 260, 1001, 1001), (5, 132, 77, 80), (300, 520, 130, 133), (1, 256, 4095, 4095), (2500, 2048, 201, 203)])
def test_input_gradient_of_unaligned_rows(dtype, unit, M, K, N, ld):
    """16-bit gradients take part as they are: the sum's N additions lose up to 2^-23 each, and one rounding to 16 bits."""
    gen = generator(N)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen)
    dy = torch.randn((M, ld), device="cuda", generator=gen).to(dtype)[:, :N]
    dx, _, db = aecct.aap_linear_backward(dy, codes, scale, packed, w_scale, want=(True, False, True))
    d64 = dy.double()
    ref, size = d64 @ t * w_scale.double(), d64.abs() @ t.abs() * w_scale.double()
    assert ((dx.double() - ref).abs() <= unit * ref.abs() + (N + 4) * U32 * size + 2.0 ** -25).all()
    assert ((db.double() - d64.sum(0)).abs() <= (M + 4) * U32 * d64.abs().sum(0)).all()


def test_first_call_under_capture_and_on_another_stream():
    """A captured call replays with new inputs in the same tensors."""
    gen = generator(9)
    codes, scale, packed, w_scale, t = random_layer(300, 256, 200, gen)
    dy = torch.randn((300, 200), device="cuda", generator=gen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = aecct.aap_linear(codes, scale, packed, w_scale)
        few = aecct.aap_linear(codes[:2], scale[:2], packed, w_scale)
        dx, dw, db = aecct.aap_linear_backward(dy, codes, scale, packed, w_scale)
    for _ in range(2):
        codes.copy_(torch.randint(-127, 128, codes.shape, device="cuda", dtype=torch.int8, generator=gen))
        dy.normal_(generator=gen)
        graph.replay()
        assert torch.equal(y, aecct.aap_linear(codes, scale, packed, w_scale))
        assert torch.equal(few, y[:2])
        for got, ref in zip((dx, dw, db), aecct.aap_linear_backward(dy, codes, scale, packed, w_scale)):
            assert torch.equal(got, ref)


@pytest.mark.parametrize("M,K,N", [(9000, 388, 261), (9000, 516, 264), (200, 4100, 2100), (260, 2052, 4097)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_in_pairs_of_few_tiles(dtype, M, K, N):
    """Long products of few tiles are split among pairs.  In 32 bits within LONG as above; with 16-bit gradients each
    factor dy scale of dW is rounded to 8 bits, and R additions lose up to 2^-23 each."""
    gen = generator(M + K)
    codes, scale, packed, w_scale, t = random_layer(M, K, N, gen, K + 1)
    dy = torch.randn((M, N), device="cuda", generator=gen).to(dtype)
    dx, dw, db = aecct.aap_linear_backward(dy, codes, scale, packed, w_scale, weight_dtype=dtype)
    d64, q64 = dy.double(), codes.double() * scale.double()[:, None]
    half = dtype == torch.bfloat16
    for got, ref, size, R, factor in [(dx, d64 @ t * w_scale.double(), d64.abs() @ t.abs() * w_scale.double(), N, 0.0),
                                      (dw, d64.T @ q64, d64.abs().T @ q64.abs(), M, 2.0 ** -8)]:
        bound = (factor + (R + 4) * U32) * size + 2.0 ** -8 * ref.abs() if half else LONG * size
        assert ((got.double() - ref).abs() <= bound).all()
    assert ((db.double() - d64.sum(0)).abs() <= 1e-5 * d64.abs().sum(0)).all()
