"""aap_linear and aap_linear_backward on the GPU against their formulas in 64 bits.

Tolerances, from the operations (u = 2^-24).  Forward: the sum of integers is exact, scale w_scale, its
product with the sum and the bias are three roundings.  Backward: the tensor cores add R products in 32 bits, in
an order and with a rounding of their own: within R 2^-23 of the sum of the products' sizes, and, as
partial sums of products of either sign are on the whole no larger than the whole sum, within S 2^-23 of the
result in the 2-norm, S = 3 R / 16 + 8 the accumulations (up to three pieces of a factor, 16 products at
a time).  A weight gradient's factor dy scale is rounded to 8, 16 or 24 bits with its type.  The bias's
gradient adds M terms: M u.  A result in 16 bits is rounded once more."""
import ctypes

import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
FACTOR = {torch.float32: 2.0 ** -23, torch.float16: 2.0 ** -16, torch.bfloat16: 2.0 ** -9}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
SIZES = [(1, 4, 1), (1, 64, 1), (2, 128, 3), (1, 4096, 1030), (3, 8192, 40), (5, 36, 17), (7, 64, 640), (8, 256, 256), (9, 100, 33),
         (16, 512, 128), (17, 4100, 65), (37, 1024, 1030), (46, 32, 128), (64, 128, 512), (90, 128, 384), (127, 64, 129),
         (128, 128, 128), (129, 132, 257), (300, 1100, 777), (257, 320, 512), (1000, 2052, 96), (513, 512, 2048), (2500, 128, 130),
         (40, 16384, 20)]


def unpack(packed, K):
    f = (packed.reshape(-1, 1) >> torch.tensor([0, 2, 4, 6], device=packed.device, dtype=torch.uint8)) & 3
    return torch.where(f == 3, -1.0, torch.where(f == 1, 1.0, 0.0)).double().view(-1, K)


def make(M, K, N, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-127, 128, (M, K + pad), device="cuda", generator=g, dtype=torch.int8)[:, :K]
    scale = torch.exp(torch.randn(M, device="cuda", generator=g)) * 0.02
    b = torch.randint(0, 256, (N * K // 4,), device="cuda", generator=g, dtype=torch.uint8)
    packed = b & (((b << 1) & 0xAA) | 0x55)
    return codes, scale, packed, torch.full((1,), 0.037, device="cuda"), torch.randn(N, device="cuda", generator=g)


def check_forward(codes, scale, packed, ws, bias, y):
    acc = codes.double() @ unpack(packed, codes.shape[1]).T
    p = acc * scale.double()[:, None] * ws.double()
    want = p if bias is None else p + bias.double()
    assert ((y.double() - want).abs() <= 3 * U * p.abs() + (U + ROUND[y.dtype]) * want.abs() + TINY[y.dtype]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(M, K, N, dtype):
    c, s, p, w, b = make(M, K, N, M + K + N)
    check_forward(c, s, p, w, b, A.aap_linear(c, s, p, w, bias=b, dtype=dtype))
    check_forward(c, s, p, w, None, A.aap_linear(c, s, p, w, dtype=dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 30, 200])
@pytest.mark.parametrize("K,pad,at", [(64, 1, 0), (64, 16, 1), (256, 8, 4), (100, 3, 7), (1024, 16, 16), (512, 4, 2)])
def test_forward_of_rows_and_weights_that_start_anywhere(M, K, pad, at):
    N = 200
    c, s, p, w, b = make(M, K, N, 5, pad=pad)
    buf = torch.zeros(p.numel() + 32, dtype=torch.uint8, device="cuda")
    buf[at:at + p.numel()] = p
    q = buf[at:at + p.numel()]
    check_forward(c, s, q, w, b, A.aap_linear(c, s, q, w, bias=b))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 20, 150])
def test_largest_sums_are_exact(M):
    K, N = 65536, 9
    for code, byte in ((127, 0x55), (-128, 0xFF), (127, 0xFF)):
        c = torch.full((M, K), code, dtype=torch.int8, device="cuda")
        c[0, 5] = 3
        p = torch.full((N * K // 4,), byte, dtype=torch.uint8, device="cuda")
        one = torch.ones(1, device="cuda")
        y = A.aap_linear(c, torch.ones(M, device="cuda"), p, one)
        assert torch.equal(y.double(), c.double() @ unpack(p, K).T)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 40, 300])
def test_the_code_that_stands_for_nothing_is_zero(M):
    c, s, p, w, b = make(M, 128, 33, 1)
    q = p | 0xAA  # 00 -> 10, 01 -> 11
    r = torch.where(torch.zeros_like(p).bool(), p, q)
    check_forward(c, s, r, w, b, A.aap_linear(c, s, r, w, bias=b))
    dy = torch.randn((M, 33), device="cuda")
    check_backward(dy, c, s, r, w, A.aap_linear_backward(dy, c, s, r, w))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [4, 60, 260])
def test_a_scale_that_is_not_finite_stays_in_its_row(M):
    c, s, p, w, b = make(M, 256, 130, 1)
    want = A.aap_linear(c, s, p, w, bias=b)
    s2 = s.clone()
    s2[1] = float("nan")
    got = A.aap_linear(c, s2, p, w, bias=b)
    assert got[1].isnan().all()
    got[1] = want[1]
    assert torch.equal(got, want)


def check_backward(dy, codes, scale, packed, ws, out):
    dx, dw, db = out
    T, d = unpack(packed, codes.shape[1]), dy.double()
    M, N = d.shape
    q = codes.double()
    if dx is not None:
        want, size = (d @ T) * ws.double(), (d.abs() @ T.abs()) * ws.double()
        err = (dx.double() - want).abs()
        assert dx.dtype == dy.dtype
        assert (err <= (N * 2.0 ** -23 + 2 * U) * size + ROUND[dx.dtype] * want.abs() + TINY[dx.dtype]).all()
        assert err.norm() <= ((3 * N / 16 + 8) * 2.0 ** -23 + ROUND[dx.dtype]) * want.norm() + TINY[dx.dtype] * dx.numel() ** 0.5
    if dw is not None:
        f = d * scale.double()[:, None]
        want, size = f.T @ q, f.abs().T @ q.abs()
        err = (dw.double() - want).abs()
        assert (err <= (M * 2.0 ** -23 + FACTOR[dw.dtype]) * size + ROUND[dw.dtype] * want.abs() + TINY[dw.dtype]).all()
        assert err.norm() <= ((3 * M / 16 + 8) * 2.0 ** -23 + 1.5 * FACTOR[dw.dtype] + ROUND[dw.dtype]) * want.norm() + \
            TINY[dw.dtype] * dw.numel() ** 0.5
    if db is not None:
        assert ((db.double() - d.sum(0)).abs() <= (M + 1) * U * d.abs().sum(0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weights", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                           (torch.float16, torch.float16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_backward(M, K, N, dtype, weights):
    c, s, p, w, _ = make(M, K, N, M + K + N)
    dy = (torch.randn((M, N), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 0.1).to(dtype)
    check_backward(dy, c, s, p, w, A.aap_linear_backward(dy, c, s, p, w, weight_dtype=weights))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,pad", [(70, 64, 96, 8), (70, 64, 96, 1), (33, 100, 77, 3), (300, 256, 256, 64)])
def test_backward_of_rows_that_lie_apart(M, K, N, pad, dtype):
    c, s, p, w, _ = make(M, K, N, 1, pad=16 * pad)
    dy = torch.randn((M, N + pad), device="cuda").to(dtype)[:, :N]
    check_backward(dy, c, s, p, w, A.aap_linear_backward(dy, c, s, p, w))


@pytest.mark.gpu
def test_each_gradient_alone():
    c, s, p, w, _ = make(50, 128, 64, 1)
    dy = torch.randn((50, 64), device="cuda")
    every = A.aap_linear_backward(dy, c, s, p, w)
    for i in range(3):
        want = tuple(j == i for j in range(3))
        got = A.aap_linear_backward(dy, c, s, p, w, want=want)
        for j in range(3):
            assert (got[j] is None) == (j != i) and (j != i or torch.equal(got[j], every[j]))


@pytest.mark.gpu
def test_backward_against_differences():
    # y is linear in the activations and in the weights: a difference is exact but for rounding in 64 bits
    M, K, N = 5, 16, 7
    c, s, p, w, _ = make(M, K, N, 3)
    dy = torch.randn((M, N), device="cuda")
    dx, dw, db = A.aap_linear_backward(dy, c, s, p, w)
    x, W, d = c.double() * s.double()[:, None], unpack(p, K) * w.double(), dy.double()

    def loss(x, W, b):
        return ((x @ W.T + b) * d).sum()

    zero = torch.zeros(N, dtype=torch.float64, device="cuda")
    for a, grad, at in ((x, dx, 0), (W, dw, 1), (zero, db, 2)):
        for i in range(0, a.numel(), 3):
            e = torch.zeros_like(a)
            e.view(-1)[i] = 0.5
            up, down = [x, W, zero], [x, W, zero]
            up[at], down[at] = a + e, a - e
            num = (loss(*up) - loss(*down)).item()
            assert abs(num - grad.view(-1)[i].item()) <= 1e-5 * max(1.0, abs(num))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(20, 64, 40), (300, 256, 300)])
def test_a_gradient_that_is_not_finite_reaches_its_row_and_column_only(M, K, N, dtype):
    c, s, p, w, _ = make(M, K, N, 1)
    dy = torch.randn((M, N), device="cuda").to(dtype)
    want = A.aap_linear_backward(dy, c, s, p, w)
    bad = dy.clone()
    bad[3, 5], bad[7, 9] = float("inf"), float("nan")
    dx, dw, db = A.aap_linear_backward(bad, c, s, p, w)
    assert not dx[3].isfinite().all() and dx[7].isnan().all() and dw[9].isnan().all() and not dw[5].isfinite().all()
    assert db[5] == float("inf") and db[9].isnan()
    t = unpack(p, K)[5]
    assert torch.equal(dx[3][t != 0].double(), (t * float("inf"))[t != 0])  # (0 inf is not a number)
    dx[[3, 7]], dw[[5, 9]], db[[5, 9]] = want[0][[3, 7]], want[1][[5, 9]], want[2][[5, 9]]
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want))


@pytest.mark.gpu
def test_no_tokens_no_outputs_and_more_dimensions():
    c, s, p, w, b = make(12, 64, 10, 1)
    assert A.aap_linear(c[:0], s[:0], p, w).shape == (0, 10)
    assert A.aap_linear(c, s, p[:0], w).shape == (12, 0)
    dx, dw, db = A.aap_linear_backward(torch.zeros((0, 10), device="cuda"), c[:0], s[:0], p, w)
    assert dx.shape == (0, 64) and dw.shape == (10, 64) and not dw.any() and not db.any()
    dx, dw, db = A.aap_linear_backward(torch.zeros((12, 0), device="cuda"), c, s, p[:0], w)
    assert dx.shape == (12, 64) and not dx.any() and dw.shape == (0, 64) and db.shape == (0,)
    y = A.aap_linear(c.view(3, 4, 64), s.view(3, 4), p, w, bias=b)
    assert torch.equal(y.view(12, 10), A.aap_linear(c, s, p, w, bias=b))
    one = A.aap_linear(c[0], s[0], p, w)
    assert one.shape == (10,)
    dy = torch.randn((3, 4, 10), device="cuda")
    check_backward(dy.view(12, 10), c, s, p, w, [t.view(-1, t.shape[-1]) if t.dim() > 1 else t
                                                 for t in A.aap_linear_backward(dy, c.view(3, 4, 64), s.view(3, 4), p, w)])


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1, 4096, 512), (37, 4096, 512), (700, 512, 1024)])
def test_same_bits_on_every_run_and_on_another_stream(M, K, N):
    c, s, p, w, b = make(M, K, N, 1)
    dy = torch.randn((M, N), device="cuda")
    want = (A.aap_linear(c, s, p, w, bias=b),) + A.aap_linear_backward(dy, c, s, p, w)
    side = torch.cuda.Stream()
    late = torch.zeros_like(c), torch.zeros_like(dy)
    torch.cuda._sleep(50_000_000)
    late[0].copy_(c), late[1].copy_(dy)
    got = (A.aap_linear(late[0], s, p, w, bias=b, stream=side),) + A.aap_linear_backward(late[1], late[0], s, p, w, stream=side)
    del late
    other = torch.full_like(c, 7), torch.full_like(dy, 7.0)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and bool((other[0] == 7).all()) and bool((other[1] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 8, 9, 64, 65, 500])
def test_a_row_does_not_depend_on_the_others(M):
    c, s, p, w, b = make(M, 1024, 300, 1)
    one = A.aap_linear(c[M // 2:M // 2 + 1], s[M // 2:M // 2 + 1], p, w, bias=b)
    assert torch.equal(A.aap_linear(c, s, p, w, bias=b)[M // 2:M // 2 + 1], one)


@pytest.mark.gpu
def test_refusals():
    c, s, p, w, b = make(4, 64, 8, 1)
    for bad in (dict(codes=c.short()), dict(codes=c.cpu()), dict(scale=s[:3]), dict(scale=s.half()), dict(packed=p.int()),
                dict(packed=p[:-1]), dict(codes=c[:, :62]), dict(w_scale=s), dict(w_scale=w.double()), dict(bias=b[:7]),
                dict(bias=b.half()), dict(dtype=torch.int8)):
        with pytest.raises(ValueError):
            A.aap_linear(**{"codes": c, "scale": s, "packed": p, "w_scale": w, **bad})
    dy = torch.zeros((4, 8), device="cuda")
    for bad in (dict(dy=dy.double()), dict(dy=dy[:3]), dict(dy=dy[:, :7]), dict(weight_dtype=torch.float64)):
        with pytest.raises(ValueError):
            A.aap_linear_backward(**{"dy": dy, "codes": c, "scale": s, "packed": p, "w_scale": w, **bad})
    wide = torch.zeros((1, 65540), dtype=torch.int8, device="cuda")
    with pytest.raises(A.AecctError) as e:
        A.aap_linear(wide, s[:1], torch.zeros(65540 // 4, dtype=torch.uint8, device="cuda"), w)
    assert e.value.status == A.AECCT_ERR_UNSUPPORTED


def test_c_entries_refuse_before_any_device_work():
    L, P, BAD = A.load(), 0x1000, A.AECCT_ERR_INVALID_ARG
    f = lambda **k: L.aecct_aap_linear(*{**dict(q=P, ldc=8, s=P, p=P, w=P, b=None, M=1, K=8, N=3, t=0, y=P, ws=P, n=1 << 40, st=None),  # noqa: E731
                                         **k}.values())
    assert f(M=0, q=None) == A.AECCT_OK and f(N=0, y=None) == A.AECCT_OK
    for bad in (dict(M=-1), dict(N=-1), dict(K=0), dict(K=6), dict(ldc=7), dict(q=None), dict(s=None), dict(s=P + 2), dict(p=None),
                dict(w=None), dict(b=P + 1), dict(y=None), dict(y=P + 2), dict(y=P + 1, t=1), dict(t=3)):
        assert f(**bad) == BAD, bad
    assert f(K=65540, ldc=65540) == A.AECCT_ERR_UNSUPPORTED and f(M=1 << 31) == A.AECCT_ERR_UNSUPPORTED
    g = lambda **k: L.aecct_aap_linear_backward(*{**dict(dy=P, lddy=8, q=P, ldc=8, s=P, p=P, w=P, M=1, K=8, N=3, t=0, wt=0, dx=P,  # noqa: E731
                                                         dw=P, db=P, ws=P, n=1 << 40, st=None), **k}.values())
    for bad in (dict(M=-1), dict(K=5), dict(N=-1), dict(t=-1), dict(wt=3), dict(dy=None), dict(lddy=2), dict(q=None), dict(ldc=7),
                dict(s=None), dict(p=None), dict(w=None), dict(dx=P + 1), dict(dw=P + 1), dict(db=P + 1)):
        assert g(**bad) == BAD, bad
    n = ctypes.c_int64()
    assert L.aecct_aap_linear_workspace(1, 6, 1, ctypes.byref(n)) == BAD and L.aecct_aap_linear_workspace(1, 8, 1, None) == BAD
    assert L.aecct_aap_linear_backward_workspace(1, 8, 1, 4, 0, ctypes.byref(n)) == BAD
    assert np.int64(n.value) >= 0
