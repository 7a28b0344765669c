"""rms_quant and rms_quant_backward on the GPU against their formulas in 64 bits.

Tolerances, from the operations (u = 2^-24): a row's sum of squares has at most 32 terms of a thread one
after the other and 10 levels of a tree, all positive, so it is within 42 u; r within 21 u and four
roundings, scale within 28 u (1.7e-6).  The codes come from single operations that numpy rounds alike:
equal.  dx is r t - h c: each product within 64 u of its own size.  dgain adds `rows` products in some
order: within (rows + 64) u of the sum of their sizes.  A result in 16 bits is rounded once more."""
import ctypes

import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-6


def make(rows, d, dtype, seed, pad=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((rows, d + pad), device="cuda").normal_(generator=g) * size
    if rows > 2:
        x[rows // 2] = 0.0
        x[rows - 1] *= 1e-3
    return x.to(dtype)[:, :d]


def gain_of(d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 1.0 + 0.3 * torch.randn((d,), device="cuda", generator=g)


def check_forward(x, gain, residual, out):
    codes, scale, total, values = out
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(total, h)
    f = h.float().cpu().numpy()
    z = f * gain.cpu().numpy()
    alpha = np.maximum(np.abs(z).max(1, initial=0.0), np.float32(2.0 ** -100))
    q = np.rint(z * (np.float32(127.0) / alpha)[:, None])
    assert np.array_equal(codes.cpu().numpy(), q.astype(np.int8))
    rms = np.sqrt((f.astype(np.float64) ** 2).mean(1) + np.float32(EPS))
    want = alpha.astype(np.float64) / rms / 127.0
    got = scale.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= 28 * U * want).all()
    if values is not None:
        v = q.astype(np.float64) * want[:, None]
        err = np.abs(values.double().cpu().numpy() - v)
        assert (err <= (30 * U + ROUND[x.dtype]) * np.abs(v) + TINY[x.dtype]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (1, 4096), (5, 32), (37, 46), (300, 90), (129, 128), (17, 511), (9, 512),
                                    (40, 513), (7, 1001), (6, 1370), (5, 5120), (3, 8191), (3, 16384), (2, 16392), (2, 32768)])
def test_forward(rows, d, dtype):
    x, r, g = make(rows, d, dtype, 1), make(rows, d, dtype, 2, size=2.0), gain_of(d, 3)
    check_forward(x, g, r, A.rms_quant(x, g, residual=r, eps=EPS, want_values=True))
    check_forward(x, g, None, A.rms_quant(x, g, eps=EPS))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [1, 3, 8, 64])
@pytest.mark.parametrize("d", [33, 64, 1000, 2048])
def test_rows_that_lie_apart(d, pad, dtype):
    x, r, g = make(19, d, dtype, 4, pad=pad), make(19, d, dtype, 5, pad=2 * pad), gain_of(d, 6)
    assert not x.is_contiguous()
    check_forward(x, g, r, A.rms_quant(x, g, residual=r, eps=EPS, want_values=True))


@pytest.mark.gpu
def test_shapes_of_more_dimensions_and_no_rows():
    g = gain_of(96, 1)
    x = make(6 * 7, 96, torch.bfloat16, 2).view(6, 7, 96)
    codes, scale, total, _ = A.rms_quant(x, g, eps=EPS)
    assert codes.shape == x.shape and scale.shape == (6, 7) and total is x
    check_forward(x.reshape(-1, 96), g, None, (codes.view(-1, 96), scale.view(-1), x.reshape(-1, 96), None))
    t = x.transpose(0, 1)  # rows an unequal distance apart
    codes, scale, _, _ = A.rms_quant(t, g, eps=EPS)
    check_forward(t.reshape(-1, 96), g, None, (codes.view(-1, 96), scale.view(-1), t.reshape(-1, 96), None))
    one = A.rms_quant(x[0, 0], g, eps=EPS)
    assert one[0].shape == (96,) and one[1].shape == ()
    none = A.rms_quant(x[:0], g, residual=x[:0], eps=EPS, want_values=True)
    assert none[0].shape == (0, 7, 96) and none[1].shape == (0, 7)
    dx, dg = A.rms_quant_backward(x[:0], x[:0], g)
    assert dx.shape == (0, 7, 96) and not dg.any()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [40, 128, 4096])
def test_rows_that_are_not_finite_leave_the_others_alone(d):
    x, g = make(12, d, torch.float32, 7), gain_of(d, 8)
    want = A.rms_quant(x, g, eps=EPS, want_values=True)
    y = x.clone()
    y[3, d // 2], y[5, 0], y[7, d - 1] = float("nan"), float("inf"), -float("inf")
    got = A.rms_quant(y, g, eps=EPS, want_values=True)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[3, 5, 7]] = True
    assert got[1][bad].isnan().all()
    for a, b in zip((got[0], got[1], got[3]), (want[0], want[1], want[3])):
        assert torch.equal(a[~bad], b[~bad])


@pytest.mark.gpu
def test_largest_and_smallest_rows():
    g = torch.ones(256, device="cuda")
    x = torch.ones((4, 256), device="cuda") * torch.tensor([1e18, 1e-18, 1e-32, 0.0], device="cuda")[:, None]
    codes, scale, _, values = A.rms_quant(x, g, eps=0.0, want_values=True)
    assert (codes[:2] == 127).all() and torch.allclose(values[:2], torch.ones_like(values[:2]), rtol=1e-5, atol=0)
    assert (codes[3] == 0).all()
    # under 2^-100 the scale does not follow the row down any further
    assert (codes[2] == int(np.rint(1e-32 * 127 * 2.0 ** 100))).all()


def formula64(dy, h, gain, dsum):
    dy, h, gain = dy.double(), h.double(), gain.double()
    d = h.shape[1]
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + float(np.float32(EPS)))
    t = dy * gain
    a, b = r * t, h * r ** 3 * (t * h).mean(1, keepdim=True)
    size = a.abs() + h.abs() * r ** 3 * (t * h).abs().mean(1, keepdim=True)
    dx = a - b + (dsum.double() if dsum is not None else 0.0)
    if dsum is not None:
        size = size + dsum.double().abs()
    p = dy * h * r
    return dx, size, p.sum(0), p.abs().sum(0)


def check_backward(dy, h, gain, dsum, dx, dgain):
    want, size, wg, sg = formula64(dy, h, gain, dsum)
    assert dx.dtype == h.dtype
    assert ((dx.double() - want).abs() <= 64 * U * size + ROUND[h.dtype] * want.abs() + TINY[h.dtype]).all()
    assert ((dgain.double() - wg).abs() <= (h.shape[0] + 64) * U * sg).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (1, 4096), (5, 32), (2000, 46), (20000, 90), (3001, 128), (700, 511), (333, 513),
                                    (500, 1001), (600, 1370), (900, 5120), (31, 8191), (200, 16384), (20, 16392), (7, 32768)])
def test_backward(rows, d, dtype):
    dy, h, ds, g = make(rows, d, dtype, 1, size=0.1), make(rows, d, dtype, 2, size=2.0), make(rows, d, dtype, 3), gain_of(d, 4)
    check_backward(dy, h, g, ds, *A.rms_quant_backward(dy, h, g, dtotal=ds, eps=EPS))
    check_backward(dy, h, g, None, *A.rms_quant_backward(dy, h, g, eps=EPS))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,pad", [(64, 8), (64, 1), (1001, 3), (2048, 64)])
def test_backward_of_rows_that_lie_apart(d, pad, dtype):
    dy, h, ds, g = make(70, d, dtype, 1, pad), make(70, d, dtype, 2, 2 * pad), make(70, d, dtype, 3, 3 * pad), gain_of(d, 4)
    check_backward(dy, h, g, ds, *A.rms_quant_backward(dy, h, g, dtotal=ds, eps=EPS))


@pytest.mark.gpu
def test_backward_against_differences():
    # the loss sum(dy * norm(h)), norm in 64 bits without the rounding that is passed straight through.
    # Central differences with step s: s^2 / 6 of the third derivative (under 1e2 here), 1e-7 of rounding
    rows, d = 2, 48
    dy, h, g = make(rows, d, torch.float32, 1), make(rows, d, torch.float32, 2, size=2.0), gain_of(d, 4)
    dx, dgain = A.rms_quant_backward(dy, h, g, eps=EPS)
    w, a, b = (t.double().cpu() for t in (dy, h, g))

    def loss(a, b):
        return (w * a * b / torch.sqrt(a.square().mean(1, keepdim=True) + EPS)).sum()

    s = 1e-4
    for i in range(rows):
        for j in range(0, d, 5):
            e = torch.zeros_like(a)
            e[i, j] = s
            num = (loss(a + e, b) - loss(a - e, b)) / (2 * s)
            assert abs(num - dx[i, j].item()) <= 5e-6
    for j in range(d):
        e = torch.zeros_like(b)
        e[j] = s
        assert abs((loss(a, b + e) - loss(a, b - e)) / (2 * s) - dgain[j].item()) <= 5e-6


@pytest.mark.gpu
def test_same_bits_on_every_run_and_in_every_batch():
    dy, h, g = make(5000, 384, torch.bfloat16, 1), make(5000, 384, torch.bfloat16, 2), gain_of(384, 3)
    a, b = A.rms_quant(h, g, want_values=True), A.rms_quant(h[1234:1300], g, want_values=True)
    for p, q in zip(a, b):
        assert torch.equal(p[1234:1300], q)
    first, again = A.rms_quant_backward(dy, h, g), A.rms_quant_backward(dy, h, g)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.gpu
def test_sum_in_place_of_the_residual():
    x, r, g = make(50, 256, torch.bfloat16, 1), make(50, 256, torch.bfloat16, 2), gain_of(256, 3)
    want = A.rms_quant(x, g, residual=r)
    for into in (x.clone(), r.clone()):
        src = [t if into is not t else into for t in (x, r)]
        codes, scale = torch.empty_like(want[0]), torch.empty_like(want[1])
        a = into if torch.equal(into, x) else x
        b = into if torch.equal(into, r) else r
        st = A.load().aecct_rms_quant(a.data_ptr(), 256, b.data_ptr(), 256, g.data_ptr(), 50, 256, 2, EPS, into.data_ptr(),
                                      codes.data_ptr(), scale.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
        assert st == A.AECCT_OK and len(src) == 2
        torch.cuda.synchronize()
        assert torch.equal(into, want[2]) and torch.equal(codes, want[0]) and torch.equal(scale, want[1])


@pytest.mark.gpu
def test_on_another_stream():
    x, g = make(64, 256, torch.float32, 1), gain_of(256, 2)
    want = A.rms_quant(x, g, residual=x, want_values=True)
    wantb = A.rms_quant_backward(x, x, g)
    side = torch.cuda.Stream()
    y = torch.zeros_like(x)
    torch.cuda._sleep(50_000_000)
    y.copy_(x)
    got = A.rms_quant(y, g, residual=y, want_values=True, stream=side)
    gotb = A.rms_quant_backward(y, y, g, stream=side)
    del y
    other = torch.full_like(x, 7.0)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + gotb, want + wantb)) and bool((other == 7.0).all())


@pytest.mark.gpu
def test_refusals():
    x, g = make(4, 64, torch.float32, 1), gain_of(64, 2)
    for bad in (dict(x=x.double()), dict(x=x.cpu()), dict(gain=g[:63]), dict(gain=g.half()), dict(residual=x.half()),
                dict(residual=x[:3])):
        with pytest.raises(ValueError):
            A.rms_quant(**{"x": x, "gain": g, **bad})
    for bad in (dict(dy=x.int()), dict(total=x[:, :32]), dict(dtotal=x.half()), dict(gain=g[None])):
        with pytest.raises(ValueError):
            A.rms_quant_backward(**{"dy": x, "total": x, "gain": g, **bad})
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(A.AecctError):
            A.rms_quant(x, g, eps=eps)
    wide = torch.zeros((1, 32769), device="cuda")
    with pytest.raises(A.AecctError) as e:
        A.rms_quant(wide, wide[0])
    assert e.value.status == A.AECCT_ERR_UNSUPPORTED


def test_c_entries_refuse_before_any_device_work():
    L, P, OK, BAD = A.load(), 0x1000, A.AECCT_OK, A.AECCT_ERR_INVALID_ARG
    q = lambda **k: L.aecct_rms_quant(*{**dict(x=P, ldx=8, res=None, ldr=0, gain=P, rows=1, d=8, t=0, eps=1e-6, sum=None,  # noqa: E731
                                               codes=P, scale=P, values=None, s=None), **k}.values())
    assert q(rows=0, x=None) == OK
    for bad in (dict(rows=-1), dict(d=0), dict(t=3), dict(t=-1), dict(x=None), dict(x=P + 2), dict(ldx=7), dict(gain=None),
                dict(codes=None), dict(scale=None), dict(res=P, ldr=8), dict(res=P, ldr=7, sum=P), dict(res=P + 1, ldr=8, sum=P),
                dict(values=P + 1, t=2), dict(eps=-1.0)):
        assert q(**bad) == BAD, bad
    assert q(d=32769, ldx=32769) == A.AECCT_ERR_UNSUPPORTED
    b = lambda **k: L.aecct_rms_quant_backward(*{**dict(dy=P, lddy=8, h=P, ldh=8, ds=None, ldd=0, gain=P, rows=1, d=8, t=0,  # noqa: E731
                                                        eps=1e-6, dx=P, dg=P, w=P, n=1 << 30, s=None), **k}.values())
    for bad in (dict(rows=-1), dict(d=0), dict(t=9), dict(dy=None), dict(h=None), dict(lddy=7), dict(ldh=7), dict(ds=P, ldd=7),
                dict(dx=None), dict(dg=None), dict(w=None), dict(w=P + 8), dict(n=0), dict(eps=float("nan"))):
        if "n" in bad and not torch.cuda.is_available():
            continue  # (a workspace's size depends on the GPU)
        assert b(**bad) == BAD, bad
    n = ctypes.c_int64()
    assert L.aecct_rms_quant_backward_workspace(-1, 8, ctypes.byref(n)) == BAD
    assert L.aecct_rms_quant_backward_workspace(1, 8, None) == BAD
