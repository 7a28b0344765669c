"""clip_gradients on the GPU against its formula in 64 bits.

Tolerances, from the operations (u = 2^-24): a thread adds at most 64 squares in 32 bits, the rest is in 64,
so the sum is within 65 u and the norm within 34 u (2.1e-6); the factor within 37 u, and a product is
rounded to the gradient's type (fp16: to a step of 2^-24 where it is subnormal)."""
import ctypes
import math

import numpy as np
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-6


def make(sizes, dtypes, seed, size=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, device="cuda", generator=g) * size).to(t) for n, t in zip(sizes, dtypes)]


def check(grads, max_norm, norm, out):
    want = math.sqrt(math.fsum((g.double() ** 2).sum().item() for g in grads))
    assert norm.shape == () and abs(norm.item() - want) <= 35 * U * want
    c = min(1.0, max_norm / (want + EPS))
    for g, o in zip(grads, out):
        v = g.double() * c
        assert o.dtype == g.dtype
        if c == 1.0:
            assert torch.equal(o, g)
        assert ((o.double() - v).abs() <= (40 * U + ROUND[g.dtype]) * v.abs() + TINY[g.dtype]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("max_norm", [0.5, 1e4])
@pytest.mark.parametrize("sizes", [[1], [0], [], [0, 5, 0], [16384], [16383, 16385], [3, 1, 7, 100003, 2], [1 << 20, 12345, 1 << 16],
                                   [17] * 64, [33] * 65, [50] * 513, [5] * 1500 + [40000]])
def test_sizes(sizes, max_norm):
    grads = make(sizes, [DTYPES[j % 3] for j in range(len(sizes))], len(sizes))
    out = [torch.full_like(g, 9.0) for g in grads]
    norm = A.clip_gradients(grads, max_norm, out=out)
    check(grads, max_norm, norm, out)
    kept = [g.clone() for g in grads]
    again = A.clip_gradients(grads, max_norm)  # in place
    assert torch.equal(norm, again) and all(torch.equal(g, o) for g, o in zip(grads, out))
    check(kept, max_norm, again, grads)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at,to", [(1, 0), (0, 1), (3, 5), (8, 8)])
def test_tensors_that_do_not_start_on_16_bytes(at, to, dtype):
    src, dst = make([70000], [dtype], 3)[0], torch.zeros(70000, device="cuda", dtype=dtype)
    grads, out = [src[at:at + 50000]], [dst[to:to + 50000]]
    check(grads, 1.0, A.clip_gradients(grads, 1.0, out=out), out)
    assert not dst[:to].any() and not dst[to + 50000:].any()


@pytest.mark.gpu
def test_more_elements_than_one_round_of_the_grid():
    grads = make([40_000_003, 5], [torch.bfloat16, torch.float32], 1, size=0.01)
    out = [torch.empty_like(g) for g in grads]
    check(grads, 1.0, A.clip_gradients(grads, 1.0, out=out), out)


@pytest.mark.gpu
def test_values_that_are_not_finite():
    for bad, nan in ((float("inf"), False), (float("nan"), True), (1e30, False)):
        g = make([1000, 1000], [torch.float32] * 2, 1)
        g[1][77] = bad
        norm = A.clip_gradients(g, 1.0)
        assert norm.isnan() if nan else norm.isinf()
        assert g[0].isnan().all() if nan else not g[0].any()


@pytest.mark.gpu
def test_no_gradient_at_all():
    g = [torch.zeros(1000, device="cuda")]
    assert A.clip_gradients(g, 1.0).item() == 0.0 and not g[0].any()
    assert A.clip_gradients([], 1.0).item() == 0.0


@pytest.mark.gpu
def test_same_bits_on_every_run_and_on_another_stream():
    sizes = [4096 * 37 + 5] * 20
    grads = make(sizes, [torch.float32] * 20, 5)
    out = [torch.empty_like(g) for g in grads]
    norm = A.clip_gradients(grads, 1.0, out=out)
    side = torch.cuda.Stream()
    late = [torch.zeros_like(g) for g in grads]
    torch.cuda._sleep(50_000_000)
    for a, b in zip(late, grads):
        a.copy_(b)
    again = A.clip_gradients(late, 1.0, stream=side)
    side.synchronize()
    assert torch.equal(norm, again) and all(torch.equal(a, b) for a, b in zip(late, out))


@pytest.mark.gpu
def test_refusals():
    g = make([10, 10], [torch.float32] * 2, 1)
    for grads, kw in (([g[0].double()], {}), ([g[0].cpu()], {}), ([g[0][::2]], {}), (g, dict(out=g[:1])),
                      (g, dict(out=[g[0], g[1].half()])), (g, dict(out=[g[0], g[1][:5]]))):
        with pytest.raises(ValueError):
            A.clip_gradients(grads, 1.0, **kw)
    for m, eps in ((0.0, 1e-6), (-1.0, 1e-6), (float("nan"), 1e-6), (float("inf"), 1e-6), (1.0, -1e-6), (1.0, float("nan"))):
        with pytest.raises(A.AecctError):
            A.clip_gradients(g, m, eps=eps)


def test_c_entry_refuses_before_any_device_work():
    L, P, BAD = A.load(), 0x1000, A.AECCT_ERR_INVALID_ARG
    ptr = np.array([P, P], np.uintp)
    odd = np.array([P, P + 2], np.uintp)
    lens, types = np.array([4, 4], np.int64), np.array([0, 0], np.int32)
    size = ctypes.c_int64()
    assert L.aecct_clip_workspace(2, ctypes.byref(size)) == A.AECCT_OK and size.value > 0
    assert L.aecct_clip_workspace(-1, ctypes.byref(size)) == BAD and L.aecct_clip_workspace(1, None) == BAD
    d = lambda a: a.ctypes.data if a is not None else None  # noqa: E731

    def call(n=2, g=ptr, ln=lens, t=types, o=ptr, m=1.0, eps=1e-6, norm=P, w=P, wb=1 << 30):
        return L.aecct_clip_gradients(n, d(g), d(ln), d(t), d(o), m, eps, norm, w, wb, None)

    for bad in (dict(n=-1), dict(g=None), dict(ln=None), dict(t=None), dict(o=None), dict(g=odd), dict(o=odd), dict(norm=None),
                dict(norm=P + 1), dict(w=None), dict(w=P + 4), dict(wb=8), dict(m=0.0), dict(eps=-1.0),
                dict(ln=np.array([4, -1], np.int64)), dict(t=np.array([0, 3], np.int32)), dict(g=np.zeros(2, np.uintp))):
        assert call(**bad) == BAD, bad
