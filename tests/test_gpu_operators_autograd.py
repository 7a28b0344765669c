"""The operators record nothing for autograd, and say so instead of dropping a gradient."""
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def tensors(M=12, K=64, N=20):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dy, w = (torch.randn(s, device="cuda", generator=g) for s in ((M, K), (M, K), (M, N), (N, K)))
    return x, r, torch.rand(K, device="cuda", generator=g) + 0.5, w, torch.randn(N, device="cuda", generator=g), dy


def needs(t):
    return t.clone().requires_grad_()


def test_tensors_that_require_a_gradient_are_refused():
    x, r, gain, w, b, dy = tensors()
    (t,), ws, _ = A.aap_ternarize([w])
    codes, scale, total, _ = A.rms_quant(x, gain, residual=r)
    calls = [lambda: A.rms_quant(needs(x), gain), lambda: A.rms_quant(x, needs(gain)), lambda: A.rms_quant(x, gain, residual=needs(r)),
             lambda: A.rms_quant_backward(needs(x), total, gain), lambda: A.rms_quant_backward(x, total, needs(gain)),
             lambda: A.rms_quant_backward(x, needs(total), gain), lambda: A.rms_quant_backward(x, total, gain, dtotal=needs(r)),
             lambda: A.aap_linear(codes, needs(scale), t, ws), lambda: A.aap_linear(codes, scale, t, needs(ws)),
             lambda: A.aap_linear(codes, scale, t, ws, bias=needs(b)), lambda: A.aap_linear_backward(needs(dy), codes, scale, t, ws)]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad():
            call()


class Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, weight, bias):
        (t,), ws, _ = A.aap_ternarize([weight])
        codes, scale, total, _ = A.rms_quant(x, gain)
        ctx.save_for_backward(codes, scale, total, gain, t, ws)
        return A.aap_linear(codes, scale, t, ws, bias=bias, dtype=x.dtype)

    @staticmethod
    def backward(ctx, dy):
        codes, scale, total, gain, t, ws = ctx.saved_tensors
        dn, dw, db = A.aap_linear_backward(dy, codes, scale, t, ws)
        dx, dgain = A.rms_quant_backward(dn, total, gain)
        return dx, dgain, dw, db


def test_in_a_function_of_autograd():
    x, _, gain, w, b, dy = tensors()
    inputs = [needs(v) for v in (x, gain, w, b)]
    y = Layer.apply(*inputs)
    y.backward(dy)
    (t,), ws, _ = A.aap_ternarize([w])
    codes, scale, total, _ = A.rms_quant(x, gain)
    assert torch.equal(y.detach(), A.aap_linear(codes, scale, t, ws, bias=b))
    dn, dw, db = A.aap_linear_backward(dy, codes, scale, t, ws)
    dx, dgain = A.rms_quant_backward(dn, total, gain)
    for got, want in zip(inputs, (dx, dgain, dw, db)):
        assert torch.equal(got.grad, want)
