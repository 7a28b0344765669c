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


def test_tensors_with_a_tangent_are_refused():
    import torch.autograd.forward_ad as fw

    x, r, gain, w, b, dy = tensors()
    (t,), ws, _ = A.aap_ternarize([w])
    codes, scale, total, _ = A.rms_quant(x, gain, residual=r)
    cache = A.kv_cache(2, 2, 4, 16)
    half = A.kv_cache(2, 2, 4, 16, dtype=torch.float16)
    for c in (cache, half):
        for s in c:
            if s is not None:
                s.zero_()
    table, n = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")
    k = torch.randn((1, 2, 16), device="cuda")
    u = torch.rand((12,), device="cuda")
    each = torch.ones((12,), device="cuda")
    calls = [lambda d: A.rms_quant(d(x), gain), lambda d: A.rms_quant(x, d(gain)), lambda d: A.rms_quant(x, gain, residual=d(r)),
             lambda d: A.rms_quant_backward(d(x), total, gain), lambda d: A.rms_quant_backward(x, total, gain, dtotal=d(r)),
             lambda d: A.aap_linear(codes, d(scale), t, ws), lambda d: A.aap_linear(codes, scale, t, ws, bias=d(b)),
             lambda d: A.aap_linear_backward(d(dy), codes, scale, t, ws), lambda d: A.kv_append(d(k), k, cache, table, n),
             lambda d: A.kv_append(k, d(k), cache, table, n), lambda d: A.kv_append(k, k, cache._replace(v_scale=d(cache.v_scale)), table, n),
             lambda d: A.kv_read(cache._replace(k_scale=d(cache.k_scale)), table, n, None, 1), lambda d: A.kv_read(half._replace(v=d(half.v)), table, n, None, 1),
             lambda d: A.paged_attention(d(k), cache, table, n), lambda d: A.paged_attention(k.half(), half._replace(k=d(half.k)), table, n),
             lambda d: A.sample(d(x), u), lambda d: A.sample(x, d(u)), lambda d: A.sample(x, u, temperature=d(each))]
    with fw.dual_level():
        dual = lambda v: fw.make_dual(v, torch.ones_like(v))  # noqa: E731
        for i, call in enumerate(calls):
            for on in (True, False):
                with torch.set_grad_enabled(on), pytest.raises(ValueError, match="tangents"):
                    call(dual)
                    pytest.fail(f"call {i} was not refused")
            call(lambda v: fw.unpack_dual(dual(v)).primal)
        # in a function that says what its tangents are, forward mode is off
        class Norm(torch.autograd.Function):
            @staticmethod
            def forward(v):
                codes, scale, _, _ = A.rms_quant(v, gain)
                return codes.float() * scale.reshape(-1, 1)

            @staticmethod
            def setup_context(ctx, inputs, output):
                pass

            @staticmethod
            def jvp(ctx, tangent):
                return 2 * tangent

        y = fw.unpack_dual(Norm.apply(dual(x)))
        assert (y.tangent == 2).all() and (y.primal - x * gain).isfinite().all()
    for call in calls:
        call(lambda v: v)
