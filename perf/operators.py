"""The operators of training and serving AAP layers at any width, and what their performance is
measured on: the calls that a user makes of them, through paper_2410_05911_gb300.aecct.

Three operators, the first two with their gradients, each direction a "kind" of case:

  norm         rms_quant: the residual's addition, root-mean-square norm and eq. Quant: one int8
               row of codes with one scale per token.
  norm_grad    rms_quant_backward: the gradients of the input (and so of the residual stream) and
               of the gain, the rounding passed straight through.
  linear       aap_linear: the ternary product of those codes with 2-bit weights (eq. AAPLinear).
  linear_grad  aap_linear_backward: the gradients of the activations, the weights and the bias.
  clip         clip_gradients: the global norm over every gradient of a model, and the gradients
               scaled down to it.

Rows are tokens: the tokens of received words (a BCH(63,36) word has 90, a BCH(31,16) word 46) or
the positions of a prompt, from one token to long batches. Widths run from the decoder's 32 to the
usual ones of large models, odd ones among them.
"""
import math

import torch

own = False

DTYPES = dict(fp32=torch.float32, bf16=torch.bfloat16, fp16=torch.float16)
SIZE = dict(fp32=4, bf16=2, fp16=2)
EPS = 1e-6
ALPHA_MIN = 2.0 ** -100  # the least absmax a row is scaled by
MAX_NORM = 1.0


def listed():
    return [
        # one token while a sequence is being written: latency
        dict(name="norm_token", kind="norm", rows=1, width=4096, dtype="bf16", residual=True, pad=0),
        # a training batch of 4,096 BCH(63,36) words at the decoder's largest width, in its own type
        dict(name="norm_words", kind="norm", rows=368640, width=128, dtype="fp32", residual=True, pad=0),
        # rows of an odd width that lie apart in a wider tensor, the first norm of a network (no residual)
        dict(name="norm_odd", kind="norm", rows=10007, width=1001, dtype="fp16", residual=False, pad=23),
        # the backward pass over a long prompt, or a batch of prompts
        dict(name="norm_grad_prompt", kind="norm_grad", rows=8192, width=4096, dtype="bf16", residual=True, pad=0),
        # a ragged batch at a width that no vector load divides
        dict(name="norm_grad_odd", kind="norm_grad", rows=4999, width=1370, dtype="fp16", residual=True, pad=5),
        # one token through a square projection: the weights' bytes, and latency
        dict(name="linear_token", kind="linear", rows=1, k=4096, n=4096, dtype="bf16", bias=False),
        # 37 requests, a token each, through a feed-forward layer's first product
        dict(name="linear_requests", kind="linear", rows=37, k=4096, n=16384, dtype="bf16", bias=True),
        # a long prompt: bound by the tensor cores
        dict(name="linear_prompt", kind="linear", rows=8192, k=4096, n=4096, dtype="bf16", bias=True),
        # the same prompt's backward pass
        dict(name="linear_grad_prompt", kind="linear_grad", rows=8192, k=4096, n=4096, dtype="bf16", weights="bf16"),
        # 256 words through the decoder's own feed-forward layer, in 32 bits
        dict(name="linear_grad_words", kind="linear_grad", rows=23040, k=128, n=512, dtype="fp32", weights="fp32"),
        # the gradients of the deepest decoder, N = 10 blocks of d = 128: 160 tensors, most of them small
        dict(name="clip_decoder", kind="clip", layers=10, d=128, dtype="fp32", norm=2.5),
        # the gradients of a large model's blocks, matrices in 16 bits and vectors in 32
        dict(name="clip_large", kind="clip", layers=6, d=2048, dtype="bf16", norm=40.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _usual(v, by):
    """v rounded down to a multiple of `by`; multiples of 1,024 to a power of two."""
    v = max(by, v // by * by)
    return v if v % 1024 else 1 << (v.bit_length() - 1)


def draw(rng):
    kind = rng.choices(("norm", "norm_grad", "linear", "linear_grad", "clip"), (0.22, 0.2, 0.25, 0.2, 0.13))[0]
    dtype = rng.choice(("bf16", "bf16", "fp32", "fp16"))
    if kind in ("norm", "norm_grad"):
        width = _log_int(rng, 32, 8192)
        width = rng.choice((width | 1, _usual(width, 8), _usual(width, 64)))
        rows = _log_int(rng, 1, max(2, min(400000, (45 if kind == "norm" else 24) * 10 ** 6 // width)))
        return dict(kind=kind, rows=rows, width=width, dtype=dtype, residual=rng.random() < 0.7,
                    pad=rng.choice((0, 0, 8, rng.randint(1, 64))))
    if kind == "clip":
        d = rng.choice((32, 64, 128, _log_int(rng, 80, 2000) | 1))
        layers = rng.randint(1, max(1, min(12, int(6.0 * 2048 ** 2 / d ** 2))))
        return dict(kind=kind, layers=layers, d=d, dtype=dtype, norm=rng.choice((0.3, 2.5, 40.0)))
    k, n = 4 * (_log_int(rng, 8, 2048) | 1), _log_int(rng, 32, 8192) | 1
    k, n = rng.choice(((k, n), (_usual(k, 64), _usual(n, 16))))
    rows = _log_int(rng, 1, max(2, min(60000, 120 * 10 ** 9 // (k * n), 10 ** 8 // (k + n))))
    if kind == "linear":
        return dict(kind=kind, rows=rows, k=k, n=n, dtype=dtype, bias=rng.random() < 0.6)
    return dict(kind=kind, rows=rows, k=k, n=n, dtype=dtype, weights=rng.choice((dtype, "fp32")))


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _rows(g, rows, width, dtype, pad, size):
    """Activations or gradients [rows, width] that lie in a tensor `pad` wider: rows of different sizes,
    a few columns much larger than the others, and some rows of zeros (padding tokens)."""
    x = torch.empty((rows, width + pad), device="cuda").normal_(generator=g)
    x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=g)) * size
    x[:, torch.randint(0, width, (max(1, width // 256),), device="cuda", generator=g)] *= 8.0
    if rows > 1:
        x[torch.rand((rows,), device="cuda", generator=g) < 0.02] = 0.0
    return x.to(DTYPES[dtype])[:, :width]


def _gain(g, width):
    return 1.0 + 0.2 * torch.randn((width,), device="cuda", generator=g)


def _shapes(case):
    """The tensors of a model in blocks of d, F = 4 d: 6 weight matrices, 6 biases and 4 norm vectors each."""
    d = case["d"]
    block = [(d, d)] * 4 + [(4 * d, d), (d, 4 * d)] + [(d,)] * 4 + [(4 * d,), (d,)] + [(d,)] * 4
    return block * case["layers"]


def _views(shapes, dtypes):
    """One buffer for each type, and a tensor of each shape in them, 256 bytes apart at least."""
    flat, at = {}, {}
    for s, t in zip(shapes, dtypes):
        at[t] = at.get(t, 0) + -(-math.prod(s) // 128) * 128
    for t in at:
        flat[t], at[t] = torch.zeros(at[t], device="cuda", dtype=DTYPES[t]), 0
    views = []
    for s, t in zip(shapes, dtypes):
        views.append(flat[t][at[t]:at[t] + math.prod(s)].view(s))
        at[t] += -(-math.prod(s) // 128) * 128
    return flat, views


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, st = case["kind"], dict(case=case)
    if kind == "norm":
        st["x"] = _rows(g, case["rows"], case["width"], case["dtype"], case["pad"], 1.0)
        st["residual"] = _rows(g, case["rows"], case["width"], case["dtype"], 0, 2.0) if case["residual"] else None
        st["gain"] = _gain(g, case["width"])
    elif kind == "norm_grad":
        st["dy"] = _rows(g, case["rows"], case["width"], case["dtype"], case["pad"], 0.05)
        st["total"] = _rows(g, case["rows"], case["width"], case["dtype"], 0, 2.0)
        st["dtotal"] = _rows(g, case["rows"], case["width"], case["dtype"], 0, 0.05) if case["residual"] else None
        st["gain"] = _gain(g, case["width"])
    elif kind == "clip":
        shapes = _shapes(case)
        dtypes = [case["dtype"] if len(s) == 2 else "fp32" for s in shapes]
        size = case["norm"] / math.sqrt(sum(math.prod(s) for s in shapes))
        st["grads"] = [torch.empty(s, device="cuda").normal_(generator=g).mul_(size).to(DTYPES[t]) for s, t in zip(shapes, dtypes)]
        st["flat"], st["out"] = _views(shapes, dtypes)
    else:
        rows, k, n = case["rows"], case["k"], case["n"]
        x = _rows(g, rows, k, "fp32", 0, 1.0)
        alpha = x.abs().amax(1).clamp_min(ALPHA_MIN)
        st["codes"] = torch.round(x * (127.0 / alpha)[:, None]).to(torch.int8)
        st["scale"] = alpha / 127.0
        b = torch.randint(0, 256, (n * k // 4,), device="cuda", generator=g, dtype=torch.uint8)
        st["packed"] = b & (((b << 1) & 0xAA) | 0x55)  # no field is 10: half of the weights are 0
        st["w_scale"] = torch.rand((1,), device="cuda", generator=g) * 0.02 + 0.01
        if kind == "linear":
            st["bias"] = 0.1 * torch.randn((n,), device="cuda", generator=g) if case["bias"] else None
        else:
            st["dy"] = _rows(g, rows, n, case["dtype"], 0, 0.05)
    return st


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return (_own if own else _plain)[kind](st)


def _unpack(packed, k):
    """2-bit fields, the lowest first: 00 = 0, 01 = +1, 11 = -1."""
    f = (packed[:, None] >> torch.tensor([0, 2, 4, 6], device="cuda", dtype=torch.uint8)) & 3
    return (f & 1).float().view(-1, k) - (f & 2).float().view(-1, k)


def _norm(st):
    dtype = DTYPES[st["case"]["dtype"]]
    h = st["x"].float()
    if st["residual"] is not None:
        h = (h + st["residual"].float()).to(dtype)
        total, h = h, h.float()
    z = h * st["gain"]
    alpha = z.abs().amax(1, keepdim=True).clamp_min(ALPHA_MIN)
    q = torch.round(z * torch.div(torch.full_like(alpha, 127.0), alpha))
    scale = alpha * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) / 127.0
    out = dict(codes=q.to(torch.int8), scale=scale[:, 0], values=(q * scale).to(dtype))
    return dict(out, total=total) if st["residual"] is not None else out


def _norm_grad(st):
    h, dy = st["total"].float(), st["dy"].float()
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    t = dy * st["gain"]
    dx = r * t - h * (r * r * r * (t * h).mean(1, keepdim=True))
    if st["dtotal"] is not None:
        dx = dx + st["dtotal"].float()
    return dict(dx=dx.to(DTYPES[st["case"]["dtype"]]), dgain=(dy * (h * r)).sum(0))


def _linear(st):
    acc = st["codes"].float() @ _unpack(st["packed"], st["case"]["k"]).T
    y = acc * (st["scale"] * st["w_scale"])[:, None]
    return dict(y=(y if st["bias"] is None else y + st["bias"]).to(DTYPES[st["case"]["dtype"]]))


def _linear_grad(st):
    c = st["case"]
    dy = st["dy"].float()
    dx = (dy @ _unpack(st["packed"], c["k"])) * st["w_scale"]
    dw = (dy * st["scale"][:, None]).T @ st["codes"].float()
    return dict(dx=dx.to(DTYPES[c["dtype"]]), dw=dw.to(DTYPES[c["weights"]]), db=dy.sum(0))


def _clip(st):
    norm = torch.stack([g.float().square().sum() for g in st["grads"]]).sum().sqrt()
    by = torch.clamp(MAX_NORM / (norm + EPS), max=1.0)
    for g, o in zip(st["grads"], st["out"]):
        o.copy_(g.float() * by)
    return dict(norm=norm, grads=st["flat"])


def _own_norm(st):
    from paper_2410_05911_gb300 import aecct

    codes, scale, total, values = aecct.rms_quant(st["x"], st["gain"], residual=st["residual"], eps=EPS, want_values=True)
    out = dict(codes=codes, scale=scale, values=values)
    return dict(out, total=total) if st["residual"] is not None else out


def _own_norm_grad(st):
    from paper_2410_05911_gb300 import aecct

    dx, dgain = aecct.rms_quant_backward(st["dy"], st["total"], st["gain"], dtotal=st["dtotal"], eps=EPS)
    return dict(dx=dx, dgain=dgain)


def _own_linear(st):
    from paper_2410_05911_gb300 import aecct

    return dict(y=aecct.aap_linear(st["codes"], st["scale"], st["packed"], st["w_scale"], bias=st["bias"],
                                   dtype=DTYPES[st["case"]["dtype"]]))


def _own_linear_grad(st):
    from paper_2410_05911_gb300 import aecct

    dx, dw, db = aecct.aap_linear_backward(st["dy"], st["codes"], st["scale"], st["packed"], st["w_scale"],
                                           weight_dtype=DTYPES[st["case"]["weights"]])
    return dict(dx=dx, dw=dw, db=db)


def _own_clip(st):
    from paper_2410_05911_gb300 import aecct

    return dict(norm=aecct.clip_gradients(st["grads"], MAX_NORM, eps=EPS, out=st["out"]), grads=st["flat"])


_plain = dict(norm=_norm, norm_grad=_norm_grad, linear=_linear, linear_grad=_linear_grad, clip=_clip)
_own = dict(norm=_own_norm, norm_grad=_own_norm_grad, linear=_own_linear, linear_grad=_own_linear_grad, clip=_own_clip)


# ------------------------------------------------------------------------------------------
# the work of a pass
# ------------------------------------------------------------------------------------------
def work(case):
    kind, s = case["kind"], SIZE[case["dtype"]]
    if kind == "clip":
        shapes = _shapes(case)
        size = sum(math.prod(x) * (s if len(x) == 2 else 4) for x in shapes)
        return dict(bytes=2.0 * size + 4, flops=3.0 * sum(math.prod(x) for x in shapes))
    if kind in ("norm", "norm_grad"):
        rows, size = case["rows"], float(case["rows"]) * case["width"]
        if kind == "norm":  # the input, the codes and their values; the residual, read and written
            return dict(bytes=size * (2 * s + 1 + (2 * s if case["residual"] else 0)) + 4.0 * (rows + case["width"]), flops=8.0 * size)
        return dict(bytes=size * (3 * s + (s if case["residual"] else 0)) + 8.0 * case["width"], flops=12.0 * size)
    m, k, n = float(case["rows"]), float(case["k"]), float(case["n"])
    reads = m * k + 4 * m + n * k / 4 + 4
    if kind == "linear":
        return dict(bytes=reads + m * n * s + (4 * n if case["bias"] else 0), flops=2 * m * n * k)
    return dict(bytes=reads + m * n * s + m * k * s + n * k * SIZE[case["weights"]] + 4 * n, flops=4 * m * n * k)


# ------------------------------------------------------------------------------------------
# the same values in 64 bits
# ------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    d = lambda name: st[name].double()  # noqa: E731
    if kind == "clip":
        parts = [(g.double() ** 2).sum().item() for g in st["grads"]]
        norm = math.sqrt(math.fsum(parts))
        by = min(1.0, MAX_NORM / (norm + EPS))
        flat = {t: torch.zeros(v.shape, dtype=torch.float64, device="cuda") for t, v in st["flat"].items()}
        for g, o in zip(st["grads"], st["out"]):
            t = next(t for t in flat if DTYPES[t] == o.dtype)
            at = o.storage_offset()
            flat[t][at:at + o.numel()] = (g.double() * by).reshape(-1)
        return dict(norm=norm, grads=flat)
    if kind == "norm":
        h = d("x")
        out = {}
        if st["residual"] is not None:  # the sum as it is kept, in the stream's own type
            h = out["total"] = (h + d("residual")).to(DTYPES[case["dtype"]]).double()
        mean = torch.einsum("ij,ij->i", h, h) / case["width"]
        y = h * d("gain") / torch.sqrt(mean + EPS)[:, None]
        least = ALPHA_MIN / torch.sqrt(mean + EPS)
        alpha = torch.maximum(torch.linalg.vector_norm(y, ord=math.inf, dim=1), least)
        q = torch.round(127.0 * y / alpha[:, None])
        return dict(out, codes=None, scale=alpha / 127.0, values=q * alpha[:, None] / 127.0)
    if kind == "norm_grad":
        h, dy, width = d("total"), d("dy"), case["width"]
        rms = torch.sqrt(torch.einsum("ij,ij->i", h, h) / width + EPS)[:, None]
        unit = h / rms
        t = dy * d("gain")
        dx = (t - unit * (torch.einsum("ij,ij->i", t, unit) / width)[:, None]) / rms
        return dict(dx=dx if st["dtotal"] is None else dx + d("dtotal"), dgain=torch.einsum("ij,ij->j", dy, unit))
    f = torch.stack([(st["packed"] >> s) % 4 for s in (0, 2, 4, 6)], 1).reshape(case["n"], case["k"])
    w = torch.where(f == 3, -1.0, f.double()) * d("w_scale")
    x = d("codes") * d("scale")[:, None]
    if kind == "linear":
        y = x @ w.T
        return dict(y=y if st["bias"] is None else y + d("bias"))
    return dict(dx=d("dy") @ w, dw=d("dy").T @ x, db=torch.ones(case["rows"], dtype=torch.float64, device="cuda") @ d("dy"))
