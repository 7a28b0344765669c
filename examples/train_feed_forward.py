"""A feed-forward block of AAP linear layers, trained and then served a token at a time.

  total = x + residual                      (the residual stream)
  h     = relu(Quant(norm(total) g1) W1^T + b1)
  y     = total + Quant(norm(h) g2) W2^T + b2

Each norm with its residual addition and eq. Quant is one call (rms_quant), each product of int8 codes and
2-bit weights another (aap_linear), and so are their gradients; clip_gradients takes the gradients of all
parameters at once.  The weights that the optimiser moves are float32; aap_ternarize makes each step's
ternary ones, and the gradients pass straight through it.

    python examples/train_feed_forward.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_05911_gb300 import aecct  # noqa: E402


def parameters(d: int, hidden: int, seed: int = 0) -> dict:
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def uniform(n, k):
        return (torch.rand((n, k), device="cuda", generator=gen) * 2 - 1) * k ** -0.5

    return dict(w1=uniform(hidden, d), b1=torch.zeros(hidden, device="cuda"), g1=torch.ones(d, device="cuda"),
                w2=uniform(d, hidden), b2=torch.zeros(d, device="cuda"), g2=torch.ones(hidden, device="cuda"))


def ternary(p: dict):
    """The 2-bit weights of both layers, and their scales (one element each)."""
    (t1, t2), scale, _ = aecct.aap_ternarize([p["w1"], p["w2"]])
    return (t1, scale[0:1]), (t2, scale[1:2])


def forward(p: dict, weights, x, residual):
    """y, and what the backward pass reads."""
    w1, w2 = weights
    q1, s1, total, _ = aecct.rms_quant(x, p["g1"], residual=residual)
    h = torch.relu(aecct.aap_linear(q1, s1, *w1, bias=p["b1"], dtype=x.dtype))
    q2, s2, _, _ = aecct.rms_quant(h, p["g2"])
    y = total + aecct.aap_linear(q2, s2, *w2, bias=p["b2"], dtype=x.dtype)
    return y, (q1, s1, total, h, q2, s2)


def backward(p: dict, weights, saved, dy):
    """The gradients of the parameters, and that of x and of residual alike."""
    w1, w2 = weights
    q1, s1, total, h, q2, s2 = saved
    g = {}
    dn, g["w2"], g["b2"] = aecct.aap_linear_backward(dy, q2, s2, *w2)
    dh, g["g2"] = aecct.rms_quant_backward(dn, h, p["g2"])
    dh = torch.where(h > 0, dh, torch.zeros_like(dh))
    dn, g["w1"], g["b1"] = aecct.aap_linear_backward(dh, q1, s1, *w1)
    dx, g["g1"] = aecct.rms_quant_backward(dn, total, p["g1"], dtotal=dy)
    return g, dx


def train(steps: int = 60, tokens: int = 512, d: int = 128, hidden: int = 512, dtype=torch.bfloat16, rate: float = 3e-3,
          max_norm: float = 1.0, seed: int = 0):
    """Fits y to a fixed linear map of normed rows.  Returns the parameters, the losses and the gradients' norms."""
    p = parameters(d, hidden, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    teacher = torch.randn((d, d), device="cuda", generator=gen) * d ** -0.5
    optimiser = torch.optim.Adam(list(p.values()), lr=rate)
    losses, norms = [], []
    for _ in range(steps):
        x = torch.randn((tokens, d), device="cuda", generator=gen).to(dtype)
        residual = torch.randn((tokens, d), device="cuda", generator=gen).to(dtype)
        total = x.float() + residual.float()
        target = total + total @ teacher
        weights = ternary(p)
        y, saved = forward(p, weights, x, residual)
        off = y.float() - target
        losses.append((off * off).mean())
        grads, _ = backward(p, weights, saved, (off * (2.0 / off.numel())).to(dtype))
        norms.append(aecct.clip_gradients(list(grads.values()), max_norm))
        for name, value in p.items():
            value.grad = grads[name]
        optimiser.step()
    return p, [float(v) for v in losses], [float(v) for v in norms]


def serve(p: dict, x, residual):
    """The block's outputs, one row (token) at a time."""
    weights = ternary(p)
    return torch.cat([forward(p, weights, x[i:i + 1], residual[i:i + 1])[0] for i in range(x.shape[0])])


def main() -> None:
    p, losses, norms = train()
    for i in range(0, len(losses), 10):
        print(f"step {i:3d}  loss {losses[i]:.4f}  norm of the gradients {norms[i]:.3f}")
    print(f"last      loss {losses[-1]:.4f}")
    x, r = torch.randn((2, 16, 128), device="cuda").to(torch.bfloat16)
    together = forward(p, ternary(p), x, r)[0]
    print("16 tokens one at a time and together:", "the same" if torch.equal(serve(p, x, r), together) else "differ")


if __name__ == "__main__":
    main()
