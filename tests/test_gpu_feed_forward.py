"""The operators together, as the feed-forward example uses them: the block's output and its gradients
against the same formulas in float64, training, and single tokens against a batch."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def block():
    spec = importlib.util.spec_from_file_location("train_feed_forward", os.path.join(HERE, "examples", "train_feed_forward.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def unpack(t, n):
    """2-bit codes to 0, 1, -1 in float64."""
    f = torch.stack([(t >> s) & 3 for s in (0, 2, 4, 6)], -1).reshape(n, -1)
    return (f & 1).double() * (1 - (f & 2).double())


def dequantised(q, s):
    return q.double() * s.double()[:, None]


@pytest.mark.parametrize("tokens,d,hidden", [(1, 128, 512), (37, 36, 100), (300, 128, 512)])
def test_block_against_float64(block, tokens, d, hidden):
    """The formulas in float64 on the codes that the kernels made (a code may differ where a value lies
    between two).  Every float32 step is off by at most a few 2^-23 of the terms it sums; 1e-4 of a tensor's largest value is
    ten times what sums of 512 such terms can lose."""
    p = block.parameters(d, hidden, seed=3)
    x, r, dy = (torch.randn((tokens, d), device="cuda") for _ in range(3))
    weights = block.ternary(p)
    y, saved = block.forward(p, weights, x, r)
    g, dx = block.backward(p, weights, saved, dy)
    q1, s1, total, h, q2, s2 = saved
    eps = 1e-6
    w1, w2 = (unpack(t, n) * s.double() for (t, s), n in zip(weights, (hidden, d)))

    def normed(v, gain):
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + eps) * gain

    def norm_grad(dn, v, gain):
        v = v.clone().requires_grad_()
        gain = gain.clone().requires_grad_()
        normed(v, gain).backward(dn)
        return v.grad, gain.grad

    total64 = x.double() + r.double()
    n1 = normed(total64, p["g1"].double())
    assert (dequantised(q1, s1) - n1).abs().max() <= n1.abs().max() / 127 * 0.501
    u = dequantised(q1, s1) @ w1.T + p["b1"].double()
    h64 = torch.relu(u)
    n2 = normed(h.double(), p["g2"].double())
    assert (dequantised(q2, s2) - n2).abs().max() <= n2.abs().max() / 127 * 0.501
    y64 = total64 + dequantised(q2, s2) @ w2.T + p["b2"].double()
    dn = dy.double() @ w2
    dh64, dg2 = norm_grad(dn, h.double(), p["g2"].double())
    dh64 = torch.where(h > 0, dh64, torch.zeros_like(dh64))
    dn1 = dh64 @ w1
    dx64, dg1 = norm_grad(dn1, total64, p["g1"].double())
    dx64 = dx64 + dy.double()
    want = dict(w2=dy.double().T @ dequantised(q2, s2), b2=dy.double().sum(0), g2=dg2,
                w1=dh64.T @ dequantised(q1, s1), b1=dh64.sum(0), g1=dg1)
    for name, got, ref in [("h", h, h64), ("y", y, y64), ("dx", dx, dx64)] + [(k, g[k], v) for k, v in want.items()]:
        assert (got.double() - ref).abs().max() <= 1e-4 * ref.abs().max() + 1e-12, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_lowers_the_loss(block, dtype):
    _, losses, norms = block.train(steps=60, dtype=dtype)
    assert all(v == v and v < float("inf") for v in losses + norms)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5])


def test_single_tokens_are_the_batch(block):
    """The sums of a product are exact, and a row's norm is its own: a token alone, among a few (integer
    products) and among many (tensor cores) has the same bits."""
    p = block.parameters(128, 512, seed=5)
    x, r = torch.randn((2, 40, 128), device="cuda").to(torch.bfloat16)
    weights = block.ternary(p)
    many = block.forward(p, weights, x, r)[0]
    assert torch.equal(block.serve(p, x, r), many)
    for few in (2, 3, 4, 5, 17):
        assert torch.equal(block.forward(p, weights, x[:few], r[:few])[0], many[:few])


def test_example_runs(block, capsys):
    block.main()
    assert "the same" in capsys.readouterr().out
