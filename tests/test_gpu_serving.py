"""The operators of serving together: a prompt's tokens into the cache at once, then tokens one at a time in a captured graph, and the
example that writes sequences."""
import importlib.util
import math
import os
import subprocess
import sys

import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate.py")
    spec = importlib.util.spec_from_file_location("generate", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype,cache_dtype", [(torch.bfloat16, torch.int8), (torch.float32, torch.int8), (torch.float16, torch.float16)])
def test_prompt_then_tokens_in_a_graph(dtype, cache_dtype):
    """The whole of a step in one graph, replayed with lengths that grow: projections, append, attention, logits and choice."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    batch, heads, kv, dim, page, vocab, steps = 3, 8, 2, 64, 16, 500, 6
    wide, prompt = (heads + 2 * kv) * dim, [21, 1, 40]
    (wq,), sq, _ = A.aap_ternarize([rand(wide, 256) / 16])
    (wo,), so, _ = A.aap_ternarize([rand(vocab, heads * dim) / 16])
    gain, gain_o = torch.rand((256,), device="cuda", generator=g) + 0.5, torch.ones(heads * dim, device="cuda")
    columns = -(-(max(prompt) + steps) // page)
    table = torch.randperm(batch * columns, device="cuda", generator=g).int().view(batch, columns)
    cache = A.kv_cache(batch * columns, kv, page, dim, dtype=cache_dtype)
    lengths = torch.tensor(prompt, **I32)

    def project(x):
        codes, scale, _, _ = A.rms_quant(x, gain)
        return A.aap_linear(codes, scale, wq, sq, dtype=dtype).view(len(x), -1, dim).split([heads, kv, kv], dim=1)

    # the prompts, ragged
    rows = torch.tensor([0, 21, 22, 62], **I32)
    x0 = rand(62, 256).to(dtype)
    _, k0, v0 = project(x0)
    A.kv_append(k0, v0, cache, table, lengths, rows=rows)

    x, u = torch.zeros((batch, 256), device="cuda", dtype=dtype), torch.zeros((batch,), device="cuda")

    def step():
        q, k, v = project(x)
        A.kv_append(k, v, cache, table, lengths)
        out, lse = A.paged_attention(q, cache, table, lengths, want_lse=True)
        codes, scale, _, _ = A.rms_quant(out.reshape(batch, -1), gain_o)
        logits = A.aap_linear(codes, scale, wo, so, dtype=dtype)
        return k, v, q, out, lse, logits, A.sample(logits, u, temperature=0.7, top_k=20, top_p=0.9)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lengths.add_(1)
        got = step()
    lengths.copy_(torch.tensor(prompt, **I32))
    kept = [[k0[rows[b]:rows[b + 1]]] for b in range(batch)], [[v0[rows[b]:rows[b + 1]]] for b in range(batch)]
    for n in range(steps):
        x.copy_(rand(batch, 256))
        u.copy_(torch.rand((batch,), device="cuda", generator=g))
        graph.replay()
        k, v, q, out, lse, logits, token = (t.clone() for t in got)
        for b in range(batch):
            kept[0][b].append(k[b:b + 1])
            kept[1][b].append(v[b:b + 1])
            ks, vs = (torch.cat(t[b]).double().repeat_interleave(heads // kv, 1) for t in kept)
            s = torch.einsum("hd,nhd->hn", q[b].double(), ks) / math.sqrt(dim)
            want = torch.einsum("hn,nhd->hd", torch.softmax(s, 1), vs)
            # Codes are off by half a step, 1/254 of a row's largest (0 for a 16-bit cache).  Keys: a score is off by that of sum |q| kmax, and
            # a weight by a factor of exp(2 of it) at most; values: by 1/254 of the largest; and the result's own rounding.
            step_of = 0.0 if cache_dtype is not torch.int8 else 1 / 254
            ds = step_of * q[b].double().abs().sum(1) * ks.abs().amax(2).amax(0) / math.sqrt(dim) + 1e-3
            most = vs.abs().amax(2).amax(0)
            tol = (torch.exp(2 * ds) - 1 + step_of + 2.0 ** -8) * most
            assert ((out[b].double() - want).abs() <= tol[:, None]).all()
            assert ((lse[b].double() - torch.logsumexp(s, 1)).abs() <= ds + 1e-3).all()
        # the same calls outside of the graph give the same bits
        assert torch.equal(A.paged_attention(q, cache, table, lengths)[0], out)
        assert torch.equal(A.sample(logits, u, temperature=0.7, top_k=20, top_p=0.9), token)
        assert ((token >= 0) & (token < vocab)).all()
    assert lengths.tolist() == [p + steps for p in prompt]
    for b in range(batch):  # the whole cache read back
        n = prompt[b] + steps
        ks, vs = A.kv_read(cache, table[b:b + 1], torch.tensor([n], **I32), torch.tensor([0, n], **I32), n)
        for read, t in ((ks, kept[0][b]), (vs, kept[1][b])):
            src = torch.cat(t).float()
            step_of = 0.0 if cache_dtype is not torch.int8 else 1 / 254
            assert ((read - src).abs() <= (step_of + 2.0 ** -20) * src.abs().amax(2, keepdim=True)).all()


def test_example():
    m = example()
    model = m.Model(vocab=300, layers=2)
    prompts = [[1, 2, 3], [5], [7, 8, 9, 10, 11]]
    together = m.generate(model, prompts, new=12)
    assert [len(s) for s in together] == [len(p) + 12 for p in prompts]
    assert all(s[:len(p)] == p and all(0 <= t < 300 for t in s) for s, p in zip(together, prompts))
    assert m.generate(model, prompts, new=12) == together
    greedy = m.generate(model, prompts[:1], new=8, temperature=0.0)
    assert greedy[0][:3] == prompts[0] and len(greedy[0]) == 11


FIRST_CALLS = r"""
import torch
from paper_2410_05911_gb300 import aecct as A
A.load()
g = torch.Generator(device="cuda").manual_seed(1)
rand = lambda *s: torch.randn(s, device="cuda", generator=g)
def arrays(batch, length):
    columns = -(-length // 16)
    table = torch.arange(batch * columns, device="cuda", dtype=torch.int32).view(batch, columns)
    cache = A.kv_cache(batch * columns, 2, 16, 64)
    for t in cache:
        t.zero_()
    n = torch.full((batch,), length, device="cuda", dtype=torch.int32)
    rows = torch.arange(batch + 1, device="cuda", dtype=torch.int32) * length
    return cache, table, n, rows, rand(batch * length, 2, 64), rand(batch, 8, 64)
few, many, long = arrays(2, 100), arrays(400, 50), arrays(3, 5000)
logits, u = rand(4, 50021), torch.rand((4,), device="cuda", generator=g)
def step():
    out = []
    for cache, table, n, rows, x, q in (few, many, long):
        A.kv_append(x, x, cache, table, n, rows=rows)
        out += [*A.paged_attention(q, cache, table, n, want_lse=True), *A.kv_read(cache, table, n, rows, len(x))]
    return out + [A.sample(logits, u, top_p=0.9), A.sample(logits[:, :1000], u, top_k=20)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
got = [t.clone() for t in got]
assert all(torch.equal(a, b) for a, b in zip(got, step())) and got[0].any()
print("same")
"""


def test_first_calls_of_a_process_in_a_capture():
    """Nothing of a call needs one before it outside of the graph."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
