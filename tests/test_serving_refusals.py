"""What the C entries of the paged cache, the attention over it and the sampling refuse before any device work, and tensors of
another device in Python: no GPU is needed."""
import ctypes
import math

import pytest

from paper_2410_05911_gb300 import aecct as A

P, BAD, FAR = 0x1000, A.AECCT_ERR_INVALID_ARG, A.AECCT_ERR_UNSUPPORTED


def cache(**kw):
    return A.KVPages(**{**dict(k=P, v=P, k_scale=P, v_scale=P, pages=8, page_size=16, heads=2, head_dim=64, ld=64, dtype=3), **kw})


def seqs(**kw):
    return A.KVSequences(**{**dict(table=P, lengths=P, ldt=4, batch=3, columns=4), **kw})


CACHES = [(dict(k=None), BAD), (dict(v=P + 8), BAD), (dict(k_scale=None), BAD), (dict(v_scale=P + 2), BAD), (dict(pages=-1), BAD), (dict(page_size=0), BAD),
          (dict(heads=0), BAD), (dict(head_dim=0), BAD), (dict(ld=63), BAD), (dict(ld=72), BAD), (dict(dtype=0), BAD), (dict(dtype=4), BAD), (dict(head_dim=257, ld=272), FAR),
          (dict(heads=1 << 20), FAR), (dict(page_size=1 << 20), FAR), (dict(pages=1 << 31), FAR), (dict(ld=(1 << 20) + 16), BAD), (dict(dtype=2, ld=68), BAD)]
SEQS = [(dict(table=None), BAD), (dict(lengths=None), BAD), (dict(lengths=P + 1), BAD), (dict(ldt=3), BAD), (dict(batch=-1), BAD), (dict(columns=-1), BAD),
        (dict(columns=1 << 28, ldt=1 << 28), FAR), (dict(batch=1 << 24), FAR)]


def append(c=None, s=None, rows=P, total=5, k=P, kr=128, kh=64, v=P, vr=128, vh=64, dtype=2):
    return A.load().aecct_kv_append(c or cache(), s or seqs(), rows, total, k, kr, kh, v, vr, vh, dtype, None)


def read(c=None, s=None, rows=P, total=5, k=P, v=P, dtype=2):
    return A.load().aecct_kv_read(c or cache(), s or seqs(), rows, total, k, v, dtype, None)


def attend(c=None, s=None, first=None, q=P, row=512, head=64, heads=8, dtype=2, scale=0.1, out=P, lse=None, w=P, wb=1 << 40):
    return A.load().aecct_paged_attention(c or cache(), s or seqs(), first, q, row, head, heads, dtype, scale, out, lse, w, wb, None)


@pytest.mark.parametrize("call", [append, read, attend])
def test_caches_and_sequences(call):
    for kw, status in CACHES:
        assert call(c=cache(**kw)) == status, kw
    for kw, status in SEQS:
        assert call(s=seqs(**kw)) == status, kw


def test_append_and_read():
    for kw in (dict(total=-1), dict(dtype=3), dict(dtype=-1), dict(rows=None), dict(rows=P + 2), dict(k=None), dict(v=P + 1), dict(kr=-1), dict(vh=-1),
               dict(c=cache(dtype=1)), dict(c=cache(dtype=2), dtype=0)):
        assert append(**kw) == BAD, kw
    assert append(total=1 << 31) == FAR and append(total=0) == 0 and append(s=seqs(batch=0)) == 0
    for kw in (dict(total=-1), dict(dtype=3), dict(rows=None), dict(rows=P + 2), dict(k=None), dict(v=P + 1)):
        assert read(**kw) == BAD, kw
    assert read(total=1 << 31) == FAR and read(total=0) == 0


def test_attention():
    for kw in (dict(first=P + 2), dict(q=None), dict(q=P + 1), dict(row=-1), dict(head=-1), dict(heads=7), dict(heads=0), dict(dtype=3), dict(scale=math.inf),
               dict(scale=math.nan), dict(out=None), dict(out=P + 1), dict(lse=P + 2), dict(c=cache(dtype=1)), dict(c=cache(dtype=1), dtype=0)):
        assert attend(**kw) == BAD, kw
    assert attend(heads=1 << 20) == FAR and attend(s=seqs(batch=0)) == 0
    L, size = A.load(), ctypes.c_int64()
    assert L.aecct_paged_attention_workspace(3, 8, 2, 64, 2, 3, None) == BAD
    for args in ((-1, 8, 2, 64, 2, 3), (3, 7, 2, 64, 2, 3), (3, 8, 0, 64, 2, 3), (3, 8, 2, 0, 2, 3), (3, 8, 2, 64, 3, 3), (3, 8, 2, 64, 0, 2), (3, 8, 2, 64, 0, 0)):
        assert L.aecct_paged_attention_workspace(*args, ctypes.byref(size)) == BAD, args
    assert L.aecct_paged_attention_workspace(3, 8, 2, 257, 2, 3, ctypes.byref(size)) == FAR
    assert L.aecct_paged_attention_workspace(0, 8, 2, 64, 2, 3, ctypes.byref(size)) == 0 and size.value == 0


def test_sample():
    def call(x=P, ld=100, rows=4, vocab=100, dtype=0, u=P, tokens=P, null=False, **kw):
        s = A.SampleSettings(**{**dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0), **kw})
        return A.load().aecct_sample(x, ld, rows, vocab, dtype, u, None if null else s, tokens, None)

    for kw in (dict(x=None), dict(x=P + 2), dict(ld=99), dict(rows=-1), dict(vocab=0), dict(dtype=3), dict(u=None), dict(u=P + 1), dict(tokens=None), dict(tokens=P + 4),
               dict(null=True), dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=-0.5), dict(top_p=math.inf), dict(min_p=-1.0),
               dict(temperature_dev=P + 1), dict(top_k_dev=P + 2), dict(top_p_dev=P + 3), dict(min_p_dev=P + 1)):
        assert call(**kw) == BAD, kw
    assert call(vocab=(1 << 19) + 1, ld=1 << 20) == FAR and call(rows=1 << 31) == FAR and call(rows=0) == 0


def test_tensors_of_another_device_are_refused():
    torch = pytest.importorskip("torch")

    class Elsewhere(torch.Tensor):
        """A tensor of a type and shape, without memory, on a device that is not the current one."""

        @staticmethod
        def __new__(cls, shape, dtype):
            return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device=torch.device("cuda:63"))

        @classmethod
        def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
            raise AssertionError(f"{func} of a tensor that should have been refused")

    rows, scale = Elsewhere((4, 2, 16, 64), torch.int8), Elsewhere((4, 2, 16), torch.float32)
    c = A.KVCache(rows, rows, scale, scale)
    x, table, n = Elsewhere((3, 2, 64), torch.bfloat16), Elsewhere((3, 4), torch.int32), Elsewhere((3,), torch.int32)
    for call in (lambda: A.kv_append(x, x, c, table, n), lambda: A.kv_read(c, table, n, None, 3), lambda: A.paged_attention(x, c, table, n),
                 lambda: A.sample(Elsewhere((3, 100), torch.float32), Elsewhere((3,), torch.float32))):
        with pytest.raises(ValueError, match="cuda:63, which is not the current CUDA device"):
            call()


def test_a_scale_that_overflows_in_powers_of_two():
    """Scores are taken in powers of two: scale log2 e has to be finite too."""
    for scale in (2.4e38, -2.4e38, 3.4e38, -math.inf):
        assert attend(scale=scale) == BAD, scale
