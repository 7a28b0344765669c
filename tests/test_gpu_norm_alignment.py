"""rms_quant and rms_quant_backward on tensors whose first row starts anywhere: rows come to shared memory by copies of whole
16-byte lines, and what lies outside of these at a tensor's two ends by ordinary loads.  With more rows than the GPU holds at
a time the place of the first row takes a later one.  Tolerances are those of the tests of aligned rows."""
import pytest
from test_gpu_norm import DTYPES, EPS, check_backward, check_forward, gain_of, make

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIZES = [(1, 513), (2, 300), (7, 1001), (20011, 257), (11003, 520), (6007, 1370), (700, 8200)]


def shifted(t, at, pad=0):
    """t, `at` elements behind a 16-byte boundary and rows `pad` further apart; the elements around it are not numbers."""
    rows, d = t.shape
    room = torch.full((at + rows * (d + pad) + 8,), float("nan"), device="cuda", dtype=t.dtype)
    v = room[at:at + rows * (d + pad)].view(rows, d + pad)[:, :d]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at,pad", [(1, 0), (3, 5)])
@pytest.mark.parametrize("rows,d", SIZES)
def test_forward(rows, d, at, pad, dtype):
    x, r, g = shifted(make(rows, d, dtype, 1), at, pad), shifted(make(rows, d, dtype, 2, size=2.0), 2 * at), gain_of(d, 3)
    check_forward(x, g, r, A.rms_quant(x, g, residual=r, eps=EPS, want_values=True))
    check_forward(x, g, None, A.rms_quant(x, g, eps=EPS))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at,pad", [(1, 0), (3, 5)])
@pytest.mark.parametrize("rows,d", SIZES)
def test_backward(rows, d, at, pad, dtype):
    dy, h = shifted(make(rows, d, dtype, 1, size=0.1), at, pad), shifted(make(rows, d, dtype, 2, size=2.0), 2 * at)
    ds, g = shifted(make(rows, d, dtype, 3), 3 * at), gain_of(d, 4)
    check_backward(dy, h, g, ds, *A.rms_quant_backward(dy, h, g, dtotal=ds, eps=EPS))
    check_backward(dy, h, g, None, *A.rms_quant_backward(dy, h, g, eps=EPS))


@pytest.mark.parametrize("rows,d", [(20011, 257), (6007, 1371)])
@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_sum_in_place(rows, d, at, into):
    """The sum over x or the residual: a copy of a row reads a few bytes of its neighbours, which others write meanwhile, and
    uses none of them."""
    x, r, g = shifted(make(rows, d, torch.bfloat16, 1), at), shifted(make(rows, d, torch.bfloat16, 2), at + 1), gain_of(d, 3)
    want = A.rms_quant(x, g, residual=r, eps=EPS)
    codes, scale, out = torch.empty_like(want[0]), torch.empty_like(want[1]), x if into == "x" else r
    status = A.load().aecct_rms_quant(x.data_ptr(), d, r.data_ptr(), d, g.data_ptr(), rows, d, 2, EPS, out.data_ptr(), codes.data_ptr(),
                                      scale.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
    assert status == A.AECCT_OK
    torch.cuda.synchronize()
    assert torch.equal(out, want[2]) and torch.equal(codes, want[0]) and torch.equal(scale, want[1])


@pytest.mark.parametrize("codes_at,sum_at,values_at", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (3, 5, 7)])
@pytest.mark.parametrize("rows,d", [(5, 64), (11003, 520), (300, 4096)])
def test_outputs_that_start_anywhere(rows, d, codes_at, sum_at, values_at):
    x, r, g = make(rows, d, torch.bfloat16, 1), make(rows, d, torch.bfloat16, 2), gain_of(d, 3)
    n = rows * d
    rooms = [torch.full((n + 16,), 9, device="cuda", dtype=t) for t in (torch.int8, torch.bfloat16, torch.bfloat16)]
    codes, total, values = (room[at:at + n].view(rows, d) for room, at in zip(rooms, (codes_at, sum_at, values_at)))
    scale = torch.empty(rows, device="cuda")
    status = A.load().aecct_rms_quant(x.data_ptr(), d, r.data_ptr(), d, g.data_ptr(), rows, d, 2, EPS, total.data_ptr(), codes.data_ptr(),
                                      scale.data_ptr(), values.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert status == A.AECCT_OK
    check_forward(x, g, r, (codes, scale, total, values))
    for room, at in zip(rooms, (codes_at, sum_at, values_at)):
        assert (room[:at] == 9).all() and (room[at + n:] == 9).all()
