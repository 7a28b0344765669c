"""The operators launch on the current CUDA device, and refuse tensors that lie on another one before anything is
allocated or launched.  The tensors here have a device and a shape, and no memory: no GPU is needed."""
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")

class Elsewhere(torch.Tensor):
    """A tensor of a type and shape, without memory, on a device that is not the current one: there is none of this number."""

    @staticmethod
    def __new__(cls, shape, dtype):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device=torch.device("cuda:63"))

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} of a tensor that should have been refused")


def test_tensors_of_another_device_are_refused():
    x, gain = Elsewhere((4, 64), torch.float32), Elsewhere((64,), torch.float32)
    codes, scale = Elsewhere((4, 64), torch.int8), Elsewhere((4,), torch.float32)
    packed, one, dy = Elsewhere((8 * 16,), torch.uint8), Elsewhere((1,), torch.float32), Elsewhere((4, 8), torch.float32)
    for call in (lambda: A.rms_quant(x, gain, residual=x), lambda: A.rms_quant_backward(x, x, gain),
                 lambda: A.aap_linear(codes, scale, packed, one), lambda: A.aap_linear_backward(dy, codes, scale, packed, one),
                 lambda: A.clip_gradients([x, gain], 1.0), lambda: A.clip_gradients([x], 1.0, out=[x])):
        with pytest.raises(ValueError, match="cuda:63, which is not the current CUDA device"):
            call()
