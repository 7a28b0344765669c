"""The operators launch on the current CUDA device, and refuse tensors that lie on another one before anything is
allocated or launched.  The tensors here have a device and a shape, and no memory: no GPU is needed."""
import pytest

from paper_2410_05911_gb300 import aecct as A

torch = pytest.importorskip("torch")
fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")


@pytest.fixture
def elsewhere():
    """Makes tensors on a device that is not the current one: there is none of this number."""
    mode = fake_tensor.FakeTensorMode()

    def make(shape, dtype):
        return fake_tensor.FakeTensor(mode, torch.empty(shape, dtype=dtype, device="meta"), torch.device("cuda:63"))

    return make


def test_tensors_of_another_device_are_refused(elsewhere):
    x, gain = elsewhere((4, 64), torch.float32), elsewhere((64,), torch.float32)
    codes, scale = elsewhere((4, 64), torch.int8), elsewhere((4,), torch.float32)
    packed, one, dy = elsewhere((8 * 16,), torch.uint8), elsewhere((1,), torch.float32), elsewhere((4, 8), torch.float32)
    for call in (lambda: A.rms_quant(x, gain, residual=x), lambda: A.rms_quant_backward(x, x, gain),
                 lambda: A.aap_linear(codes, scale, packed, one), lambda: A.aap_linear_backward(dy, codes, scale, packed, one),
                 lambda: A.clip_gradients([x, gain], 1.0), lambda: A.clip_gradients([x], 1.0, out=[x])):
        with pytest.raises(ValueError, match="cuda:63, which is not the current CUDA device"):
            call()
