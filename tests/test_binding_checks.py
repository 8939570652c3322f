"""What the binding's calls that train a router take for a tensor: type, shape, device and strides, without a GPU."""
import pytest
import torch

from paper_2503_09716_amd.binding import _typed


class OnDevice:
    """A CPU tensor that says it lives on a GPU."""

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index

    is_cuda = True


def f32(*n):
    return torch.zeros(n)


def test_shapes_that_hold_the_same_rows():
    for t, shape in [(f32(6, 4), (6, 4)), (f32(24), (6, 4)), (f32(2, 3, 4), (6, 4)), (f32(2, 3), (6,)), (f32(6, 1), (6,)), (f32(), (1,)), (f32(1), (1,)),
                     (f32(0), (0, 4)), (f32(0, 4), (0, 4))]:
        assert _typed(OnDevice(t), torch.float32, shape, 0) == t.data_ptr()
    assert _typed(None, torch.float32, (6, 4), 0) is None


@pytest.mark.parametrize("t,shape", [(f32(4, 6), (6, 4)), (f32(3, 8), (6, 4)), (f32(6, 5), (6, 4)), (f32(23), (6, 4)), (f32(8, 4)[::2], (4, 4)), (f32(6, 4).t(), (4, 6)),
                                     (f32(6, 4).double(), (6, 4)), (f32(6, 4).bfloat16(), (6, 4)), (f32(0), (1,))])
def test_other_rows_types_and_strides_are_refused(t, shape):
    with pytest.raises(AssertionError):
        _typed(OnDevice(t), torch.float32, shape, 0)


def test_tensors_of_another_device_are_refused():
    t = f32(6, 4)
    for at, wanted in ((1, 0), (0, 1), (-1, 0)):
        with pytest.raises(AssertionError):
            _typed(OnDevice(t, at), torch.float32, (6, 4), wanted)
    with pytest.raises(AssertionError):
        _typed(t, torch.float32, (6, 4), 0)       # in host memory
