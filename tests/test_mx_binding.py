"""What the binding's calls on 4-bit expert weights take for their buffers, without a GPU: a recorder stands for the library's calls."""
import pytest
import torch

from paper_2503_09716_amd import MxRows, WeightList, binding, make_shape
from paper_2503_09716_amd.binding import Moe, WeightListStruct
from test_binding_checks import OnDevice


class Recorder:
    """The library's own host functions, and nothing that would reach a GPU."""

    def __init__(self):
        self.calls = []
        self.lib = binding.load_library()

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.lib, name)
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def moe(monkeypatch):
    m = Moe.__new__(Moe)
    m.lib, m.device, m.h = Recorder(), 0, None
    m.y_dtype, m.out_dtype, m.gate_packed = torch.float32, torch.bfloat16, False
    monkeypatch.setattr(binding, "_raw_stream", lambda device: None)
    return m


def at(device, shape, dtype=torch.uint8):
    return OnDevice(torch.zeros(shape, dtype=dtype), device)


def rows_on(device, rows=4, cols=64):
    return MxRows(rows, cols, at(device, int(binding.load_library().moe_mx_rows_bytes(rows, cols))))


def list_on(device, *sizes):
    lib = binding.load_library()
    weights = [[torch.zeros(int(lib.moe_mx_weight_bytes(*s)), dtype=torch.uint8) for _ in range(2)] for s in sizes]
    return WeightList(WeightListStruct(None, 2, len(sizes), 1), at(device, 256), weights)


@pytest.mark.parametrize("wrong", [None, "rows"])
def test_quantised_rows_of_another_device_are_refused(moe, wrong):
    x, q = at(0, (4, 64), torch.bfloat16), rows_on(1 if wrong else 0)
    for call in (lambda: moe.mx_quantize(x, q), lambda: moe.mx_dequantize(q, x)):
        if wrong:
            with pytest.raises(AssertionError):
                call()
        else:
            call()
    assert len(moe.lib.calls) == (0 if wrong else 2)


@pytest.mark.parametrize("wrong", [None, "rows", "list", "workspace", "strided workspace"])
def test_buffers_of_a_product_on_another_device_are_refused(moe, wrong):
    q, lst = rows_on(int(wrong == "rows")), list_on(int(wrong == "list"), (64, 32))
    ws = OnDevice(torch.zeros(2048, dtype=torch.uint8)[::2]) if wrong == "strided workspace" else at(int(wrong == "workspace"), 1024)
    args = (q, None, at(0, 3, torch.int32), lst, at(0, (4, 32), torch.float32), ws)
    if wrong:
        with pytest.raises(AssertionError):
            moe.mx_grouped_product(*args)
    else:
        moe.mx_grouped_product(*args)
    assert len(moe.lib.calls) == (0 if wrong else 1)


@pytest.mark.parametrize("wrong", [None, "list", "workspace"])
def test_buffers_of_the_layer_for_few_tokens_on_another_device_are_refused(moe, wrong):
    shape, lst = make_shape(4, 64, 128, 2, 1), list_on(int(wrong == "list"), (64, 128), (64, 128), (128, 64))
    args = (shape, at(0, (4, 64), torch.bfloat16), at(0, (64, 2), torch.bfloat16), None, lst, at(0, (4, 64), torch.bfloat16), at(int(wrong == "workspace"), 4096))
    if wrong:
        with pytest.raises(AssertionError):
            moe.layer_few(*args)
    else:
        moe.layer_few(*args)
    assert len(moe.lib.calls) == (0 if wrong else 1)


def test_rows_need_a_buffer_that_holds_them():
    n = int(binding.load_library().moe_mx_rows_bytes(4, 64))
    MxRows(4, 64, at(0, n))
    MxRows(0, 64, at(0, 0))
    for bad in (at(0, n - 1), torch.zeros(n, dtype=torch.uint8), at(0, n, torch.int8), OnDevice(torch.zeros(2 * n, dtype=torch.uint8)[::2])):
        with pytest.raises(AssertionError):
            MxRows(4, 64, bad)
