"""The layer for up to 16 tokens in the forms that large layers run, against the definition in 64 bits."""
import pytest
import torch

from paper_2503_09716_amd import Moe, make_shape
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def moe():
    m = Moe(0)
    yield m
    m.close()


@pytest.fixture(autouse=True)
def options(moe):
    yield
    moe.set_option("out_fp32", 0)
    moe.set_option("gate_packed", 0)
    torch.cuda.empty_cache()


class Large(Layer):
    """A Layer whose inputs are made on the GPU."""

    def __init__(self, moe, T, H, F, E, k, shared, fp4, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)

        def normal(shape, std, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=gen)
        self.moe, self.T, self.k, self.E, self.shared, self.fp4 = moe, T, k, E, shared, fp4
        self.shape = make_shape(T, H, F, E, k, shared)
        self.x, self.wg, self.bias = normal((T, H), 1.0), normal((H, E), 2 / H ** 0.5), normal((E,), 0.3, torch.float32)
        self.packed, self.w = [], []
        for K, N in ((H, F), (H, F), (F, H)):
            made = [normal((K, N), 0.05) for _ in range(E + shared)]
            if fp4:
                self.packed.append([moe.mx_pack_weight(m) for m in made])
                self.w.append([moe.mx_unpack_weight(p, torch.empty_like(m)).double() for p, m in zip(self.packed[-1], made)])
            else:
                self.packed.append([moe.pack_weight(m) for m in made])
                self.w.append([m.double() for m in made])
        self.list = moe.weight_list(*self.packed)
        self.workspace = moe.new_few_workspace(self.shape)
        self.workspace.fill_(0xFF)   # NaN in whatever the call reads before it writes


# Down: 16, 64 or 128 columns to a workgroup (128: MXFP4, tasks x H / 64 >= 8192, H a multiple of 128).  Gate and up: x in LDS up to 80 KiB, and one item to a workgroup or
# several.  Weights past the caches where the list is above 256 MiB.
@pytest.mark.parametrize("T,H,F,E,k,shared,fp4", [
    (16, 2816, 1088, 64, 16, 0, True),      # 128 columns, x from memory, several items of 64 columns, past the caches
    (16, 2816, 1088, 64, 16, 0, False),     # the same on bf16: 64 columns
    (16, 2752, 1088, 64, 16, 0, True),      # as many tasks, but H is no multiple of 128
    (16, 2688, 192, 256, 16, 0, True),      # 128 columns, several items, through the caches
    (16, 2688, 192, 240, 16, 1, False),
    (7, 4096, 8256, 8, 4, 0, True),         # 128 columns, x in LDS, past the caches, columns behind the last 512
    (7, 4096, 8256, 8, 4, 0, False),
    (16, 2560, 192, 256, 16, 0, True),      # 128 columns, the most x that LDS takes, through the caches
    (3, 2560, 192, 254, 16, 2, True),       # and just below the border: 64 columns
    (16, 2048, 2816, 32, 16, 1, True),      # 64 columns, x in LDS, past the caches
    (16, 2752, 512, 256, 1, 0, True),       # 16 columns, x from memory, past the caches
    (16, 2752, 128, 256, 1, 0, False),
    (1, 2048, 704, 64, 2, 0, False),        # 16 columns, x in LDS, past the caches
    (16, 5120, 1536, 30, 6, 2, True),       # most of a wide layer
])
def test_forms_of_large_layers(moe, T, H, F, E, k, shared, fp4):
    Large(moe, T, H, F, E, k, shared, fp4, seed=H + F + E).check(packed_gate=True)


@pytest.mark.parametrize("fp4", [True, False])
def test_same_bits_whatever_was_left_in_the_workspace(moe, fp4):
    """Several items to a workgroup and several workgroups to the same columns, over and over."""
    a = Large(moe, 16, 2816, 704, 64, 16, 1, fp4, seed=7)
    want = a.run(True).clone()
    for fill in (0x00, 0xFF, 0x7F):
        a.workspace.fill_(fill)
        assert torch.equal(a.run(True), want)
