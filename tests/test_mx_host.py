"""Host side of 4-bit expert weights and of the layer for few tokens: sizes, and refusals that need no GPU."""
import ctypes as C

import pytest

from paper_2503_09716_amd import binding, make_shape


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def packed(rows, contraction):
    """Bytes of `rows` rows in MXFP4: codes in blocks of 128, scales in groups of 512 from the next multiple of 256 on."""
    codes = rows * -(-contraction // 128) * 64
    return -(-codes // 256) * 256 + rows * -(-contraction // 512) * 16


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (17, 1408), (5003, 2048), (1, 544), (0, 32)])
def test_bytes_of_rows(lib, rows, cols):
    assert lib.moe_mx_rows_bytes(rows, cols) == packed(rows, cols)


@pytest.mark.parametrize("K,N", [(32, 32), (64, 96), (1408, 2048), (4096, 14336), (544, 32)])
def test_bytes_of_weights(lib, K, N):
    assert lib.moe_mx_weight_bytes(K, N) == packed(N, K)


def test_sizes_that_are_refused(lib):
    for rows, cols in [(-1, 32), (4, 0), (4, -32), (4, 48), (4, 31), (1 << 30, 1 << 20)]:
        assert lib.moe_mx_rows_bytes(rows, cols) == 0
    for K, N in [(0, 32), (32, 0), (48, 32), (32, 40), (-32, 32), (1 << 17, 1 << 17), (65536, 32768)]:
        assert lib.moe_mx_weight_bytes(K, N) == 0
    assert lib.moe_mx_weight_bytes(65536, 32736) > 0                  # 2^32 - 2^22 bytes in bf16
    for rows, experts in [(-1, 4), (4, 0), (4, 257), (4, -1)]:
        assert lib.moe_mx_workspace_bytes(rows, experts) == 0
    for experts, matrices in [(0, 1), (257, 1), (4, 0), (4, 4), (-1, 1)]:
        assert lib.moe_weight_list_bytes(experts, matrices) == 0


def test_matrices_of_very_many_columns_are_refused(lib):
    assert lib.moe_mx_weight_bytes(32, (1 << 21) - 32) == packed((1 << 21) - 32, 32)
    assert lib.moe_mx_weight_bytes(32, 1 << 21) == 0 and lib.moe_mx_weight_bytes(32, 1 << 25) == 0


def test_workspace_bytes(lib):
    # a list entry of 16 bytes for 128 rows and for every expert, and the list's header
    for rows, experts in [(0, 1), (1, 1), (100000, 160), (1 << 24, 256)]:
        n = lib.moe_mx_workspace_bytes(rows, experts)
        assert n % 256 == 0 and n >= 256 + 16 * (rows // 128 + experts)
    assert lib.moe_weight_list_bytes(256, 3) >= 256 * 3 * 8


def test_few_workspace_bytes(lib):
    def size(*args, **kw):
        return lib.moe_few_workspace_bytes(C.byref(make_shape(*args, **kw)))
    # h as fp32 rows of the picks and the shared experts, the packed gate matrix
    assert size(16, 2048, 1408, 64, 6, 2) >= 16 * 8 * 1408 * 4 + 2048 * 64 * 2
    assert size(0, 64, 64, 4, 2) > 0 and size(1, 64, 64, 1, 1) > 0 and size(16, 32768, 64, 4, 2) > 0 and size(1, 64, 65536, 4, 2) > 0
    for bad in [(17, 64, 64, 4, 2), (4, 64, 64, 40, 17), (4, 96, 64, 4, 2), (4, 64, 100, 4, 2), (4, 32832, 64, 4, 2), (4, 64, 65600, 4, 2), (-1, 64, 64, 4, 2),
                (4, 64, 64, 2, 4), (4, 64, 64, 257, 2)]:
        assert size(*bad) == 0
    assert lib.moe_few_workspace_bytes(None) == 0


def test_calls_without_a_context_fail_cleanly(lib):
    s, listed = make_shape(4, 64, 64, 4, 2), binding.WeightListStruct()
    assert lib.moe_mx_quantize(None, None, 0, 4, 64, None, None) != 0
    assert lib.moe_mx_dequantize(None, None, 4, 64, None, 0, None) != 0
    assert lib.moe_mx_pack_weight(None, None, 64, 64, None, None) != 0
    assert lib.moe_mx_unpack_weight(None, None, 64, 64, None, None) != 0
    assert lib.moe_weight_list_make(None, 4, 1, None, 1, None, 0, C.byref(listed), None) != 0
    assert lib.moe_mx_grouped_product(None, 4, 64, 64, None, 4, None, None, C.byref(listed), 0, 0, None, 0, None, 0, None) != 0
    assert lib.moe_layer_few(None, C.byref(s), None, None, None, C.byref(listed), None, None, 0, None) != 0
    assert listed.buffer is None
