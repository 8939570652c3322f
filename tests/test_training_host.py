"""Host side of the calls that train a router: sizes, and refusals that need no GPU."""
import ctypes as C

from paper_2503_09716_amd import backward_workspace_bytes, binding, make_shape


def test_backward_workspace_bytes():
    s = make_shape(3001, 2048, 64, 64, 6)
    n = backward_workspace_bytes(s)
    steps = (3001 + 31) // 32
    assert n % 256 == 0 and n >= steps * 3 * 4 * 1024 + 2048 * 64 * 2     # dl's pieces and the gate matrix at least
    assert backward_workspace_bytes(make_shape(0, 64, 64, 4, 1)) > 0      # an empty batch is a valid shape
    for bad in [make_shape(-1, 64, 64, 4, 1), make_shape(8, 64, 64, 4, 5), make_shape(8, 60, 64, 4, 1), make_shape(8, 64, 72, 4, 1),
                make_shape(8, 64, 64, 300, 1), make_shape(8, 64, 64, 4, 1, num_shared=9)]:
        assert backward_workspace_bytes(bad) == 0
    # logits and dwg below 4 GiB
    assert backward_workspace_bytes(make_shape((1 << 22) - 1, 64, 64, 256, 1)) > 0
    assert backward_workspace_bytes(make_shape(1 << 22, 64, 64, 256, 1)) == 0
    assert backward_workspace_bytes(make_shape(1, (1 << 22) - 64, 64, 256, 1)) > 0
    assert backward_workspace_bytes(make_shape(1, 1 << 22, 64, 256, 1)) == 0


def test_gradient_list_bytes():
    lib = binding.load_library()

    def size(elements, types):
        n = len(elements)
        return lib.moe_gradient_list_bytes(n, (C.c_int64 * n)(*elements), (C.c_int32 * n)(*types))
    empty, one = size([], []), size([1], [1])
    assert 0 < empty < one
    assert size([1 << 20], [1]) > size([1 << 20], [0]) > one
    assert size([0, 0], [1, 0]) == empty
    assert size([-1], [1]) == 0 and size([4], [2]) == 0 and size([1 << 50], [1]) == 0 and size([1 << 40] * 40, [1] * 40) == 0
    assert lib.moe_gradient_list_bytes(-1, None, None) == 0 and lib.moe_gradient_list_bytes(1, None, None) == 0


def test_calls_without_a_context_fail_cleanly():
    lib = binding.load_library()
    s = make_shape(8, 64, 64, 4, 2)
    assert lib.moe_balance_loss(None, C.byref(s), None, None, None, 0.0, 0.0, None, None, None, None, 0, None) != 0
    assert lib.moe_route_backward(None, C.byref(s), *[None] * 10, 0, None, 0, None) != 0
    assert lib.moe_combine_backward(None, C.byref(s), *[None] * 7) != 0
    listed = binding.GradientListStruct()
    assert lib.moe_gradient_list_make(None, 0, None, None, None, None, None, 0, C.byref(listed), None) != 0
    assert lib.moe_clip_gradients(None, C.byref(listed), 1.0, None, None) != 0
    assert listed.buffer is None
