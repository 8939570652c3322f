"""Thin ctypes binding of libmoe_mi355.so (the C ABI declared in include/moe.h).

Argument marshalling only: torch supplies device memory and the current stream; every step
of the MoE expert module runs in the library's HIP kernels.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import List, Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmoe_mi355.so")

STATIC_WORKSPACE_BYTES = 32 << 20   # MOE_STATIC_WORKSPACE_BYTES of include/moe.h

STAGES = ["route", "permute_index", "permute_gather", "plan", "ffn_gate_up", "ffn_down", "combine"]

EXPORTS = [
    "moe_create", "moe_destroy", "moe_last_error", "moe_workspace_bytes", "moe_h_scratch_bytes", "moe_set_option", "moe_pack_weight",
    "moe_gate_packed_bytes", "moe_pack_gate",
    "moe_route", "moe_permute", "moe_grouped_ffn", "moe_combine", "moe_layer", "moe_layer_static", "moe_layer_views",
    "moe_layer_streamed", "moe_stream_stats", "moe_estimate_streamed_ms", "moe_accumulate", "moe_layer_chunked",
    "moe_backward_workspace_bytes", "moe_balance_loss", "moe_route_backward", "moe_combine_backward",
    "moe_gradient_list_bytes", "moe_gradient_list_make", "moe_clip_gradients",
    "moe_mx_rows_bytes", "moe_mx_weight_bytes", "moe_mx_quantize", "moe_mx_dequantize", "moe_mx_pack_weight", "moe_mx_unpack_weight",
    "moe_weight_list_bytes", "moe_weight_list_make", "moe_mx_workspace_bytes", "moe_mx_grouped_product", "moe_few_workspace_bytes", "moe_layer_few",
    "moe_profile_enable", "moe_profile_read", "moe_profile_read_intervals", "moe_profile_mfma_ceiling",
]


class MoeShape(C.Structure):
    _fields_ = [("T", C.c_int32), ("H", C.c_int32), ("F", C.c_int32), ("E", C.c_int32), ("top_k", C.c_int32),
                ("num_shared", C.c_int32), ("renormalize", C.c_int32), ("routed_scale", C.c_float)]


class GradientListStruct(C.Structure):
    _fields_ = [("buffer", C.c_void_p), ("chunks", C.c_int32), ("one_launch", C.c_int32)]


class WeightListStruct(C.Structure):
    _fields_ = [("buffer", C.c_void_p), ("experts", C.c_int32), ("matrices", C.c_int32), ("fp4", C.c_int32)]


class MoeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("moe status %d: %s" % (status, msg))
        self.status = status


_lib = None


def load_library():
    """Loads the in-tree library (building it first only if it does not exist yet)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from .build import build
        build()
    lib = C.CDLL(LIB_PATH)
    vp, i32p, f32p = C.c_void_p, C.c_void_p, C.c_void_p
    sp = C.POINTER(MoeShape)
    tab = C.POINTER(C.c_void_p)
    lib.moe_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
    lib.moe_destroy.argtypes = [C.c_void_p]
    lib.moe_destroy.restype = None
    lib.moe_last_error.argtypes = [C.c_void_p]
    lib.moe_last_error.restype = C.c_char_p
    lib.moe_workspace_bytes.argtypes = [sp]
    lib.moe_workspace_bytes.restype = C.c_size_t
    lib.moe_h_scratch_bytes.argtypes = [sp]
    lib.moe_h_scratch_bytes.restype = C.c_size_t
    lib.moe_gate_packed_bytes.argtypes = [sp]
    lib.moe_gate_packed_bytes.restype = C.c_size_t
    lib.moe_pack_gate.argtypes = [C.c_void_p, sp, vp, vp, vp]
    lib.moe_set_option.argtypes = [C.c_void_p, C.c_char_p, C.c_int32]
    lib.moe_pack_weight.argtypes = [C.c_void_p, vp, C.c_int32, C.c_int32, vp, vp]
    lib.moe_route.argtypes = [C.c_void_p, sp, vp, vp, f32p, i32p, f32p, f32p, vp, C.c_size_t, vp]
    lib.moe_permute.argtypes = [C.c_void_p, sp, vp, i32p, vp, i32p, i32p, i32p, i32p, vp, C.c_size_t, vp]
    lib.moe_grouped_ffn.argtypes = [C.c_void_p, sp, vp, i32p, vp, i32p, tab, tab, tab, vp, vp, vp, vp, C.c_size_t, vp]
    lib.moe_combine.argtypes = [C.c_void_p, sp, vp, i32p, f32p, vp, vp, vp]
    lib.moe_layer.argtypes = [C.c_void_p, sp, vp, vp, f32p, tab, tab, tab, vp, vp, C.c_size_t, vp]
    lib.moe_layer_static.argtypes = [C.c_void_p, sp, vp, vp, f32p, tab, tab, tab, vp, vp]
    lib.moe_layer_streamed.argtypes = [C.c_void_p, sp, vp, vp, f32p, tab, tab, tab, vp, C.c_size_t, C.c_int32, C.c_int32,
                                       vp, vp, C.c_size_t, vp]
    lib.moe_accumulate.argtypes = [C.c_void_p, vp, C.c_int32, C.c_int32, C.POINTER(C.c_int32), vp, C.c_int32, vp]
    lib.moe_layer_chunked.argtypes = [C.c_void_p, sp, vp, vp, f32p, tab, tab, tab, C.c_int32, vp, vp, C.c_size_t, vp]
    lib.moe_stream_stats.argtypes = [C.c_void_p, C.POINTER(C.c_uint64), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.moe_layer_views.argtypes = [sp, vp, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                    C.POINTER(C.c_void_p)]
    lib.moe_profile_enable.argtypes = [C.c_void_p, C.c_int32]
    lib.moe_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    lib.moe_profile_read_intervals.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_float), C.c_int32,
                                               C.POINTER(C.c_int32)]
    lib.moe_profile_mfma_ceiling.argtypes = [C.c_void_p, vp, vp, C.c_size_t, C.c_int32, vp, C.c_size_t,
                                             C.POINTER(C.c_double), C.POINTER(C.c_double), vp]
    lib.moe_estimate_streamed_ms.argtypes = [sp, C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.c_double, C.c_double]
    lib.moe_estimate_streamed_ms.restype = C.c_double
    lib.moe_backward_workspace_bytes.argtypes = [sp]
    lib.moe_backward_workspace_bytes.restype = C.c_size_t
    lib.moe_balance_loss.argtypes = [C.c_void_p, sp, f32p, i32p, vp, C.c_double, C.c_double, i32p, f32p, f32p, vp, C.c_size_t, vp]
    lib.moe_route_backward.argtypes = [C.c_void_p, sp, vp, vp, f32p, i32p, f32p, f32p, vp, vp, f32p, f32p, C.c_int32, vp, C.c_size_t, vp]
    lib.moe_combine_backward.argtypes = [C.c_void_p, sp, vp, vp, i32p, f32p, f32p, vp, vp]
    i64s, i32s = C.POINTER(C.c_int64), C.POINTER(C.c_int32)
    lib.moe_gradient_list_bytes.argtypes = [C.c_int32, i64s, i32s]
    lib.moe_gradient_list_bytes.restype = C.c_size_t
    lib.moe_gradient_list_make.argtypes = [C.c_void_p, C.c_int32, tab, tab, i64s, i32s, vp, C.c_size_t, C.POINTER(GradientListStruct), vp]
    lib.moe_clip_gradients.argtypes = [C.c_void_p, C.POINTER(GradientListStruct), C.c_double, f32p, vp]
    i32, ls = C.c_int32, C.POINTER(WeightListStruct)
    for name in ("moe_mx_rows_bytes", "moe_mx_weight_bytes", "moe_weight_list_bytes", "moe_mx_workspace_bytes"):
        getattr(lib, name).argtypes = [i32, i32]
        getattr(lib, name).restype = C.c_size_t
    lib.moe_mx_quantize.argtypes = [C.c_void_p, vp, i32, i32, i32, vp, vp]
    lib.moe_mx_dequantize.argtypes = [C.c_void_p, vp, i32, i32, vp, i32, vp]
    lib.moe_mx_pack_weight.argtypes = [C.c_void_p, vp, i32, i32, vp, vp]
    lib.moe_mx_unpack_weight.argtypes = [C.c_void_p, vp, i32, i32, vp, vp]
    lib.moe_weight_list_make.argtypes = [C.c_void_p, i32, i32, tab, i32, vp, C.c_size_t, ls, vp]
    lib.moe_mx_grouped_product.argtypes = [C.c_void_p, i32, i32, i32, vp, i32, i32p, i32p, ls, i32, i32, vp, i32, vp, C.c_size_t, vp]
    lib.moe_few_workspace_bytes.argtypes = [sp]
    lib.moe_few_workspace_bytes.restype = C.c_size_t
    lib.moe_layer_few.argtypes = [C.c_void_p, sp, vp, vp, f32p, ls, vp, vp, C.c_size_t, vp]
    for name in EXPORTS:
        if name not in ("moe_few_workspace_bytes", "moe_backward_workspace_bytes", "moe_gradient_list_bytes", "moe_mx_rows_bytes", "moe_mx_weight_bytes",
                        "moe_weight_list_bytes", "moe_mx_workspace_bytes",
                        "moe_destroy", "moe_last_error", "moe_workspace_bytes", "moe_h_scratch_bytes", "moe_gate_packed_bytes",
                        "moe_estimate_streamed_ms"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def make_shape(T, H, F, E, top_k, num_shared=0, renormalize=True, routed_scale=1.0) -> MoeShape:
    return MoeShape(int(T), int(H), int(F), int(E), int(top_k), int(num_shared), 1 if renormalize else 0,
                    float(routed_scale))


def shape_of(cfg) -> MoeShape:
    return make_shape(cfg.T, cfg.H, cfg.F, cfg.E, cfg.top_k, cfg.num_shared, cfg.renormalize, cfg.routed_scale)


def workspace_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_workspace_bytes(C.byref(shape)))


def h_scratch_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_h_scratch_bytes(C.byref(shape)))


def backward_workspace_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_backward_workspace_bytes(C.byref(shape)))


def estimate_streamed_ms(shape: MoeShape, rows_per_expert, experts_per_group: int, num_slots: int, link_gbs: float,
                         ffn_tflops: float) -> float:
    """Critical-path estimate of the expert phase of Moe.layer_streamed (host arithmetic)."""
    rows = (C.c_int32 * shape.E)(*[int(r) for r in rows_per_expert])
    return float(load_library().moe_estimate_streamed_ms(C.byref(shape), rows, experts_per_group, num_slots,
                                                         link_gbs, ffn_tflops))


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensor required"
    return C.c_void_p(t.data_ptr())


def _table(ws: Sequence[torch.Tensor]):
    for w in ws:
        assert w.is_cuda and w.is_contiguous()
    return (C.c_void_p * len(ws))(*[w.data_ptr() for w in ws])


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _typed(t: Optional[torch.Tensor], dtype, shape, device: int):
    """_ptr of a tensor that the call reads or writes as `shape` of `dtype` on its device.  Flat tensors and other leading dimensions will do,
    rows of another length will not."""
    if t is None:
        return None
    if t.dtype is dtype and (t.shape == shape or _same_rows(t, shape)) and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise AssertionError("contiguous tensor of %s, %s, on cuda:%d required" % (list(shape), dtype, device))


def _same_rows(t, shape) -> bool:
    return t.numel() == math.prod(shape) and (len(shape) == 1 or t.dim() < 2 or t.shape[-1] == shape[-1])


def _buffer(t: torch.Tensor, device: int):
    """Address of a buffer that the library alone knows the inside of, on the call's device."""
    if t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise AssertionError("contiguous buffer on cuda:%d required" % device)


def _float_type(t: torch.Tensor):
    return torch.float32 if t.dtype is torch.float32 else torch.bfloat16


def _raw_stream(device: int):
    """The device's current stream; torch.cuda.current_stream() makes an object for it, which takes longer than a small kernel's launch."""
    return torch._C._cuda_getCurrentRawStream(device)


class GradientList:
    """Tensors whose gradients are clipped together (Moe.gradient_list): keeps them and the device table alive."""

    def __init__(self, struct: GradientListStruct, buffer: torch.Tensor, grads, outs):
        self.struct, self.buffer, self.grads, self.outs = struct, buffer, grads, outs


class MxRows:
    """Rows in MXFP4 (Moe.mx_quantize): `rows` of `cols` values in one opaque buffer of moe_mx_rows_bytes bytes."""

    def __init__(self, rows: int, cols: int, buffer: torch.Tensor):
        n = int(load_library().moe_mx_rows_bytes(rows, cols))
        assert buffer.dtype is torch.uint8 and buffer.is_cuda and buffer.is_contiguous() and buffer.numel() >= n, "uint8 buffer of %d bytes on a GPU required" % n
        self.rows, self.cols, self.buffer, self.device = rows, cols, buffer, buffer.get_device()

    def address(self, device: int) -> int:
        """Of the buffer, for a call on `device`."""
        if device != self.device:
            raise AssertionError("rows on cuda:%d required" % device)
        return self.buffer.data_ptr()


class WeightList:
    """Expert matrices that calls find through a device table made once (Moe.weight_list): keeps them and the table alive."""

    def __init__(self, struct: WeightListStruct, buffer: torch.Tensor, weights):
        self.struct, self.buffer, self.weights, self.device = struct, buffer, weights, buffer.get_device()
        self.bytes = [ws[0].numel() * ws[0].element_size() for ws in weights]   # of a matrix, by its number


class Moe:
    """One library context on one GPU.  Methods mirror the C entry points one to one."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = device
        h = C.c_void_p()
        st = self.lib.moe_create(C.byref(h), device)
        if st != 0 or not h:
            raise MoeError(st, "moe_create failed on device %d" % device)
        self.h = h
        self.y_dtype, self.out_dtype = torch.float32, torch.bfloat16   # as options "y_fp32" and "out_fp32" have them
        self.gate_packed = False

    def close(self):
        if getattr(self, "h", None):
            self.lib.moe_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != 0:
            raise MoeError(st, self.lib.moe_last_error(self.h).decode())

    def set_option(self, key: str, value: int):
        self._check(self.lib.moe_set_option(self.h, key.encode(), int(value)))
        if key == "y_fp32":
            self.y_dtype = torch.float32 if value else torch.bfloat16
        elif key == "out_fp32":
            self.out_dtype = torch.float32 if value else torch.bfloat16
        elif key == "gate_packed":
            self.gate_packed = bool(value)

    def new_workspace(self, shape: MoeShape) -> torch.Tensor:
        n = workspace_bytes(shape)
        if n == 0:
            raise MoeError(2, "unsupported or invalid shape")
        return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device)

    # ---- one-time weight packing -------------------------------------------------------
    def new_h_scratch(self, shape: MoeShape) -> torch.Tensor:
        return torch.empty(h_scratch_bytes(shape), dtype=torch.uint8, device="cuda:%d" % self.device)

    def pack_weight(self, w: torch.Tensor) -> torch.Tensor:
        """Logical [K, N] weight -> packed form (opaque 1-D bf16 tensor of K*N elements)."""
        rows, cols = w.shape
        out = torch.empty(rows * cols, dtype=torch.bfloat16, device=w.device)
        self._check(self.lib.moe_pack_weight(self.h, _ptr(w), rows, cols, _ptr(out), _stream()))
        return out

    def pack_gate(self, shape, wg: torch.Tensor):
        """Packed gate matrix for option "gate_packed"."""
        n = int(self.lib.moe_gate_packed_bytes(C.byref(shape)))
        if n == 0:
            return None
        out = torch.empty(n // 2, dtype=torch.bfloat16, device=wg.device)
        self._check(self.lib.moe_pack_gate(self.h, C.byref(shape), _ptr(wg), _ptr(out), _stream()))
        return out

    def pack_experts(self, w1: Sequence[torch.Tensor], w3: Sequence[torch.Tensor], w2: Sequence[torch.Tensor]):
        return ([self.pack_weight(w) for w in w1], [self.pack_weight(w) for w in w3],
                [self.pack_weight(w) for w in w2])

    # ---- staged calls ------------------------------------------------------------------
    def route(self, shape, x, wg, bias, topk_idx, topk_w, logits, workspace):
        self._check(self.lib.moe_route(self.h, C.byref(shape), _ptr(x), _ptr(wg), _ptr(bias), _ptr(topk_idx),
                                       _ptr(topk_w), _ptr(logits), _ptr(workspace), workspace.numel(), _stream()))

    def permute(self, shape, x, topk_idx, x_perm, expert_offsets, perm, inv_perm, row_token, workspace):
        self._check(self.lib.moe_permute(self.h, C.byref(shape), _ptr(x), _ptr(topk_idx), _ptr(x_perm),
                                         _ptr(expert_offsets), _ptr(perm), _ptr(inv_perm), _ptr(row_token),
                                         _ptr(workspace), workspace.numel(), _stream()))

    def grouped_ffn(self, shape, x_perm, row_token, x, expert_offsets, w1p, w3p, w2p, h_scratch, y_perm, y_shared,
                    workspace):
        self._check(self.lib.moe_grouped_ffn(self.h, C.byref(shape), _ptr(x_perm), _ptr(row_token), _ptr(x),
                                             _ptr(expert_offsets), _table(w1p), _table(w3p), _table(w2p),
                                             _ptr(h_scratch), _ptr(y_perm), _ptr(y_shared), _ptr(workspace),
                                             workspace.numel(), _stream()))

    def combine(self, shape, y_perm, inv_perm, topk_w, y_shared, out):
        self._check(self.lib.moe_combine(self.h, C.byref(shape), _ptr(y_perm), _ptr(inv_perm), _ptr(topk_w),
                                         _ptr(y_shared), _ptr(out), _stream()))

    # ---- training a router ---------------------------------------------------------------
    def new_backward_workspace(self, shape: MoeShape) -> torch.Tensor:
        """Workspace of balance_loss and route_backward."""
        n = backward_workspace_bytes(shape)
        if n == 0:
            raise MoeError(2, "unsupported or invalid shape")
        return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device)

    def balance_loss(self, shape, logits, topk_idx, keep, balance_coef, z_coef, counts, loss, dlogits, workspace):
        """keep: bool [T] or None; dlogits: fp32 [T, E] or None."""
        T, E, d = shape.T, shape.E, self.device
        self._check(self.lib.moe_balance_loss(self.h, C.byref(shape), _typed(logits, torch.float32, (T, E), d),
                                              _typed(topk_idx, torch.int32, (T, shape.top_k), d), _typed(keep, torch.bool, (T,), d),
                                              balance_coef, z_coef, _typed(counts, torch.int32, (E,), d), _typed(loss, torch.float32, (2,), d),
                                              _typed(dlogits, torch.float32, (T, E), d), _ptr(workspace), workspace.numel(), _raw_stream(d)))

    def route_backward(self, shape, x, wg, logits, topk_idx, dtopk_w, dlogits, keep, dx, dwg, dbias, accumulate, workspace):
        """dlogits, keep (bool [T]), dx and dbias may be None."""
        T, H, E, k, d = shape.T, shape.H, shape.E, shape.top_k, self.device
        f32, b16 = torch.float32, torch.bfloat16
        self._check(self.lib.moe_route_backward(self.h, C.byref(shape), _typed(x, b16, (T, H), d), _typed(wg, b16, (H, E), d),
                                                _typed(logits, f32, (T, E), d), _typed(topk_idx, torch.int32, (T, k), d),
                                                _typed(dtopk_w, f32, (T, k), d), _typed(dlogits, f32, (T, E), d), _typed(keep, torch.bool, (T,), d),
                                                _typed(dx, b16, (T, H), d), _typed(dwg, f32, (H, E), d), _typed(dbias, f32, (E,), d),
                                                1 if accumulate else 0, _ptr(workspace), workspace.numel(), _raw_stream(d)))

    def combine_backward(self, shape, dout, y_perm, inv_perm, topk_w, dtopk_w, dy_perm):
        """dout as option "out_fp32" has it, y_perm and dy_perm (or None) as "y_fp32" has them."""
        T, H, k, d = shape.T, shape.H, shape.top_k, self.device
        f32, y, R = torch.float32, self.y_dtype, T * k
        self._check(self.lib.moe_combine_backward(self.h, C.byref(shape), _typed(dout, self.out_dtype, (T, H), d), _typed(y_perm, y, (R, H), d),
                                                  _typed(inv_perm, torch.int32, (R,), d), _typed(topk_w, f32, (T, k), d),
                                                  _typed(dtopk_w, f32, (T, k), d), _typed(dy_perm, y, (R, H), d), _raw_stream(d)))

    def gradient_list(self, grads: Sequence[torch.Tensor], outs: Sequence[torch.Tensor]) -> GradientList:
        """The tensors (fp32 or bf16) that clip_gradients takes together; outs[i] receives grads[i] scaled and may be it."""
        grads, outs = list(grads), list(outs)
        assert len(grads) == len(outs)
        for g, o in zip(grads, outs):
            assert g.dtype in (torch.float32, torch.bfloat16) and o.dtype == g.dtype and o.numel() == g.numel()
            assert g.get_device() == o.get_device() == self.device and g.is_contiguous() and o.is_contiguous()
        n = len(grads)
        sizes = (C.c_int64 * n)(*[g.numel() for g in grads])
        types = (C.c_int32 * n)(*[int(g.dtype == torch.float32) for g in grads])
        buffer = torch.empty(int(self.lib.moe_gradient_list_bytes(n, sizes, types)), dtype=torch.uint8, device="cuda:%d" % self.device)
        struct = GradientListStruct()
        self._check(self.lib.moe_gradient_list_make(self.h, n, _table(grads), _table(outs), sizes, types, _ptr(buffer),
                                                    buffer.numel(), C.byref(struct), _raw_stream(self.device)))
        return GradientList(struct, buffer, grads, outs)

    def clip_gradients(self, gradients: GradientList, max_norm: float, norm):
        self._check(self.lib.moe_clip_gradients(self.h, C.byref(gradients.struct), max_norm, _typed(norm, torch.float32, (1,), self.device), _raw_stream(self.device)))

    # ---- 4-bit expert weights --------------------------------------------------------------
    def new_mx_rows(self, rows: int, cols: int) -> MxRows:
        n = int(self.lib.moe_mx_rows_bytes(rows, cols))
        if n == 0 and not (rows == 0 and cols > 0 and cols % 32 == 0):
            raise MoeError(1, "rows of columns that are no multiple of 32, or 4 GiB of them")
        return MxRows(rows, cols, torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device))

    def new_mx_weight(self, rows: int, cols: int) -> torch.Tensor:
        n = int(self.lib.moe_mx_weight_bytes(rows, cols))
        if n == 0:
            raise MoeError(1, "a matrix whose rows or columns are no multiple of 32, or of 4 GiB")
        return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device)

    def mx_quantize(self, x, q: MxRows):
        """x: bf16 or fp32 [rows, cols]."""
        self._check(self.lib.moe_mx_quantize(self.h, _typed(x, _float_type(x), (q.rows, q.cols), self.device), int(x.dtype is torch.float32), q.rows, q.cols,
                                              q.address(self.device), _raw_stream(self.device)))

    def mx_dequantize(self, q: MxRows, out):
        """out: bf16 or fp32 [rows, cols]."""
        self._check(self.lib.moe_mx_dequantize(self.h, q.address(self.device), q.rows, q.cols, _typed(out, _float_type(out), (q.rows, q.cols), self.device),
                                                int(out.dtype is torch.float32), _raw_stream(self.device)))

    def mx_pack_weight(self, w: torch.Tensor, packed: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Logical bf16 [K, N] weight -> MXFP4 (opaque 1-D uint8 tensor, `packed` if given)."""
        rows, cols = w.shape
        if packed is None:
            packed = self.new_mx_weight(rows, cols)
        n = int(self.lib.moe_mx_weight_bytes(rows, cols))
        self._check(self.lib.moe_mx_pack_weight(self.h, _typed(w, torch.bfloat16, (rows, cols), self.device), rows, cols,
                                                 _typed(packed, torch.uint8, (n,), self.device), _raw_stream(self.device)))
        return packed

    def mx_unpack_weight(self, packed: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
        """The values of a packed weight as a logical bf16 [K, N] matrix, in `out`."""
        rows, cols = out.shape
        n = int(self.lib.moe_mx_weight_bytes(rows, cols))
        self._check(self.lib.moe_mx_unpack_weight(self.h, _typed(packed, torch.uint8, (n,), self.device), rows, cols,
                                                   _typed(out, torch.bfloat16, (rows, cols), self.device), _raw_stream(self.device)))
        return out

    def weight_list(self, *weights: Sequence[torch.Tensor]) -> WeightList:
        """One to three matrices of each expert (first all experts' first, ...), packed by mx_pack_weight (uint8) or pack_weight (bf16)."""
        weights = [list(ws) for ws in weights]
        assert weights and weights[0], "matrices required"
        kind = weights[0][0].dtype
        assert kind in (torch.uint8, torch.bfloat16)
        for ws in weights:
            assert len(ws) == len(weights[0]) and all(w.dtype is kind and w.numel() == ws[0].numel() and w.get_device() == self.device and w.is_contiguous() for w in ws)
        experts, matrices = len(weights[0]), len(weights)
        buffer = torch.empty(int(self.lib.moe_weight_list_bytes(experts, matrices)), dtype=torch.uint8, device="cuda:%d" % self.device)
        struct = WeightListStruct()
        self._check(self.lib.moe_weight_list_make(self.h, experts, matrices, _table([w for ws in weights for w in ws]), int(kind is torch.uint8),
                                                  _ptr(buffer), buffer.numel(), C.byref(struct), _raw_stream(self.device)))
        return WeightList(struct, buffer, weights)

    def new_mx_workspace(self, rows: int, experts: int) -> torch.Tensor:
        """Workspace of mx_grouped_product."""
        n = int(self.lib.moe_mx_workspace_bytes(rows, experts))
        if n == 0:
            raise MoeError(1, "invalid number of rows or experts")
        return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device)

    def mx_grouped_product(self, q: MxRows, row_index, expert_offsets, weights: WeightList, out, workspace, gated: bool = False, first: int = 0):
        """out: bf16 or fp32 [rows, N]; row_index: int32 [rows] or None; weights: matrices number `first` and, gated, the next of each expert."""
        d, (rows, N) = self.device, out.shape
        assert weights.device == d, "a list on cuda:%d required" % d
        n = int(self.lib.moe_mx_weight_bytes(q.cols, N))
        assert all(b == n for b in weights.bytes[first:first + 1 + bool(gated)]), "matrices of %d x %d in MXFP4 required" % (q.cols, N)
        self._check(self.lib.moe_mx_grouped_product(self.h, rows, q.cols, N, q.address(d), q.rows, _typed(row_index, torch.int32, (rows,), d),
                                                     _typed(expert_offsets, torch.int32, (weights.struct.experts + 1,), d), C.byref(weights.struct),
                                                     first, int(gated), _typed(out, _float_type(out), (rows, N), d), int(out.dtype is torch.float32),
                                                     _buffer(workspace, d), workspace.numel(), _raw_stream(d)))

    def new_few_workspace(self, shape: MoeShape) -> torch.Tensor:
        """Workspace of layer_few."""
        n = int(self.lib.moe_few_workspace_bytes(C.byref(shape)))
        if n == 0:
            raise MoeError(2, "a shape outside the limits of layer_few")
        return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % self.device)

    def layer_few(self, shape, x, wg, bias, weights: WeightList, out, workspace):
        """The whole layer for up to 16 tokens; weights: weight_list of the gate, up and down matrices, bf16 or MXFP4."""
        T, H, F, E, d = shape.T, shape.H, shape.F, shape.E, self.device
        fp4 = weights.struct.fp4
        assert weights.device == d, "a list on cuda:%d required" % d
        gate = (int(self.lib.moe_gate_packed_bytes(C.byref(shape))) // 2,) if self.gate_packed else (H, E)
        want = [int(self.lib.moe_mx_weight_bytes(*s)) if fp4 else 2 * H * F for s in ((H, F), (H, F), (F, H))]
        assert weights.bytes == want, "three matrices of %d x %d, %d x %d and %d x %d required" % (H, F, H, F, F, H)
        self._check(self.lib.moe_layer_few(self.h, C.byref(shape), _typed(x, torch.bfloat16, (T, H), d), _typed(wg, torch.bfloat16, gate, d),
                                           _typed(bias, torch.float32, (E,), d), C.byref(weights.struct), _typed(out, self.out_dtype, (T, H), d), _buffer(workspace, d), workspace.numel(),
                                           _raw_stream(d)))

    # ---- fused call --------------------------------------------------------------------
    def layer(self, shape, x, wg, bias, w1p, w3p, w2p, out, workspace, tables=None):
        t1, t3, t2 = tables if tables is not None else (_table(w1p), _table(w3p), _table(w2p))
        self._check(self.lib.moe_layer(self.h, C.byref(shape), _ptr(x), _ptr(wg), _ptr(bias), t1, t3, t2,
                                       _ptr(out), _ptr(workspace), workspace.numel(), _stream()))

    def layer_static(self, shape, x, wg, bias, w1p, w3p, w2p, out, tables=None):
        """moe_layer with the library's built-in scratch as workspace (allocates nothing)."""
        t1, t3, t2 = tables if tables is not None else (_table(w1p), _table(w3p), _table(w2p))
        self._check(self.lib.moe_layer_static(self.h, C.byref(shape), _ptr(x), _ptr(wg), _ptr(bias), t1, t3, t2,
                                              _ptr(out), _stream()))

    def layer_streamed(self, shape, x, wg, bias, host_w1p, host_w3p, host_w2p, slots, num_slots, experts_per_group,
                       out, workspace):
        """Expert weights in pinned HOST tensors (packed layout); `slots` is a device byte buffer
        cut into num_slots equal staging slots."""
        def host_table(ws):
            for w in ws:
                assert (not w.is_cuda) and w.is_pinned() and w.is_contiguous(), "pinned host tensor required"
            return (C.c_void_p * len(ws))(*[w.data_ptr() for w in ws])
        slot_bytes = (slots.numel() * slots.element_size() // num_slots) & ~255
        self._check(self.lib.moe_layer_streamed(self.h, C.byref(shape), _ptr(x), _ptr(wg), _ptr(bias),
                                                host_table(host_w1p), host_table(host_w3p), host_table(host_w2p),
                                                _ptr(slots), slot_bytes, num_slots, experts_per_group, _ptr(out),
                                                _ptr(workspace), workspace.numel(), _stream()))

    def layer_chunked(self, shape, x, wg, bias, w1p, w3p, w2p, max_tokens_per_pass, out, workspace, tables=None):
        t1, t3, t2 = tables if tables is not None else (_table(w1p), _table(w3p), _table(w2p))
        self._check(self.lib.moe_layer_chunked(self.h, C.byref(shape), _ptr(x), _ptr(wg), _ptr(bias), t1, t3, t2,
                                               max_tokens_per_pass, _ptr(out), _ptr(workspace), workspace.numel(),
                                               _stream()))

    def accumulate(self, staging, rows_filled: int, x_microbatch) -> int:
        """Appends x_microbatch's rows to staging at row rows_filled; returns the new fill count."""
        n = C.c_int32(rows_filled)
        self._check(self.lib.moe_accumulate(self.h, _ptr(staging), staging.shape[0], staging.shape[1], C.byref(n),
                                            _ptr(x_microbatch), x_microbatch.shape[0], _stream()))
        return n.value

    def stream_stats(self):
        b, g, k = C.c_uint64(), C.c_int32(), C.c_int32()
        self._check(self.lib.moe_stream_stats(self.h, C.byref(b), C.byref(g), C.byref(k)))
        return {"bytes_copied": b.value, "groups": g.value, "experts_skipped": k.value}

    def tables(self, w1p, w3p, w2p):
        """Pre-marshalled pointer tables, so a timed loop does not rebuild them per call."""
        return _table(w1p), _table(w3p), _table(w2p)

    def layer_views(self, shape, workspace):
        """Routing results of the last layer() call, as torch views into the workspace."""
        p = [C.c_void_p() for _ in range(4)]
        st = self.lib.moe_layer_views(C.byref(shape), _ptr(workspace), *[C.byref(q) for q in p])
        if st != 0:
            raise MoeError(st, "moe_layer_views")
        base = workspace.data_ptr()
        R = shape.T * shape.top_k

        def view(ptr, nbytes, dtype, shp):
            off = ptr.value - base
            return workspace[off:off + nbytes].view(dtype).view(*shp)
        return {
            "topk_idx": view(p[0], R * 4, torch.int32, (shape.T, shape.top_k)),
            "topk_w": view(p[1], R * 4, torch.float32, (shape.T, shape.top_k)),
            "expert_offsets": view(p[2], (shape.E + 1) * 4, torch.int32, (shape.E + 1,)),
            "inv_perm": view(p[3], R * 4, torch.int32, (R,)),
        }

    # ---- profiling ---------------------------------------------------------------------
    def profile_enable(self, on: bool):
        self._check(self.lib.moe_profile_enable(self.h, 1 if on else 0))

    def profile_read_intervals(self, capacity: int = 8192):
        """{stage name: [ms, ...]} of every interval recorded since the last read, in order."""
        st = (C.c_int32 * capacity)()
        ms = (C.c_float * capacity)()
        n = C.c_int32()
        self._check(self.lib.moe_profile_read_intervals(self.h, st, ms, capacity, C.byref(n)))
        out = {s: [] for s in STAGES}
        for i in range(n.value):
            out[STAGES[st[i]]].append(float(ms[i]))
        return out

    def mfma_ceiling(self, a, b, iters: int, sink):
        """One timed launch of the register-only MFMA loop; a, b: bf16 device tensors of equal size or None.
        Returns (TFLOP/s, ms)."""
        tf, ms = C.c_double(), C.c_double()
        nbytes = 0 if a is None else min(a.numel() * a.element_size(), b.numel() * b.element_size())
        self._check(self.lib.moe_profile_mfma_ceiling(self.h, _ptr(a), _ptr(b), nbytes, iters, _ptr(sink),
                                                      sink.numel() * sink.element_size(), C.byref(tf), C.byref(ms),
                                                      _stream()))
        return tf.value, ms.value

    def profile_read(self):
        ms = (C.c_double * len(STAGES))()
        n = (C.c_int32 * len(STAGES))()
        self._check(self.lib.moe_profile_read(self.h, ms, n))
        return {s: (ms[i], n[i]) for i, s in enumerate(STAGES)}
