"""ctypes binding of libidkm.so: the same entry points as include/idkm.h, argument marshalling only.

PyTorch supplies device memory and the current HIP stream; every step of the
method runs inside the library's kernels.  There is no CPU fallback: if the
shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("IDKM_LIB", os.path.join(HERE, "libidkm.so"))

IDKM_OK = 0
STATUS_NAMES = {0: "IDKM_OK", 1: "IDKM_ERR_INVALID_ARG", 2: "IDKM_ERR_ALLOC", 3: "IDKM_ERR_DEVICE",
                4: "IDKM_ERR_NONFINITE", 5: "IDKM_ERR_NO_FORWARD", 6: "IDKM_ERR_UNSUPPORTED"}
DIST_L2, DIST_SQL2 = 0, 1
BWD_IMPLICIT, BWD_JFB, BWD_DENSE, BWD_GMRES = 0, 1, 2, 3
PATH_AUTO, PATH_STREAM, PATH_PERSISTENT = 0, 1, 2

EXPORTS = ["idkm_version", "idkm_limits", "idkm_status_string", "idkm_create", "idkm_destroy", "idkm_last_error",
           "idkm_set_path", "idkm_set_matrix_cores", "idkm_set_tile_limit", "idkm_set_spin_limit", "idkm_set_kernel_timing", "idkm_last_kernel_ms", "idkm_set_gmres_basis", "idkm_advance_sequence", "idkm_forward", "idkm_backward", "idkm_step_F", "idkm_step_JCT", "idkm_get_cotangents", "idkm_forward_noalloc", "idkm_noalloc_last_error",
           "idkm_calibrate", "idkm_code_bits", "idkm_code_words", "idkm_pack_codes", "idkm_unpack_quantize",
           "idkm_codes_linear_workspace", "idkm_codes_linear", "idkm_codes_linear_backward_workspace",
           "idkm_codes_linear_backward", "idkm_codes_linear_backward_kept", "idkm_keep8", "idkm_restore8",
           "idkm_int8_rows", "idkm_int8_linear_workspace", "idkm_int8_linear", "idkm_int8_linear_backward_workspace", "idkm_int8_linear_backward", "idkm_embedding", "idkm_embedding_backward_workspace", "idkm_embedding_backward",
           "idkm_codes_embedding", "idkm_codes_embedding_backward_workspace", "idkm_codes_embedding_backward", "idkm_group_scale", "idkm_group_unscale", "idkm_group_unscale_backward",
           "idkm_group_scale_backward", "idkm_distill_workspace", "idkm_distill",
           "idkm_batch_create", "idkm_batch_destroy", "idkm_batch_last_error", "idkm_batch_launches",
           "idkm_batch_context", "idkm_batch_forward", "idkm_batch_backward"]


class IdkmInfo(C.Structure):
    _fields_ = [("iters", C.c_int32), ("converged", C.c_int32), ("residual", C.c_double),
                ("empty_clusters", C.c_int32), ("path", C.c_int32), ("alpha", C.c_double)]


class IdkmFwdDesc(C.Structure):
    _fields_ = [("W", C.c_void_p), ("m", C.c_int64), ("d", C.c_int32), ("C0", C.c_void_p), ("k", C.c_int32),
                ("tau", C.c_float), ("tol", C.c_float), ("max_iter", C.c_int32), ("dist", C.c_int32),
                ("C_out", C.c_void_p), ("A_out", C.c_void_p), ("Wq_out", C.c_void_p), ("assign_out", C.c_void_p)]


class IdkmBwdDesc(C.Structure):
    _fields_ = [("dWq", C.c_void_p), ("mode", C.c_int32), ("tol", C.c_float), ("max_iter", C.c_int32),
                ("alpha", C.c_float), ("dW_out", C.c_void_p)]


class IdkmCodesDesc(C.Structure):
    _fields_ = [("words", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("C", C.c_void_p), ("k", C.c_int32),
                ("d", C.c_int32), ("S", C.c_void_p), ("group", C.c_int32), ("dtype", C.c_int32)]


class IdkmInt8Desc(C.Structure):
    _fields_ = [("W8", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ldw", C.c_int64), ("scale", C.c_void_p), ("dtype", C.c_int32)]


class IdkmLimits(C.Structure):
    _fields_ = [("max_k", C.c_int32), ("max_d", C.c_int32), ("max_kd", C.c_int32)]


class IdkmError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {detail}")
        self.status = status
        self.detail = detail


_lib = None


def load_library():
    """dlopen libidkm.so (built in-tree by paper_2312_07759_amd.build).  Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2312_07759_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, f32p, i32p = C.c_void_p, C.c_void_p, C.c_void_p
    lib.idkm_version.restype = C.c_int32
    lib.idkm_limits.argtypes = [C.POINTER(IdkmLimits)]
    lib.idkm_limits.restype = None
    lib.idkm_status_string.argtypes = [C.c_int]
    lib.idkm_status_string.restype = C.c_char_p
    lib.idkm_create.argtypes = [C.POINTER(vp), C.c_int]
    lib.idkm_create.restype = C.c_int
    lib.idkm_destroy.argtypes = [vp]
    lib.idkm_destroy.restype = C.c_int
    lib.idkm_last_error.argtypes = [vp]
    lib.idkm_last_error.restype = C.c_char_p
    lib.idkm_set_path.argtypes = [vp, C.c_int]
    lib.idkm_set_path.restype = C.c_int
    lib.idkm_set_tile_limit.argtypes = [vp, C.c_int64]
    lib.idkm_set_tile_limit.restype = C.c_int
    lib.idkm_set_matrix_cores.argtypes = [vp, C.c_int32]
    lib.idkm_set_matrix_cores.restype = C.c_int
    lib.idkm_set_spin_limit.argtypes = [vp, C.c_uint32]
    lib.idkm_set_spin_limit.restype = C.c_int
    lib.idkm_set_kernel_timing.argtypes = [vp, C.c_int32]
    lib.idkm_set_kernel_timing.restype = C.c_int
    lib.idkm_last_kernel_ms.argtypes = [vp, C.POINTER(C.c_float)]
    lib.idkm_last_kernel_ms.restype = C.c_int
    lib.idkm_advance_sequence.argtypes = [vp, C.c_uint32, vp]
    lib.idkm_advance_sequence.restype = C.c_int
    lib.idkm_set_gmres_basis.argtypes = [vp, C.c_int32]
    lib.idkm_set_gmres_basis.restype = C.c_int
    lib.idkm_forward.argtypes = [vp, f32p, C.c_int64, C.c_int32, f32p, C.c_int32, C.c_float, C.c_float, C.c_int32,
                                 C.c_int, f32p, f32p, f32p, i32p, C.POINTER(IdkmInfo), vp]
    lib.idkm_forward.restype = C.c_int
    lib.idkm_backward.argtypes = [vp, f32p, C.c_int, C.c_float, C.c_int32, C.c_float, f32p, C.POINTER(IdkmInfo), vp]
    lib.idkm_backward.restype = C.c_int
    lib.idkm_step_F.argtypes = [vp, f32p, C.c_int64, C.c_int32, f32p, C.c_int32, C.c_float, C.c_int, f32p, f32p, vp]
    lib.idkm_step_F.restype = C.c_int
    lib.idkm_step_JCT.argtypes = [vp, f32p, f32p, vp]
    lib.idkm_step_JCT.restype = C.c_int
    lib.idkm_forward_noalloc.argtypes = [C.c_int, f32p, C.c_int64, C.c_int32, f32p, C.c_int32, C.c_float, C.c_float,
                                         C.c_int32, C.c_int, f32p, f32p, f32p, i32p, C.POINTER(IdkmInfo), vp]
    lib.idkm_forward_noalloc.restype = C.c_int
    lib.idkm_noalloc_last_error.argtypes = []
    lib.idkm_noalloc_last_error.restype = C.c_char_p
    lib.idkm_get_cotangents.argtypes = [vp, vp, vp, vp]
    lib.idkm_get_cotangents.restype = C.c_int
    lib.idkm_calibrate.argtypes = [vp, C.c_int32, f32p, C.c_int64, C.POINTER(C.c_double), vp]
    lib.idkm_calibrate.restype = C.c_int
    lib.idkm_code_bits.argtypes = [C.c_int32]
    lib.idkm_code_bits.restype = C.c_int32
    lib.idkm_code_words.argtypes = [C.c_int64, C.c_int32]
    lib.idkm_code_words.restype = C.c_int64
    lib.idkm_pack_codes.argtypes = [vp, i32p, C.c_int64, C.c_int32, vp, vp]
    lib.idkm_pack_codes.restype = C.c_int
    lib.idkm_unpack_quantize.argtypes = [vp, vp, C.c_int64, f32p, C.c_int32, C.c_int32, f32p, vp]
    lib.idkm_unpack_quantize.restype = C.c_int
    i64, i32, desc = C.c_int64, C.c_int32, C.POINTER(IdkmCodesDesc)
    lib.idkm_codes_linear_workspace.argtypes = [desc, i64]
    lib.idkm_codes_linear_workspace.restype = i64
    lib.idkm_codes_linear.argtypes = [vp, desc, vp, i64, i64, vp, i64, vp, i64, vp]
    lib.idkm_codes_linear.restype = C.c_int
    lib.idkm_codes_linear_backward_workspace.argtypes = [desc, i64]
    lib.idkm_codes_linear_backward_workspace.restype = i64
    lib.idkm_codes_linear_backward.argtypes = [vp, desc, vp, i64, vp, i64, i64, vp, i64, vp, vp, vp, i64, vp]
    lib.idkm_codes_linear_backward.restype = C.c_int
    f32, int8 = C.c_float, C.POINTER(IdkmInt8Desc)
    lib.idkm_int8_rows.argtypes = [vp, vp, i64, i64, i64, C.c_int, vp, i64, vp, vp]
    lib.idkm_int8_rows.restype = C.c_int
    for name in ("idkm_int8_linear_workspace", "idkm_int8_linear_backward_workspace"):
        getattr(lib, name).argtypes = [int8, i64]
        getattr(lib, name).restype = i64
    lib.idkm_int8_linear.argtypes = [vp, int8, vp, i64, i64, vp, i64, vp, i64, vp]
    lib.idkm_int8_linear.restype = C.c_int
    lib.idkm_int8_linear_backward.argtypes = [vp, int8, vp, i64, i64, vp, i64, vp, i64, vp]
    lib.idkm_int8_linear_backward.restype = C.c_int
    lib.idkm_codes_linear_backward_kept.argtypes = [vp, desc, vp, vp, vp, i64, i64, vp, i64, vp, vp, vp, i64, vp]
    lib.idkm_codes_linear_backward_kept.restype = C.c_int
    lib.idkm_keep8.argtypes = [vp, vp, i64, i64, i64, C.c_int, vp, vp, vp]
    lib.idkm_keep8.restype = C.c_int
    lib.idkm_restore8.argtypes = [vp, vp, vp, i64, i64, C.c_int, vp, i64, vp]
    lib.idkm_restore8.restype = C.c_int
    lib.idkm_embedding.argtypes = [vp, vp, i64, i64, vp, i32, i64, f32, vp, i64, C.c_int, vp]
    lib.idkm_embedding.restype = C.c_int
    lib.idkm_embedding_backward_workspace.argtypes = [i64, i64, i64]
    lib.idkm_embedding_backward_workspace.restype = i64
    lib.idkm_embedding_backward.argtypes = [vp, i64, i64, vp, i32, i64, f32, vp, i64, C.c_int, vp, vp, i64, vp]
    lib.idkm_embedding_backward.restype = C.c_int
    lib.idkm_codes_embedding.argtypes = [vp, desc, vp, i32, i64, f32, vp, i64, vp]
    lib.idkm_codes_embedding.restype = C.c_int
    lib.idkm_codes_embedding_backward_workspace.argtypes = [desc, i64]
    lib.idkm_codes_embedding_backward_workspace.restype = i64
    lib.idkm_codes_embedding_backward.argtypes = [vp, desc, vp, i32, i64, f32, vp, i64, vp, vp, vp, i64, vp]
    lib.idkm_codes_embedding_backward.restype = C.c_int
    lib.idkm_group_scale.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp]
    lib.idkm_group_scale.restype = C.c_int
    lib.idkm_group_unscale.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp]
    lib.idkm_group_unscale.restype = C.c_int
    lib.idkm_group_unscale_backward.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, vp]
    lib.idkm_group_unscale_backward.restype = C.c_int
    lib.idkm_group_scale_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, vp]
    lib.idkm_group_scale_backward.restype = C.c_int
    lib.idkm_distill_workspace.argtypes = [i64, i64, i32, i32]
    lib.idkm_distill_workspace.restype = i64
    lib.idkm_distill.argtypes = [vp, vp, i64, i64, i64, C.c_int, vp, vp, i32, C.c_float, vp, vp, vp, vp, i64, vp, i64, vp]
    lib.idkm_distill.restype = C.c_int
    lib.idkm_batch_create.argtypes = [C.POINTER(vp), C.c_int, C.c_int32]
    lib.idkm_batch_create.restype = C.c_int
    lib.idkm_batch_destroy.argtypes = [vp]
    lib.idkm_batch_destroy.restype = C.c_int
    lib.idkm_batch_last_error.argtypes = [vp]
    lib.idkm_batch_last_error.restype = C.c_char_p
    lib.idkm_batch_launches.argtypes = [vp]
    lib.idkm_batch_launches.restype = C.c_int32
    lib.idkm_batch_context.argtypes = [vp, C.c_int32]
    lib.idkm_batch_context.restype = vp
    lib.idkm_batch_forward.argtypes = [vp, C.POINTER(IdkmFwdDesc), C.c_int32, C.POINTER(IdkmInfo), C.POINTER(C.c_int), vp]
    lib.idkm_batch_forward.restype = C.c_int
    lib.idkm_batch_backward.argtypes = [vp, C.POINTER(IdkmBwdDesc), C.c_int32, C.POINTER(IdkmInfo), C.POINTER(C.c_int), vp]
    lib.idkm_batch_backward.restype = C.c_int
    _lib = lib
    return lib


@dataclass
class Info:
    iters: int
    converged: bool
    residual: float
    empty_clusters: int
    path: int
    alpha: float


def _info(i: IdkmInfo) -> Info:
    return Info(int(i.iters), bool(i.converged), float(i.residual), int(i.empty_clusters), int(i.path), float(i.alpha))


def _ptr(t, dtype, shape, name):
    """Device pointer of a contiguous torch tensor after checking dtype/shape/device."""
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor in device memory")
    if t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise TypeError(f"{name} must be contiguous {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


F32, F16, BF16 = 0, 1, 2


_torch = None


def _t():
    """The torch module; this package loads without it."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _dtype(t, name):
    torch = _t()
    dt = t.dtype
    if dt is torch.bfloat16:
        return BF16
    if dt is torch.float32:
        return F32
    if dt is torch.float16:
        return F16
    raise TypeError(f"{name} must be float32, float16 or bfloat16, got {dt}")


def _rows(t, dtype, width, device, name):
    """Checks a matrix [n, width] on `device` whose rows may lie further apart than their length; elements between rows."""
    if not isinstance(t, _t().Tensor) or t.get_device() != device:
        raise TypeError(f"{name} must be in the memory of device {device}")
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 2 or shape[1] != width:
        raise TypeError(f"{name} must be {dtype} of shape (n, {width}), got {t.dtype} {tuple(shape)}")
    ld, step = t.stride()
    if shape[0] < 2:
        ld = width
    if (width > 1 and step != 1) or ld < width:
        raise TypeError(f"{name} must have contiguous rows that do not overlap")
    return ld


def _flat(t, dtype, shape, device, name):
    """Address of a contiguous tensor of this type and shape on `device`."""
    if not isinstance(t, _t().Tensor) or t.get_device() != device:
        raise TypeError(f"{name} must be in the memory of device {device}")
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


class CodesLayer:
    """A [rows, cols] layer in its stored form: `words` of Context.pack_codes of its rows' codes, one row after another, the
    codebook C [k,d] in the type of the activations, and optionally float32 scales S [rows, ceil(cols / group)] of groups of
    `group` weights of a row.  Holds the tensors; they may be changed in place between calls (not `words`' meaning)."""

    def __init__(self, words, rows, cols, Cb, S=None, group=0):
        import torch
        k, d = Cb.shape
        rows, cols, group = int(rows), int(cols), int(group)
        if cols < 1 or rows < 1 or cols % d:
            raise ValueError(f"rows and cols must be at least 1 and cols a multiple of d = {d}, got {rows} x {cols}")
        if (S is None) != (group == 0) or group < 0:
            raise ValueError("scales and their group go together")
        if S is not None and group < cols and (group % 32 or group % d):
            raise ValueError("a group shorter than a row must be a multiple of 32 and of d")
        self.dtype, self.code = Cb.dtype, _dtype(Cb, "C")
        self.device = Cb.get_device()
        p = _ptr(Cb, Cb.dtype, (k, d), "C")
        nwords = code_words(rows * cols // d, k)
        if nwords < 0:
            raise ValueError(f"a codebook of {k} codewords is not supported")
        w = _ptr(words, torch.int32, (nwords,), "words")
        groups = -(-cols // group) if group else 0
        s = _ptr(S, torch.float32, (rows, groups), "S")
        for t in (words, S):
            if t is not None and t.device.index != self.device:
                raise TypeError("words, C and S must be on one device")
        self.rows, self.cols, self.k, self.d, self.group, self.groups = rows, cols, k, d, group, groups
        self.words, self.C, self.S = words, Cb, S
        self._desc = IdkmCodesDesc(w, rows, cols, p, k, d, s, min(group, 2**31 - 1), self.code)
        self._at = C.byref(self._desc)
        self._bytes = {}  # workspace sizes by (call, tokens)

    def workspace_bytes(self, n, backward=False, lookup=False):
        """Bytes that codes_linear (or codes_linear_backward, or codes_embedding_backward) of n tokens works in; raises for a layer it refuses."""
        key = (n, backward, lookup)
        b = self._bytes.get(key)
        if b is None:
            lib = load_library()
            b = (lib.idkm_codes_embedding_backward_workspace if lookup else
                 lib.idkm_codes_linear_backward_workspace if backward else lib.idkm_codes_linear_workspace)(self._at, n)
            if len(self._bytes) > 4096:
                self._bytes.clear()
            self._bytes[key] = b
        return b


class Kept8:
    """Activations [n, cols] of `dtype` in 8 bits, as Context.keep8 gives them: Q int8 [n, 32 b] and the powers of two E uint8 [n, b] of
    blocks of 32 columns, b = ceil(cols / 32)."""

    def __init__(self, Q, E, cols, dtype):
        torch, blocks = _t(), -(-cols // 32)
        if Q.dim() != 2 or Q.dtype is not torch.int8 or Q.shape[1] != 32 * blocks or not Q.is_contiguous() or not Q.is_cuda:
            raise TypeError(f"Q must be contiguous int8 of shape (n, {32 * blocks}) in device memory")
        if E.dtype is not torch.uint8 or E.shape != (Q.shape[0], blocks) or not E.is_contiguous() or E.device != Q.device:
            raise TypeError(f"E must be contiguous uint8 of shape {(Q.shape[0], blocks)} beside Q")
        self.Q, self.E, self.cols, self.dtype = Q, E, cols, dtype
        self.code = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}.get(dtype)
        if self.code is None:
            raise TypeError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
        self.device, self.shape = Q.get_device(), (Q.shape[0], cols)


class Int8Layer:
    """A [rows, cols] layer in 8-bit integers W8 (int8) with a float32 scale [rows] for each row, for activations of `dtype`.  Context.int8_layer
    makes one of weights or of a stored layer.  The integers are laid out here, once, in whole steps of 128 columns; W8 itself is used where it has those
    and is aligned (and may then be changed in place, as may the scales).  cols: of W8's columns the first `cols` are the layer's."""

    def __init__(self, W8, scale, dtype, cols=None):
        torch = _t()
        if not isinstance(W8, torch.Tensor) or not W8.is_cuda or W8.dtype is not torch.int8 or W8.dim() != 2 or not W8.is_contiguous():
            raise TypeError("W8 must be a contiguous int8 matrix in device memory")
        rows, width = W8.shape
        cols = width if cols is None else int(cols)
        if rows < 1 or not 1 <= cols <= width:
            raise ValueError(f"rows and cols must be at least 1, got {rows} x {cols} of {width}")
        self.code = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}.get(dtype)
        if self.code is None:
            raise TypeError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
        self.device, self.dtype, self.rows, self.cols = W8.get_device(), dtype, rows, cols
        s = _flat(scale, torch.float32, (rows,), self.device, "scale")
        if width % 128 or W8.data_ptr() % 16:
            laid = W8.new_zeros(rows, -(-cols // 128) * 128)
            laid[:, :cols] = W8[:, :cols]
            W8 = laid
        self.W8, self.scale = W8, scale
        self._desc = IdkmInt8Desc(W8.data_ptr(), rows, cols, W8.shape[1], s, self.code)
        self._at = C.byref(self._desc)
        self._bytes = {}  # workspace sizes by (tokens, backward)
        if load_library().idkm_int8_linear_workspace(self._at, 0) < 0:
            raise ValueError(f"a layer of {rows} x {cols} is not supported")

    def workspace_bytes(self, n, backward=False):
        key = (n, backward)
        b = self._bytes.get(key)
        if b is None:
            lib = load_library()
            b = (lib.idkm_int8_linear_backward_workspace if backward else lib.idkm_int8_linear_workspace)(self._at, n)
            if len(self._bytes) > 4096:
                self._bytes.clear()
            self._bytes[key] = b
        return b


class Context:
    """Owns an idkm_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, device: int = 0):
        self._lib = load_library()
        h = C.c_void_p()
        st = self._lib.idkm_create(C.byref(h), int(device))
        if st != IDKM_OK:
            raise IdkmError(st, "idkm_create failed")
        self._h = h
        self.device = int(device)
        self._keep = None
        self._distill_bytes = {}  # workspace sizes by shape

    def close(self):
        if getattr(self, "_h", None):
            self._lib.idkm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != IDKM_OK:
            raise IdkmError(st, self._lib.idkm_last_error(self._h).decode())

    def set_path(self, path: int):
        self._check(self._lib.idkm_set_path(self._h, int(path)))

    def set_tile_limit(self, nbytes: int):
        self._check(self._lib.idkm_set_tile_limit(self._h, int(nbytes)))

    def set_matrix_cores(self, enable: bool):
        self._check(self._lib.idkm_set_matrix_cores(self._h, 1 if enable else 0))

    def advance_sequence(self, n: int):
        self._check(self._lib.idkm_advance_sequence(self._h, int(n), _stream()))

    def set_gmres_basis(self, basis: int):
        self._check(self._lib.idkm_set_gmres_basis(self._h, int(basis)))

    def set_kernel_timing(self, enable: bool):
        self._check(self._lib.idkm_set_kernel_timing(self._h, 1 if enable else 0))

    def last_kernel_ms(self) -> float:
        """idkm_last_kernel_ms: event time of the last persistent launch (needs set_kernel_timing(True))."""
        ms = C.c_float()
        self._check(self._lib.idkm_last_kernel_ms(self._h, C.byref(ms)))
        return float(ms.value)

    def set_spin_limit(self, polls: int):
        self._check(self._lib.idkm_set_spin_limit(self._h, int(polls)))

    def forward(self, W, C0, tau, tol, max_iter, dist, want_A=False, want_Wq=True, want_assign=False, out=None):
        """idkm_forward.  W [m,d], C0 [k,d] float32 device tensors.  Returns dict(C, A, Wq, assign, info).
        `out` may hold preallocated tensors under the keys C, A, Wq, assign (as a training loop would keep them)."""
        import torch
        m, d = W.shape
        k = C0.shape[0]
        dev = W.device
        out = out or {}
        Cout = out.get("C")
        if Cout is None:
            Cout = torch.empty((k, d), dtype=torch.float32, device=dev)
        A = out.get("A") if want_A else None
        if want_A and A is None:
            A = torch.empty((m, k), dtype=torch.float32, device=dev)
        Wq = out.get("Wq") if want_Wq else None
        if want_Wq and Wq is None:
            Wq = torch.empty((m, d), dtype=torch.float32, device=dev)
        asg = out.get("assign") if want_assign else None
        if want_assign and asg is None:
            asg = torch.empty((m,), dtype=torch.int32, device=dev)
        info = IdkmInfo()
        st = self._lib.idkm_forward(self._h, _ptr(W, torch.float32, (m, d), "W"), m, d,
                                    _ptr(C0, torch.float32, (k, d), "C0"), k, float(tau), float(tol), int(max_iter),
                                    int(dist), _ptr(Cout, torch.float32, (k, d), "C_out"),
                                    _ptr(A, torch.float32, (m, k), "A_out"), _ptr(Wq, torch.float32, (m, d), "Wq_out"),
                                    _ptr(asg, torch.int32, (m,), "assign_out"), C.byref(info), _stream())
        self._check(st)
        self._keep = W  # the library borrows W until backward
        return dict(C=Cout, A=A, Wq=Wq, assign=asg, info=_info(info))

    def backward(self, dWq, mode, tol=1e-6, max_iter=1000, alpha=1.0, out=None):
        """idkm_backward.  dWq [m,d] float32 device tensor.  Returns dict(dW, info); `out` may be a preallocated dW."""
        import torch
        dW = out if out is not None else torch.empty_like(dWq)
        info = IdkmInfo()
        st = self._lib.idkm_backward(self._h, _ptr(dWq, torch.float32, dWq.shape, "dWq"), int(mode), float(tol),
                                     int(max_iter), float(alpha), _ptr(dW, torch.float32, dWq.shape, "dW_out"),
                                     C.byref(info), _stream())
        self._check(st)
        return dict(dW=dW, info=_info(info))

    def get_cotangents(self, k, d):
        """idkm_get_cotangents: (v, g) of the last backward as float64 numpy arrays [k,d]."""
        import numpy as np
        v = np.empty((k, d), dtype=np.float64)
        g = np.empty((k, d), dtype=np.float64)
        self._check(self._lib.idkm_get_cotangents(self._h, v.ctypes.data_as(C.c_void_p), g.ctypes.data_as(C.c_void_p),
                                                  _stream()))
        return v, g

    def calibrate(self, kind, buf=None):
        """idkm_calibrate: 0 lane-ops/s, 1 exponentials/s, 2 bytes/s of a streaming read of `buf` (float32 tensor),
        3-5 exponentials/s beside 1, 2, 4 FMAs, 6-8 float32 matrix multiply-adds/s (16x16x4, 16x16x4 with vector FMAs
        between, 4x4x1)."""
        import torch
        r = C.c_double()
        n = 0 if buf is None else buf.numel()
        ptr = None if buf is None else _ptr(buf, torch.float32, buf.shape, "buf")
        self._check(self._lib.idkm_calibrate(self._h, int(kind), ptr, n, C.byref(r), _stream()))
        return float(r.value)

    def pack_codes(self, assign, k):
        """idkm_pack_codes: int32 [m] device tensor -> int32 tensor holding the uint32 words of the b-bit stream."""
        import torch
        m = assign.shape[0]
        words = torch.empty((max(code_words(m, k), 0),), dtype=torch.int32, device=assign.device)
        st = self._lib.idkm_pack_codes(self._h, _ptr(assign, torch.int32, (m,), "assign"), m, int(k),
                                       C.c_void_p(words.data_ptr()), _stream())
        self._check(st)
        return words

    def unpack_quantize(self, words, m, Cb):
        """idkm_unpack_quantize: stream words + codebook [k,d] -> q(W, C) [m,d]."""
        import torch
        k, d = Cb.shape
        out = torch.empty((m, d), dtype=torch.float32, device=Cb.device)
        st = self._lib.idkm_unpack_quantize(self._h, _ptr(words, torch.int32, (code_words(m, k),), "words"), m,
                                            _ptr(Cb, torch.float32, (k, d), "C"), k, d,
                                            _ptr(out, torch.float32, (m, d), "Wh_out"), _stream())
        self._check(st)
        return out

    def _raw_stream(self):
        """The current stream of this context's device, which need not be the current device."""
        return _t()._C._cuda_getCurrentRawStream(self.device)

    def codes_linear(self, layer, X, out=None):
        """idkm_codes_linear: X [n, cols] in the layer's type -> X w^T [n, rows].  Rows of X and `out` may lie apart."""
        dev = self.device
        if layer.device != dev:
            raise TypeError(f"the layer must be in the memory of device {dev}")
        ldx = _rows(X, layer.dtype, layer.cols, dev, "X")
        n = X.shape[0]
        if out is None:
            out = X.new_empty(n, layer.rows)
            ldy = layer.rows
        else:
            ldy = _rows(out, layer.dtype, layer.rows, dev, "out")
            if out.shape[0] != n:
                raise TypeError(f"out must have {n} rows")
        need = layer.workspace_bytes(n)
        ws = X.new_empty(need, dtype=_t().uint8) if need > 0 else None
        st = self._lib.idkm_codes_linear(self._h, layer._at, X.data_ptr(), n, ldx, out.data_ptr(), ldy,
                                         ws.data_ptr() if need > 0 else None, need, self._raw_stream())
        if st:
            self._check(st)
        return out

    def codes_linear_backward(self, layer, X, dY, want_dX=True, want_dC=True, want_dS=True):
        """idkm_codes_linear_backward: dict of dX [n, cols] in the layer's type and float32 dC [k, d] and, for a layer with
        scales, dS [rows, groups].  X may be None if only dX is wanted, and may be a Kept8."""
        torch, dev = _t(), self.device
        if layer.device != dev:
            raise TypeError(f"the layer must be in the memory of device {dev}")
        ldy = _rows(dY, layer.dtype, layer.rows, dev, "dY")
        n = dY.shape[0]
        want_dS = want_dS and layer.S is not None
        ldx, kept = 0, isinstance(X, Kept8)
        if X is not None:
            if not kept:
                ldx = _rows(X, layer.dtype, layer.cols, dev, "X")
            elif X.dtype is not layer.dtype or X.cols != layer.cols or X.device != dev:
                raise TypeError(f"X must be {layer.dtype} of shape (n, {layer.cols}), kept in the memory of device {dev}")
            if X.shape[0] != n:
                raise TypeError(f"X must have {n} rows")
        elif want_dC or want_dS:
            raise TypeError("X is needed for dC and dS")
        res = {}
        if want_dX:
            res["dX"] = dY.new_empty(n, layer.cols)
        if want_dC:
            res["dC"] = dY.new_empty(layer.k, layer.d, dtype=torch.float32)
        if want_dS:
            res["dS"] = dY.new_empty(layer.rows, layer.groups, dtype=torch.float32)
        need = layer.workspace_bytes(n, True)
        ws = dY.new_empty(need, dtype=torch.uint8) if need > 0 else None
        at = {key: t.data_ptr() for key, t in res.items()}
        rest = (dY.data_ptr(), ldy, n, at.get("dX"), layer.cols, at.get("dC"), at.get("dS"), ws.data_ptr() if need > 0 else None, need,
                self._raw_stream())
        if kept:
            st = self._lib.idkm_codes_linear_backward_kept(self._h, layer._at, X.Q.data_ptr(), X.E.data_ptr(), *rest)
        else:
            st = self._lib.idkm_codes_linear_backward(self._h, layer._at, X.data_ptr() if X is not None else None, ldx, *rest)
        self._check(st)
        return res

    def keep8(self, X):
        """idkm_keep8: X [n, cols] in 8 bits, a Kept8 that restore8 and codes_linear_backward take."""
        torch = _t()
        if not isinstance(X, torch.Tensor) or X.dim() != 2:
            raise TypeError("X must be a matrix")
        code, (n, cols) = _dtype(X, "X"), X.shape
        ldx = _rows(X, X.dtype, cols, self.device, "X")
        blocks = -(-cols // 32)
        kept = Kept8.__new__(Kept8)
        kept.Q, kept.E = Q, E = X.new_empty(n, 32 * blocks, dtype=torch.int8), X.new_empty(n, blocks, dtype=torch.uint8)
        kept.cols, kept.dtype, kept.code, kept.device, kept.shape = cols, X.dtype, code, self.device, (n, cols)
        st = self._lib.idkm_keep8(self._h, X.data_ptr(), n, cols, ldx, code, Q.data_ptr(), E.data_ptr(), self._raw_stream())
        if st:
            self._check(st)
        return kept

    def restore8(self, kept, out=None):
        """idkm_restore8: the activations [n, cols] that `kept` stands for, in their type."""
        if kept.device != self.device:
            raise TypeError(f"the activations must be in the memory of device {self.device}")
        n, cols = kept.shape
        if out is None:
            out, ldx = kept.Q.new_empty(n, cols, dtype=kept.dtype), cols
        else:
            ldx = _rows(out, kept.dtype, cols, self.device, "out")
            if out.shape[0] != n:
                raise TypeError(f"out must have {n} rows")
        st = self._lib.idkm_restore8(self._h, kept.Q.data_ptr(), kept.E.data_ptr(), n, cols, kept.code, out.data_ptr(), ldx, self._raw_stream())
        if st:
            self._check(st)
        return out

    def _int8_rows(self, X):
        """The same in whole steps of 128 columns."""
        torch = _t()
        if not isinstance(X, torch.Tensor) or X.dim() != 2:
            raise TypeError("X must be a matrix")
        code, (n, cols) = _dtype(X, "X"), X.shape
        ldx = _rows(X, X.dtype, cols, self.device, "X")
        Q, scale = X.new_empty(n, -(-cols // 128) * 128, dtype=torch.int8), X.new_empty(n, dtype=torch.float32)
        st = self._lib.idkm_int8_rows(self._h, X.data_ptr(), n, cols, ldx, code, Q.data_ptr(), Q.shape[1], scale.data_ptr(), self._raw_stream())
        if st:
            self._check(st)
        return Q, scale

    def int8_rows(self, X):
        """idkm_int8_rows: (Q int8 [n, cols], scale float32 [n]) of X [n, cols], rows of any of the three types."""
        Q, scale = self._int8_rows(X)
        return Q[:, :X.shape[1]], scale

    def int8_layer(self, weights, dtype=None):
        """An Int8Layer of a matrix [rows, cols] of weights, or of a CodesLayer, whose weights are written out for it (in float32, 2^26 at a time); for
        activations of `dtype` (the weights' own unless given)."""
        torch, dtype = _t(), dtype or weights.dtype
        if not isinstance(weights, CodesLayer):
            return Int8Layer(*self._int8_rows(weights), dtype, weights.shape[1])
        rows, cols = weights.rows, weights.cols
        wide = CodesLayer(weights.words, rows, cols, weights.C.float(), weights.S, weights.group)
        panel, parts = max(1, 2 ** 26 // cols), []
        for r in range(0, rows, panel):
            ids = torch.arange(r, min(r + panel, rows), device=weights.words.device)
            parts.append(self._int8_rows(self.codes_embedding(wide, ids)))
        Q, scale = (part[0] if len(parts) == 1 else torch.cat(part) for part in zip(*parts))
        return Int8Layer(Q, scale, dtype, cols)

    def int8_linear(self, layer, X, out=None):
        """idkm_int8_linear: X [n, cols] in the layer's type -> Y [n, rows], the product of X's rows and an Int8Layer's in 8-bit integers."""
        dev = self.device
        if layer.device != dev:
            raise TypeError(f"the layer must be in the memory of device {dev}")
        ldx = _rows(X, layer.dtype, layer.cols, dev, "X")
        n = X.shape[0]
        if out is None:
            out, ldy = X.new_empty(n, layer.rows), layer.rows
        else:
            ldy = _rows(out, layer.dtype, layer.rows, dev, "out")
            if out.shape[0] != n:
                raise TypeError(f"out must have {n} rows")
        need = layer.workspace_bytes(n)
        ws = X.new_empty(need, dtype=_t().uint8) if need > 0 else None
        st = self._lib.idkm_int8_linear(self._h, layer._at, X.data_ptr(), n, ldx, out.data_ptr(), ldy, ws.data_ptr() if need > 0 else None, need,
                                        self._raw_stream())
        if st:
            self._check(st)
        return out

    def int8_linear_backward(self, layer, dY):
        """idkm_int8_linear_backward: dX [n, cols] from dY [n, rows], both in the layer's type."""
        dev = self.device
        if layer.device != dev:
            raise TypeError(f"the layer must be in the memory of device {dev}")
        ldy = _rows(dY, layer.dtype, layer.rows, dev, "dY")
        n = dY.shape[0]
        dX = dY.new_empty(n, layer.cols)
        need = layer.workspace_bytes(n, True)
        ws = dY.new_empty(need, dtype=_t().uint8) if need > 0 else None
        st = self._lib.idkm_int8_linear_backward(self._h, layer._at, dY.data_ptr(), ldy, n, dX.data_ptr(), layer.cols,
                                                 ws.data_ptr() if need > 0 else None, need, self._raw_stream())
        if st:
            self._check(st)
        return dX

    def _tokens(self, ids):
        """Address, bytes of an id and number of tokens' ids, int32 or int64 and contiguous in one dimension."""
        torch = _t()
        if not isinstance(ids, torch.Tensor) or ids.get_device() != self.device:
            raise TypeError(f"ids must be in the memory of device {self.device}")
        wide = ids.dtype is torch.int64
        if not (wide or ids.dtype is torch.int32) or ids.dim() != 1 or not ids.is_contiguous():
            raise TypeError(f"ids must be contiguous int32 or int64 of one dimension, got {ids.dtype} {tuple(ids.shape)}")
        return ids.data_ptr(), 8 if wide else 4, ids.shape[0]

    def _looked_up(self, out, n, cols, dtype, ids):
        if out is None:
            return ids.new_empty(n, cols, dtype=dtype), cols
        ldy = _rows(out, dtype, cols, self.device, "out")
        if out.shape[0] != n:
            raise TypeError(f"out must have {n} rows")
        return out, ldy

    def embedding(self, W, ids, alpha=1.0, dtype=None, out=None):
        """idkm_embedding: rows ids [n] (int32 or int64; a negative one is padding, a row of zeros) of the float32 table W [rows, cols], times
        alpha, in `dtype` (float32 unless given, or `out`'s)."""
        torch = _t()
        if W.dim() != 2:
            raise TypeError(f"W must be a matrix, got {tuple(W.shape)}")
        w = _flat(W, torch.float32, W.shape, self.device, "W")
        at, width, n = self._tokens(ids)
        rows, cols = W.shape
        dtype = out.dtype if dtype is None and out is not None else dtype or torch.float32
        out, ldy = self._looked_up(out, n, cols, dtype, ids)
        st = self._lib.idkm_embedding(self._h, w, rows, cols, at, width, n, alpha, out.data_ptr(), ldy, _dtype(out, "out"), self._raw_stream())
        if st:
            self._check(st)
        return out

    def embedding_backward(self, dY, ids, rows, alpha=1.0):
        """idkm_embedding_backward: dW [rows, cols] float32 from dY [n, cols], zero in the rows of which there is no token."""
        torch = _t()
        at, width, n = self._tokens(ids)
        if dY.dim() != 2 or dY.shape[0] != n:
            raise TypeError(f"dY must have {n} rows")
        code, cols = _dtype(dY, "dY"), dY.shape[1]
        ldy = _rows(dY, dY.dtype, cols, self.device, "dY")
        dW = dY.new_empty(rows, cols, dtype=torch.float32)
        need = self._lib.idkm_embedding_backward_workspace(rows, cols, n)
        ws = dY.new_empty(need, dtype=torch.uint8) if need > 0 else None
        st = self._lib.idkm_embedding_backward(self._h, rows, cols, at, width, n, alpha, dY.data_ptr(), ldy, code, dW.data_ptr(),
                                               ws.data_ptr() if need > 0 else None, need, self._raw_stream())
        if st:
            self._check(st)
        return dW

    def codes_embedding(self, layer, ids, alpha=1.0, out=None):
        """idkm_codes_embedding: rows ids [n] of a table in its stored form (a CodesLayer), times alpha, [n, cols] in the layer's type."""
        if layer.device != self.device:
            raise TypeError(f"the layer must be in the memory of device {self.device}")
        at, width, n = self._tokens(ids)
        out, ldy = self._looked_up(out, n, layer.cols, layer.dtype, ids)
        st = self._lib.idkm_codes_embedding(self._h, layer._at, at, width, n, alpha, out.data_ptr(), ldy, self._raw_stream())
        if st:
            self._check(st)
        return out

    def codes_embedding_backward(self, layer, ids, dY, alpha=1.0, want_dC=True, want_dS=True):
        """idkm_codes_embedding_backward: dict of float32 dC [k, d] and, for a layer with scales, dS [rows, groups]."""
        torch, dev = _t(), self.device
        if layer.device != dev:
            raise TypeError(f"the layer must be in the memory of device {dev}")
        at, width, n = self._tokens(ids)
        ldy = _rows(dY, layer.dtype, layer.cols, dev, "dY")
        if dY.shape[0] != n:
            raise TypeError(f"dY must have {n} rows")
        res = {}
        if want_dC:
            res["dC"] = dY.new_empty(layer.k, layer.d, dtype=torch.float32)
        if want_dS and layer.S is not None:
            res["dS"] = dY.new_empty(layer.rows, layer.groups, dtype=torch.float32)
        need = layer.workspace_bytes(n, lookup=True)
        ws = dY.new_empty(need, dtype=torch.uint8) if need > 0 else None
        to = {key: t.data_ptr() for key, t in res.items()}
        st = self._lib.idkm_codes_embedding_backward(self._h, layer._at, at, width, n, alpha, dY.data_ptr(), ldy, to.get("dC"), to.get("dS"),
                                                     ws.data_ptr() if need > 0 else None, need, self._raw_stream())
        if st:
            self._check(st)
        return res

    def _grouped(self, t, group, name):
        """Address of a float32 [rows, cols] tensor, and the shape of its groups' scales."""
        shape = t.shape
        if len(shape) != 2:
            raise TypeError(f"{name} must be a matrix, got {tuple(shape)}")
        rows, cols = shape
        return _flat(t, _t().float32, shape, self.device, name), rows, cols, (rows, -(-cols // group) if group > 0 else 0)

    def group_scale(self, W, group):
        """idkm_group_scale: W [rows, cols] float32 -> (S [rows, ceil(cols / group)], Z = W / S)."""
        w, rows, cols, scales = self._grouped(W, group, "W")
        S, Z = W.new_empty(*scales), _t().empty_like(W)
        st = self._lib.idkm_group_scale(self._h, w, rows, cols, group, S.data_ptr(), Z.data_ptr(), self._raw_stream())
        if st:
            self._check(st)
        return S, Z

    def group_unscale(self, Zq, S, group):
        """idkm_group_unscale: S Zq."""
        z, rows, cols, scales = self._grouped(Zq, group, "Zq")
        s = _flat(S, Zq.dtype, scales, self.device, "S")
        Wq = _t().empty_like(Zq)
        st = self._lib.idkm_group_unscale(self._h, z, s, rows, cols, group, Wq.data_ptr(), self._raw_stream())
        if st:
            self._check(st)
        return Wq

    def group_unscale_backward(self, dWq, Zq, S, group):
        """idkm_group_unscale_backward: (dZq, dS)."""
        z, rows, cols, scales = self._grouped(Zq, group, "Zq")
        g = _flat(dWq, Zq.dtype, Zq.shape, self.device, "dWq")
        s = _flat(S, Zq.dtype, scales, self.device, "S")
        dZq, dS = _t().empty_like(Zq), _t().empty_like(S)
        st = self._lib.idkm_group_unscale_backward(self._h, g, z, s, rows, cols, group, dZq.data_ptr(), dS.data_ptr(),
                                                   self._raw_stream())
        if st:
            self._check(st)
        return dZq, dS

    def group_scale_backward(self, Z, S, group, dZ, dS=None):
        """idkm_group_scale_backward: dW from the gradients of Z and, optionally, of S."""
        z, rows, cols, scales = self._grouped(Z, group, "Z")
        g = _flat(dZ, Z.dtype, Z.shape, self.device, "dZ")
        s = _flat(S, Z.dtype, scales, self.device, "S")
        ds = _flat(dS, Z.dtype, scales, self.device, "dS") if dS is not None else None
        dW = _t().empty_like(Z)
        st = self._lib.idkm_group_scale_backward(self._h, z, s, g, ds, rows, cols, group, dW.data_ptr(), self._raw_stream())
        if st:
            self._check(st)
        return dW

    def distill(self, logits, index, teacher, tau, weight=None, out=None):
        """idkm_distill: (loss [n], lse [n]) of logits [n, V] against the teacher's list (index int32, teacher float32, both
        [n, top]; a negative index is no entry, entries of one index stay apart in the loss), and with weight [n] also the
        gradient of (weight * loss).sum() in the logits; `out` (which may be the logits themselves) receives it."""
        torch, dev = _t(), self.device
        code = _dtype(logits, "logits")
        if logits.dim() != 2 or index.dim() != 2:
            raise TypeError("logits and index must be matrices")
        n, V = logits.shape
        top = index.shape[1]
        ldz = _rows(logits, logits.dtype, V, dev, "logits")
        t = _flat(teacher, torch.float32, (n, top), dev, "teacher")
        i = _flat(index, torch.int32, (n, top), dev, "index")
        w = _flat(weight, torch.float32, (n,), dev, "weight") if weight is not None else None
        loss, lse = teacher.new_empty(n), teacher.new_empty(n)
        ldd = V
        if weight is None:
            if out is not None:
                raise TypeError("the gradient needs weights")
        elif out is None:
            out = torch.empty_like(logits) if ldz == V else logits.new_empty(n, V)
        else:
            ldd = _rows(out, logits.dtype, V, dev, "out")
            if out.shape[0] != n:
                raise TypeError(f"out must have {n} rows")
        key = (n, V, top, code)
        need = self._distill_bytes.get(key)
        if need is None:
            if len(self._distill_bytes) > 4096:
                self._distill_bytes.clear()
            need = self._distill_bytes[key] = self._lib.idkm_distill_workspace(n, V, top, code)
        ws = logits.new_empty(need, dtype=torch.uint8) if need > 0 else None
        st = self._lib.idkm_distill(self._h, logits.data_ptr(), n, V, ldz, code, i, t, top, tau, w, loss.data_ptr(), lse.data_ptr(),
                                    out.data_ptr() if out is not None else None, ldd, ws.data_ptr() if need > 0 else None, need,
                                    self._raw_stream())
        if st:
            self._check(st)
        return (loss, lse) if weight is None else (loss, lse, out)

    def step_F(self, W, Cb, tau, dist):
        """idkm_step_F: one evaluation of F at Cb.  Returns (C+ [k,d], n [k])."""
        import torch
        m, d = W.shape
        k = Cb.shape[0]
        Cp = torch.empty((k, d), dtype=torch.float32, device=W.device)
        n = torch.empty((k,), dtype=torch.float32, device=W.device)
        st = self._lib.idkm_step_F(self._h, _ptr(W, torch.float32, (m, d), "W"), m, d,
                                   _ptr(Cb, torch.float32, (k, d), "C"), k, float(tau), int(dist),
                                   _ptr(Cp, torch.float32, (k, d), "Cplus_out"), _ptr(n, torch.float32, (k,), "n_out"),
                                   _stream())
        self._check(st)
        self._keep = W
        return Cp, n

    def step_JCT(self, g):
        """idkm_step_JCT: (dF/dC)^T g at the state left by step_F / forward."""
        import torch
        out = torch.empty_like(g)
        st = self._lib.idkm_step_JCT(self._h, _ptr(g, torch.float32, g.shape, "g"),
                                     _ptr(out, torch.float32, g.shape, "out"), _stream())
        self._check(st)
        return out


def forward_noalloc(W, C0, tau, tol, max_iter, dist, out, device: int = 0, want_info: bool = True):
    """idkm_forward_noalloc.  `out` holds the caller's preallocated device tensors: C [k,d] (required) and
    optionally A [m,k], Wq [m,d], assign int32 [m].  Returns Info, or None when want_info is False (then the solve
    is only enqueued on the current stream)."""
    import torch
    lib = load_library()
    m, d = W.shape
    k = C0.shape[0]
    info = IdkmInfo()
    st = lib.idkm_forward_noalloc(int(device), _ptr(W, torch.float32, (m, d), "W"), m, d,
                                  _ptr(C0, torch.float32, (k, d), "C0"), k, float(tau), float(tol), int(max_iter),
                                  int(dist), _ptr(out["C"], torch.float32, (k, d), "C_out"),
                                  _ptr(out.get("A"), torch.float32, (m, k), "A_out"),
                                  _ptr(out.get("Wq"), torch.float32, (m, d), "Wq_out"),
                                  _ptr(out.get("assign"), torch.int32, (m,), "assign_out"),
                                  C.byref(info) if want_info else None, _stream())
    if st != IDKM_OK:
        raise IdkmError(st, lib.idkm_noalloc_last_error().decode())
    return _info(info) if want_info else None


def code_bits(k: int) -> int:
    return int(load_library().idkm_code_bits(int(k)))


def code_words(m: int, k: int) -> int:
    return int(load_library().idkm_code_words(int(m), int(k)))


class Batch:
    """Owns an idkm_batch: one context per layer; forward/backward over all layers in as few launches as fit."""

    def __init__(self, n_layers: int, device: int = 0):
        self._lib = load_library()
        h = C.c_void_p()
        st = self._lib.idkm_batch_create(C.byref(h), int(device), int(n_layers))
        if st != IDKM_OK:
            raise IdkmError(st, "idkm_batch_create failed")
        self._h = h
        self.n_layers = int(n_layers)
        self._keep = None

    def close(self):
        if getattr(self, "_h", None):
            self._lib.idkm_batch_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def launches(self) -> int:
        return int(self._lib.idkm_batch_launches(self._h))

    def set_path(self, path: int):
        for i in range(self.n_layers):
            st = self._lib.idkm_set_path(self._lib.idkm_batch_context(self._h, i), int(path))
            if st != IDKM_OK:
                raise IdkmError(st, "idkm_set_path failed")

    def context_set_spin_limit(self, i: int, polls: int):
        """idkm_set_spin_limit on the i-th layer's context."""
        st = self._lib.idkm_set_spin_limit(self._lib.idkm_batch_context(self._h, int(i)), int(polls))
        if st != IDKM_OK:
            raise IdkmError(st, "idkm_set_spin_limit failed")

    def _finish(self, st, statuses, strict):
        if st != IDKM_OK and strict:
            raise IdkmError(st, self._lib.idkm_batch_last_error(self._h).decode())
        return [int(x) for x in statuses]

    def forward(self, layers, tau, tol, max_iter, dist, want_Wq=True, want_assign=False, strict=True):
        """idkm_batch_forward.  layers: list of (W [m,d], C0 [k,d]) float32 device tensors (shapes may differ);
        tau may be a scalar or one value per layer.  Returns a list of dict(C, Wq, assign, info, status)."""
        import torch
        n = len(layers)
        taus = list(tau) if hasattr(tau, "__len__") else [tau] * n
        descs = (IdkmFwdDesc * n)()
        infos = (IdkmInfo * n)()
        statuses = (C.c_int * n)()
        outs = []
        for i, (W, C0) in enumerate(layers):
            m, d = W.shape
            k = C0.shape[0]
            Cout = torch.empty((k, d), dtype=torch.float32, device=W.device)
            Wq = torch.empty((m, d), dtype=torch.float32, device=W.device) if want_Wq else None
            asg = torch.empty((m,), dtype=torch.int32, device=W.device) if want_assign else None
            descs[i] = IdkmFwdDesc(_ptr(W, torch.float32, (m, d), "W"), m, d, _ptr(C0, torch.float32, (k, d), "C0"), k,
                                   float(taus[i]), float(tol), int(max_iter), int(dist),
                                   _ptr(Cout, torch.float32, (k, d), "C_out"), None,
                                   _ptr(Wq, torch.float32, (m, d), "Wq_out"), _ptr(asg, torch.int32, (m,), "assign_out"))
            outs.append(dict(C=Cout, Wq=Wq, assign=asg))
        st = self._lib.idkm_batch_forward(self._h, descs, n, infos, statuses, _stream())
        sts = self._finish(st, statuses, strict)
        self._keep = [W for W, _ in layers]  # the library borrows every W until the backward
        for i, o in enumerate(outs):
            o["info"] = _info(infos[i])
            o["status"] = sts[i]
        return outs

    def backward(self, dWqs, mode, tol=1e-6, max_iter=1000, alpha=1.0, strict=True):
        """idkm_batch_backward.  dWqs: one [m,d] float32 device tensor per layer.  Returns list of dict(dW, info, status)."""
        import torch
        n = len(dWqs)
        descs = (IdkmBwdDesc * n)()
        infos = (IdkmInfo * n)()
        statuses = (C.c_int * n)()
        outs = []
        for i, g in enumerate(dWqs):
            dW = torch.empty_like(g)
            descs[i] = IdkmBwdDesc(_ptr(g, torch.float32, g.shape, "dWq"), int(mode), float(tol), int(max_iter),
                                   float(alpha), _ptr(dW, torch.float32, g.shape, "dW_out"))
            outs.append(dict(dW=dW))
        st = self._lib.idkm_batch_backward(self._h, descs, n, infos, statuses, _stream())
        sts = self._finish(st, statuses, strict)
        for i, o in enumerate(outs):
            o["info"] = _info(infos[i])
            o["status"] = sts[i]
        return outs


def limits():
    lib = load_library()
    lim = IdkmLimits()
    lib.idkm_limits(C.byref(lim))
    return dict(max_k=lim.max_k, max_d=lim.max_d, max_kd=lim.max_kd)
