"""ctypes binding of libgelo.so: the same entry points as include/gelo.h, taking torch
tensors for device memory.  Argument marshalling only: every step runs in the HIP kernels.
There is no fallback: if the shared library is missing or the tensors are not on a GPU,
the calls raise."""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, byref, c_char_p, c_double, c_float, c_int, c_int64, c_uint32, c_uint64,
                    c_void_p)

import torch

GELO_F32, GELO_BF16 = 0, 1
GELO_ORTHOGONAL, GELO_GAUSSIAN, GELO_CONDITIONED, GELO_STRUCTURED, GELO_BLOCK_ORTHOGONAL, GELO_REFLECTOR_PRODUCT = 0, 1, 2, 3, 4, 5
GELO_NORM_MEDIAN, GELO_NORM_MEAN = 0, 1
GELO_ROPE_HALF, GELO_ROPE_PAIRS = 0, 1
GELO_OK = 0
STATUS_NAMES = ["GELO_OK", "GELO_EINVAL", "GELO_ESHAPE", "GELO_EDTYPE", "GELO_EALIGN", "GELO_ENOMEM",
                "GELO_ECOND", "GELO_ESINGULAR", "GELO_EREUSE", "GELO_ESTATE", "GELO_EHIP"]
GELO_MAX_N = 5120
GELO_BATCH_WINDOW = 4096
GELO_STATIC_MAX_N = 128
GELO_MAX_BATCH_DRAW = 48
GELO_STATIC_SCRATCH_BYTES = 16 << 20
GELO_NORM_MAX_D = 65536
GELO_ADAPT_MAX_RANK, GELO_ADAPT_MAX_PARTS = 128, 4

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgelo.so")


class _KvCacheStruct(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("n_pages", c_int), ("n_kv_heads", c_int), ("page_rows", c_int), ("head_dim", c_int),
                ("page_stride", c_int64), ("head_stride", c_int64), ("row_stride", c_int64)]


class _SeqBatchStruct(ctypes.Structure):
    _fields_ = [("n_seqs", c_int), ("n_rows", c_int), ("max_rows", c_int), ("max_kv_len", c_int),
                ("row_start", c_void_p), ("kv_len", c_void_p), ("page_table", c_void_p), ("table_ld", c_int64)]


class _KvCacheFp4Struct(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("n_pages", c_int), ("n_kv_heads", c_int), ("page_rows", c_int), ("head_dim", c_int),
                ("page_stride", c_int64), ("head_stride", c_int64)]


class _AdaptersStruct(ctypes.Structure):
    _fields_ = [("a", c_void_p), ("b", c_void_p), ("scale", c_void_p), ("n_adapters", c_int), ("rank", c_int), ("n_parts", c_int),
                ("part_end", c_int * GELO_ADAPT_MAX_PARTS), ("a_stride", c_int64), ("lda", c_int64), ("b_stride", c_int64), ("ldb", c_int64)]


# name -> (restype, argtypes); mirrors include/gelo.h one to one
SIGNATURES = {
    "gelo_create": (c_int, [POINTER(c_void_p), c_int, c_uint64, c_int]),
    "gelo_destroy": (c_int, [c_void_p]),
    "gelo_last_error": (c_char_p, [c_void_p]),
    "gelo_status_string": (c_char_p, [c_int]),
    "gelo_sample_mixing": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_double, c_int, c_uint64,
                                   POINTER(c_void_p), c_void_p]),
    "gelo_set_batch_floor": (c_int, [c_void_p, c_uint64]),
    "gelo_get_batch_floor": (c_int, [c_void_p, POINTER(c_uint64)]),
    "gelo_reserve": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_int]),
    "gelo_sample_mixing_batch": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_uint64, c_int, POINTER(c_void_p), c_void_p]),
    "gelo_chain": (c_int, [c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p, c_float, c_int, c_void_p, c_void_p, c_void_p,
                           c_void_p]),
    "gelo_mix": (c_int, [c_void_p, c_void_p, c_int, c_void_p, c_int64, c_float, c_int, c_void_p, c_int64, c_void_p]),
    "gelo_project": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_int64,
                             c_void_p, c_int64, c_void_p]),
    "gelo_unmix": (c_int, [c_void_p, c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
    "gelo_mixing_free": (c_int, [c_void_p, c_void_p]),
    "gelo_mixing_info": (c_int, [c_void_p, c_void_p, POINTER(c_int), POINTER(c_int), POINTER(c_int), POINTER(c_int),
                                 POINTER(c_int)]),
    "gelo_qkv_forward_static": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_float,
                                        c_int, c_uint64, c_void_p, c_void_p, c_void_p, c_void_p]),
    "gelo_fp8_weight_bytes": (c_int, [c_int, c_int, POINTER(ctypes.c_size_t)]),
    "gelo_prepare_weight_fp8": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p]),
    "gelo_project_fp8": (c_int, [c_void_p, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p]),
    "gelo_debug_quantize_rows_fp8": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]),
    "gelo_measure_matrix_rate": (c_int, [c_void_p, c_int, c_int, c_int, POINTER(c_double), POINTER(c_double), c_void_p]),
    "gelo_rms_norm": (c_int, [c_void_p, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_float, c_void_p, c_int64,
                              c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p]),
    "gelo_project_fp8_codes": (c_int, [c_void_p, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]),
    "gelo_rope_table": (c_int, [c_void_p, c_int, c_int, c_int, c_double, c_double, c_double, c_double, c_double, c_void_p, c_void_p]),
    "gelo_rope_append": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_int, c_int,
                                 c_void_p, c_int, c_void_p, c_int64, c_void_p]),
    "gelo_attention": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_float, c_int,
                               c_void_p, c_int64, c_void_p]),
    "gelo_reserve_attention": (c_int, [c_void_p, c_int]),
    "gelo_fp4_page_bytes": (c_int, [c_int, c_int, POINTER(ctypes.c_size_t)]),
    "gelo_rope_append_fp4": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_int, c_int,
                                     c_void_p, c_int, c_void_p, c_int64, c_void_p]),
    "gelo_cache_rows_fp4": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
    "gelo_attention_fp4": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_float, c_int,
                                   c_void_p, c_int64, c_void_p]),
    "gelo_adapt": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
    "gelo_reserve_adapt": (c_int, [c_void_p, c_int, c_int, c_int, c_int]),
    "gelo_debug_philox_words": (c_int, [c_void_p, c_uint32, c_uint32, c_uint64, c_uint32, c_uint32, c_void_p, c_void_p]),
    "gelo_mixing_export_table": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "gelo_qkv_forward": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_float,
                                 c_int, c_double, c_int, c_uint64, c_void_p, c_void_p, c_void_p, c_void_p]),
    "gelo_mixing_export": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_int),
                                   POINTER(c_float), c_void_p]),
}

_lib = None


class GeloError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else status}: {message}")
        self.status = status


def load_library() -> ctypes.CDLL:
    """Loads libgelo.so (built in-tree by `build.py`); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_05035_amd.build` "
                               "(there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (restype, argtypes) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = restype
            fn.argtypes = argtypes
        _lib = lib
    return _lib


def _check(ctx, status: int):
    if status != GELO_OK:
        msg = load_library().gelo_last_error(ctx) if ctx else b""
        raise GeloError(status, (msg or b"").decode())


# not torch's public names: a build may lack them
_raw_stream, _current_device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream(stream):
    if stream is None and (_raw_stream is None or _current_device is None):
        stream = torch.cuda.current_stream()
    if stream is None:
        # the current stream's handle alone: torch.cuda.current_stream() makes an object around it, 2.7 us of a call's 9
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return _raw_stream(_current_device())
    return c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GELO_F32
    if t.dtype == torch.bfloat16:
        return GELO_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _matrix(t: torch.Tensor, name: str):
    """(pointer, leading dimension) of a 2-D row-major device tensor."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (shape[1] > 1 and stride[1] != 1):
        raise ValueError(f"{name} must be a row-major 2-D tensor")
    return t.data_ptr(), stride[0] if shape[0] > 1 else max(stride[0], shape[1])


def gelo_create(device: int = 0, seed: int = 0, allow_batch_reuse: bool = False) -> c_void_p:
    ctx = c_void_p()
    st = load_library().gelo_create(byref(ctx), device, seed, int(allow_batch_reuse))
    if st != GELO_OK:
        raise GeloError(st, "gelo_create failed")
    return ctx


def gelo_destroy(ctx) -> None:
    _check(None, load_library().gelo_destroy(ctx))


def gelo_sample_mixing(ctx, kind: int, n_data: int, k_shield: int, d: int, dtype: int, cond_max: float = 1e3,
                       max_attempts: int = 64, batch_id: int = 0, stream=None) -> c_void_p:
    mixing = c_void_p()
    _check(ctx, load_library().gelo_sample_mixing(ctx, kind, n_data, k_shield, d, dtype, cond_max, max_attempts,
                                                  batch_id, byref(mixing), _stream(stream)))
    return mixing


def gelo_sample_mixing_batch(ctx, kind: int, n_data: int, k_shield: int, d: int, dtype: int, first_batch_id: int,
                             count: int, stream=None):
    """`count` mixing objects for consecutive batch ids from one launch (decode-shaped batches)."""
    arr = (c_void_p * count)()
    _check(ctx, load_library().gelo_sample_mixing_batch(ctx, kind, n_data, k_shield, d, dtype, first_batch_id, count,
                                                        arr, _stream(stream)))
    return [c_void_p(arr[i]) for i in range(count)]


def gelo_chain(ctx, mixing, H: torch.Tensor, W: torch.Tensor, Z: torch.Tensor, U: torch.Tensor, Y: torch.Tensor,
               shield_scale: float = 10.0, stat: int = GELO_NORM_MEDIAN, stream=None) -> torch.Tensor:
    """mix + project + unmix for a mixing object drawn earlier, one call."""
    for name, t in (("H", H), ("W", W), ("Z", Z), ("U", U), ("Y", Y)):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != H.dtype:
            raise ValueError(f"{name} must be a contiguous GPU tensor of H's dtype")
    p = W.shape[1]
    if W.shape[0] != H.shape[1] or Y.shape[1] != p or Z.shape[1] != p:
        raise GeloError(2, "W, Y and Z do not fit together")
    _check_against_mixing(ctx, mixing, (("H", H, "n_data", "d"), ("U", U, "n", "d"), ("Y", Y, "n", None), ("Z", Z, "n_data", None)))
    _check(ctx, load_library().gelo_chain(ctx, mixing, _dtype_code(H), p, c_void_p(H.data_ptr()), c_void_p(W.data_ptr()),
                                          shield_scale, stat, c_void_p(Z.data_ptr()), c_void_p(U.data_ptr()),
                                          c_void_p(Y.data_ptr()), _stream(stream)))
    return Z


def gelo_mixing_info(ctx, mixing):
    """(n_data, k_shield, d, dtype code, kind) the mixing object was drawn for."""
    v = [c_int() for _ in range(5)]
    _check(ctx, load_library().gelo_mixing_info(ctx, mixing, *[byref(x) for x in v]))
    return tuple(x.value for x in v)


def _check_against_mixing(ctx, mixing, tensors):
    """`tensors`: (name, tensor, rows expected ('n' or 'n_data'), width expected ('d' or None)).  The C ABI
    sees raw pointers; here the tensors carry shapes and types, so every mismatch that would make a kernel
    leave the caller's buffers is refused before the call."""
    n_data, k, d, code, _ = gelo_mixing_info(ctx, mixing)
    rows = {"n": n_data + k, "n_data": n_data}
    for name, t, r, w in tensors:
        if _dtype_code(t) != code:
            raise GeloError(3, f"{name} is {t.dtype} but the mixing object was drawn for {'bf16' if code == GELO_BF16 else 'f32'}")
        if t.dim() != 2 or t.shape[0] != rows[r] or (w == "d" and t.shape[1] != d):
            raise GeloError(2, f"{name} has shape {tuple(t.shape)}; this mixing object needs {rows[r]} rows"
                               + (f" of width {d}" if w == "d" else ""))


def gelo_mix(ctx, mixing, H: torch.Tensor, U: torch.Tensor, shield_scale: float = 10.0,
             stat: int = GELO_NORM_MEDIAN, stream=None) -> torch.Tensor:
    hp, ldh = _matrix(H, "H")
    up, ldu = _matrix(U, "U")
    _check_against_mixing(ctx, mixing, (("H", H, "n_data", "d"), ("U", U, "n", "d")))
    _check(ctx, load_library().gelo_mix(ctx, mixing, _dtype_code(H), hp, ldh, shield_scale, stat, up, ldu, _stream(stream)))
    return U


def gelo_project(ctx, U: torch.Tensor, W: torch.Tensor, Y: torch.Tensor, stream=None) -> torch.Tensor:
    up, ldu = _matrix(U, "U")
    wp, ldw = _matrix(W, "W")
    yp, ldy = _matrix(Y, "Y")
    n, d = U.shape
    p = W.shape[1]
    if W.shape[0] != d or tuple(Y.shape) != (n, p) or not (U.dtype == W.dtype == Y.dtype):
        raise ValueError("shape or dtype mismatch in gelo_project")
    _check(ctx, load_library().gelo_project(ctx, _dtype_code(U), n, d, p, up, ldu, wp, ldw, yp, ldy, _stream(stream)))
    return Y


def gelo_unmix(ctx, mixing, Y: torch.Tensor, Z: torch.Tensor, stream=None) -> torch.Tensor:
    yp, ldy = _matrix(Y, "Y")
    zp, ldz = _matrix(Z, "Z")
    if Y.shape[1] != Z.shape[1]:
        raise GeloError(2, "Y and Z must have the same width")
    _check_against_mixing(ctx, mixing, (("Y", Y, "n", None), ("Z", Z, "n_data", None)))
    _check(ctx, load_library().gelo_unmix(ctx, mixing, _dtype_code(Y), Y.shape[1], yp, ldy, zp, ldz, _stream(stream)))
    return Z


def gelo_mixing_free(ctx, mixing) -> None:
    _check(ctx, load_library().gelo_mixing_free(ctx, mixing))


def gelo_qkv_forward(ctx, kind: int, H: torch.Tensor, W: torch.Tensor, Z: torch.Tensor, k_shield: int = 0,
                     shield_scale: float = 10.0, stat: int = GELO_NORM_MEDIAN, cond_max: float = 1e3,
                     max_attempts: int = 64, batch_id: int = 0, U: torch.Tensor | None = None,
                     Y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    for name, t in (("H", H), ("W", W), ("Z", Z), ("U", U), ("Y", Y)):
        if t is not None and (not t.is_cuda or not t.is_contiguous() or t.dtype != H.dtype):
            raise ValueError(f"{name} must be a contiguous GPU tensor of H's dtype")
    n_data, d = H.shape
    p = W.shape[1]
    n = n_data + k_shield
    if W.shape[0] != d or tuple(Z.shape) != (n_data, p):
        raise ValueError("shape mismatch in gelo_qkv_forward")
    if (U is not None and tuple(U.shape) != (n, d)) or (Y is not None and tuple(Y.shape) != (n, p)):
        raise ValueError("U must be n x d and Y n x p")
    _check(ctx, load_library().gelo_qkv_forward(
        ctx, kind, _dtype_code(H), n_data, k_shield, d, p, c_void_p(H.data_ptr()), c_void_p(W.data_ptr()),
        shield_scale, stat, cond_max, max_attempts, batch_id, c_void_p(Z.data_ptr()),
        c_void_p(U.data_ptr()) if U is not None else None, c_void_p(Y.data_ptr()) if Y is not None else None,
        _stream(stream)))
    return Z


def gelo_qkv_forward_static(ctx, kind: int, H: torch.Tensor, W: torch.Tensor, Z: torch.Tensor, U: torch.Tensor,
                            Y: torch.Tensor, k_shield: int = 0, shield_scale: float = 10.0,
                            stat: int = GELO_NORM_MEDIAN, batch_id: int = 0, stream=None) -> torch.Tensor:
    """The chain for one decode-shaped batch through the entry point that allocates nothing."""
    for name, t in (("H", H), ("W", W), ("Z", Z), ("U", U), ("Y", Y)):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != H.dtype:
            raise ValueError(f"{name} must be a contiguous GPU tensor of H's dtype")
    n_data, d = H.shape
    p = W.shape[1]
    n = n_data + k_shield
    if W.shape[0] != d or tuple(Z.shape) != (n_data, p) or tuple(U.shape) != (n, d) or tuple(Y.shape) != (n, p):
        raise ValueError("shape mismatch in gelo_qkv_forward_static")
    _check(ctx, load_library().gelo_qkv_forward_static(
        ctx, kind, _dtype_code(H), n_data, k_shield, d, p, c_void_p(H.data_ptr()), c_void_p(W.data_ptr()),
        shield_scale, stat, batch_id, c_void_p(Z.data_ptr()), c_void_p(U.data_ptr()), c_void_p(Y.data_ptr()),
        _stream(stream)))
    return Z


def gelo_reserve(ctx, kind: int, dtype: int, n_data: int, k_shield: int, d: int, p: int = 0,
                 max_attempts: int = 64, mixings: int = 1) -> None:
    _check(ctx, load_library().gelo_reserve(ctx, kind, dtype, n_data, k_shield, d, p, max_attempts, mixings))


def gelo_set_batch_floor(ctx, first_unused: int) -> None:
    _check(ctx, load_library().gelo_set_batch_floor(ctx, first_unused))


def gelo_get_batch_floor(ctx) -> int:
    v = c_uint64()
    _check(ctx, load_library().gelo_get_batch_floor(ctx, byref(v)))
    return v.value


def gelo_fp8_weight_bytes(d: int, p: int) -> int:
    v = ctypes.c_size_t()
    st = load_library().gelo_fp8_weight_bytes(d, p, byref(v))
    if st != GELO_OK:
        raise GeloError(st, "gelo_fp8_weight_bytes")
    return v.value


def gelo_prepare_weight_fp8(ctx, W: torch.Tensor, stream=None) -> torch.Tensor:
    """The FP8 form of a bf16 weight (d x p): a uint8 device buffer holding the codes of W^T and the column scales."""
    if W.dtype != torch.bfloat16:
        raise TypeError("the 8-bit projection takes a bf16 weight")
    wp, ldw = _matrix(W, "W")
    d, p = W.shape
    Wq = torch.empty(gelo_fp8_weight_bytes(d, p), dtype=torch.uint8, device="cuda")
    _check(ctx, load_library().gelo_prepare_weight_fp8(ctx, d, p, wp, ldw, c_void_p(Wq.data_ptr()), _stream(stream)))
    return Wq


def _prepared(Wq: torch.Tensor, d: int, p: int):
    if Wq.dtype != torch.uint8 or Wq.numel() != gelo_fp8_weight_bytes(d, p):
        raise GeloError(2, "Wq is not the prepared form of a d x p weight")
    if not Wq.is_cuda or not Wq.is_contiguous():
        raise ValueError("Wq must be a contiguous GPU tensor")


def gelo_project_fp8(ctx, U: torch.Tensor, Wq: torch.Tensor, p: int, Y: torch.Tensor, stream=None) -> torch.Tensor:
    up, ldu = _matrix(U, "U")
    yp, ldy = _matrix(Y, "Y")
    n, d = U.shape
    if U.dtype != torch.bfloat16 or Y.dtype != torch.bfloat16 or tuple(Y.shape) != (n, p):
        raise ValueError("U and Y must be bf16, Y n x p")
    _prepared(Wq, d, p)
    _check(ctx, load_library().gelo_project_fp8(ctx, n, d, p, up, ldu, c_void_p(Wq.data_ptr()), yp, ldy, _stream(stream)))
    return Y


def gelo_project_fp8_codes(ctx, codes: torch.Tensor, scales: torch.Tensor, Wq: torch.Tensor, p: int, Y: torch.Tensor, stream=None) -> torch.Tensor:
    """The 8-bit projection of rows that are codes with scales already (gelo_rms_norm writes them)."""
    cp, ldq = _matrix(codes, "codes")
    yp, ldy = _matrix(Y, "Y")
    n, d = codes.shape
    if codes.dtype != torch.uint8 or Y.dtype != torch.bfloat16 or tuple(Y.shape) != (n, p):
        raise ValueError("codes must be uint8, Y bf16 and n x p")
    _vector(scales, "scales", torch.float32, n)
    _prepared(Wq, d, p)
    _check(ctx, load_library().gelo_project_fp8_codes(ctx, n, d, p, cp, ldq, scales.data_ptr(), Wq.data_ptr(), yp, ldy, _stream(stream)))
    return Y


class KvCache:
    """A paged cache: K and V of shape (pages, key heads, rows of a page, width of a head) in any order of memory (permuted views) as
    long as a head's row is contiguous and both have the same strides.  Describes the tensors and keeps them alive."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor):
        if K.dim() != 4 or K.shape != V.shape or K.dtype != V.dtype:
            raise ValueError("K and V must be of one type and shape: pages, key heads, rows of a page, width of a head")
        if not K.is_cuda or not V.is_cuda or K.device != V.device:
            raise ValueError("K and V must live on one GPU")
        # (the stride of a dimension of one entry says nothing)
        strides, other = ([x.stride(i) if x.shape[i] > 1 else K.shape[3] for i in range(3)] for x in (K, V))
        if strides != other or (K.shape[3] > 1 and (K.stride(3) != 1 or V.stride(3) != 1)):
            raise ValueError("K and V must have the same strides, the last of them 1")
        self.K, self.V, self.torch_dtype, self.dtype = K, V, K.dtype, _dtype_code(K)
        n_pages, n_kv_heads, page_rows, head_dim = K.shape
        self.n_kv_heads, self.page_rows, self.head_dim = n_kv_heads, page_rows, head_dim
        self.struct = _KvCacheStruct(K.data_ptr(), V.data_ptr(), n_pages, n_kv_heads, page_rows, head_dim, *strides)
        self.address = ctypes.addressof(self.struct)


def gelo_fp4_page_bytes(page_rows: int, head_dim: int) -> int:
    """Bytes of a head's piece of a page of a cache of 4 bits."""
    v = ctypes.c_size_t()
    st = load_library().gelo_fp4_page_bytes(page_rows, head_dim, byref(v))
    if st != GELO_OK:
        raise GeloError(st, f"page_rows={page_rows} must be a power of two from 16 on, head_dim={head_dim} a multiple of 32")
    return v.value


class KvCacheFp4:
    """A paged cache of 4 bits (see gelo_kv_cache_fp4 in include/gelo.h): K and V are uint8 of shape (pages, key heads, gelo_fp4_page_bytes(page_rows,
    head_dim)), the last dimension contiguous, both with the same strides.  Describes the tensors and keeps them alive."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, page_rows: int, head_dim: int):
        piece = gelo_fp4_page_bytes(page_rows, head_dim)
        if K.dtype != torch.uint8 or V.dtype != torch.uint8 or K.dim() != 3 or K.shape != V.shape or K.shape[2] != piece:
            raise ValueError(f"K and V must be uint8 of one shape: pages, key heads, {piece} bytes")
        if not K.is_cuda or not V.is_cuda or K.device != V.device:
            raise ValueError("K and V must live on one GPU")
        # (the stride of a dimension of one entry says nothing)
        strides, other = ([x.stride(i) if x.shape[i] > 1 else (piece + 15) // 16 * 16 for i in range(2)] for x in (K, V))
        if strides != other or K.stride(2) != 1 or V.stride(2) != 1:
            raise ValueError("K and V must have the same strides, the last of them 1")
        self.K, self.V = K, V
        self.n_kv_heads, self.page_rows, self.head_dim = K.shape[1], page_rows, head_dim
        self.struct = _KvCacheFp4Struct(K.data_ptr(), V.data_ptr(), K.shape[0], K.shape[1], page_rows, head_dim, *strides)
        self.address = ctypes.addressof(self.struct)


def _of_4_bits(cache) -> None:
    """A cache of values has the same fields in front, so the library would take its strides for bytes."""
    if not isinstance(cache, KvCacheFp4):
        raise TypeError(f"cache must be a KvCacheFp4, not a {type(cache).__name__}")


class Adapters:
    """Low-rank adapters beside one projection (see gelo_adapters in include/gelo.h): A (adapters, parts x rank, width of H), B (adapters, columns of Z, rank),
    rows contiguous; scale: a float32 factor to each, or None; part_ends: the columns where the parts of a fused projection end (None: one part).  Describes the
    tensors and keeps them alive."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None, part_ends=None):
        part_ends = [B.shape[1]] if part_ends is None else [int(x) for x in part_ends]
        if A.dim() != 3 or B.dim() != 3 or A.dtype != B.dtype or A.shape[0] != B.shape[0] or A.shape[1] != len(part_ends) * B.shape[2]:
            raise ValueError("A must be adapters x (parts x rank) x width and B adapters x columns x rank, of one type")
        if not 1 <= len(part_ends) <= GELO_ADAPT_MAX_PARTS or part_ends[-1] != B.shape[1]:
            raise ValueError(f"part_ends={part_ends}: up to {GELO_ADAPT_MAX_PARTS} parts, the last of which ends at column {B.shape[1]}")
        if not A.is_cuda or not B.is_cuda or A.device != B.device:
            raise ValueError("A and B must live on one GPU")
        if any(t.shape[2] > 1 and t.stride(2) != 1 for t in (A, B)):
            raise ValueError("rows of A and B must be contiguous")
        if scale is not None:
            _vector(scale, "scale", torch.float32, A.shape[0])
        count, _, self.d = A.shape
        _, self.p, rank = B.shape
        self.A, self.B, self.scale, self.torch_dtype, self.dtype = A, B, scale, A.dtype, _dtype_code(A)
        # (the stride of a dimension of one entry says nothing)
        steps = [t.stride(i) if t.shape[i] > 1 else t.shape[2] for t in (A, B) for i in range(2)]
        self.struct = _AdaptersStruct(A.data_ptr(), B.data_ptr(), None if scale is None else scale.data_ptr(), count, rank, len(part_ends),
                                      (c_int * GELO_ADAPT_MAX_PARTS)(*part_ends), *steps)
        self.address = ctypes.addressof(self.struct)


class SeqBatch:
    """Which rows of a batch and which pages of a cache belong to which sequence (see gelo_seq_batch in include/gelo.h): kv_len
    (n_seqs), page_table (n_seqs x pages) and row_start (n_seqs + 1, or None: one row each) are int32 tensors on the GPU, read when the
    kernels run."""

    def __init__(self, kv_len: torch.Tensor, page_table: torch.Tensor, max_kv_len: int, row_start: torch.Tensor | None = None, max_rows: int = 1):
        n_seqs = kv_len.shape[0] if kv_len.dim() == 1 else 0
        _vector(kv_len, "kv_len", torch.int32, n_seqs)
        if row_start is not None:
            _vector(row_start, "row_start", torch.int32, n_seqs + 1)
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.shape[0] != n_seqs:
            raise ValueError("page_table must be an int32 tensor with a row per sequence")
        if not -2 ** 31 <= max_rows < 2 ** 31:
            raise ValueError(f"max_rows={max_rows} does not fit 32 bits")
        tp, table_ld = _matrix(page_table, "page_table")     # (rows closer than max_kv_len takes, an expanded table's too, are refused by the library)
        self.kv_len, self.page_table, self.row_start = kv_len, page_table, row_start
        self.n_seqs, self.pages, self.max_kv_len = n_seqs, page_table.shape[1], max_kv_len
        self.struct = _SeqBatchStruct(n_seqs, n_seqs, max_rows, max_kv_len, None if row_start is None else row_start.data_ptr(), kv_len.data_ptr(), tp, table_ld)
        self.described = n_seqs, self.struct, ctypes.addressof(self.struct)


def _vector(t: torch.Tensor, name: str, dtype, count: int):
    if not t.is_cuda or t.dtype != dtype or t.shape != (count,) or (count > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous GPU vector of {count} {dtype}")


def _described(batch: SeqBatch, rows: int, cache: KvCache):
    """(rows, structure, its address) of the batch for matrices of `rows` rows; to be held while the address is in use.  Another number of rows
    gets another structure: threads may share a batch."""
    if batch.pages * cache.page_rows < batch.max_kv_len:
        raise GeloError(2, f"max_kv_len={batch.max_kv_len} rows do not fit {batch.pages} pages of {cache.page_rows}")
    described = batch.described
    if rows != described[0]:
        if batch.row_start is None:
            raise GeloError(2, f"{rows} rows, but every one of {batch.n_seqs} sequences brings one")
        struct = _SeqBatchStruct.from_buffer_copy(batch.struct)
        struct.n_rows = rows
        batch.described = described = rows, struct, ctypes.addressof(struct)
    return described


def gelo_rms_norm(ctx, X: torch.Tensor, gamma: torch.Tensor, eps: float, H: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                  residual_out: torch.Tensor | None = None, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, stream=None):
    """h = X + residual into residual_out, h / rms(h) * gamma into H and, as 8-bit codes with row scales, into codes and scales."""
    shape, dtype = X.shape, X.dtype
    n, d = shape
    xp, ldx = _matrix(X, "X")
    rp = op = hp = None
    ldr = ldo = ldh = 0
    if residual is not None:
        if residual.dtype != dtype or residual.shape != shape:
            raise ValueError("residual must be of X's dtype and shape")
        rp, ldr = _matrix(residual, "residual")
    if residual_out is not None:
        if residual_out.dtype != dtype or residual_out.shape != shape:
            raise ValueError("residual_out must be of X's dtype and shape")
        op, ldo = _matrix(residual_out, "residual_out")
    if H is not None:
        if H.dtype != dtype or H.shape != shape:
            raise ValueError("H must be of X's dtype and shape")
        hp, ldh = _matrix(H, "H")
    _vector(gamma, "gamma", dtype, d)
    cp, ldq, sp = None, 0, None
    if codes is not None or scales is not None:
        if codes is None or scales is None or codes.dtype != torch.uint8 or codes.shape != shape:
            raise ValueError("codes must be uint8 of X's shape and come with scales")
        cp, ldq = _matrix(codes, "codes")
        _vector(scales, "scales", torch.float32, n)
        sp = scales.data_ptr()
    status = load_library().gelo_rms_norm(ctx, _dtype_code(X), n, d, xp, ldx, rp, ldr, gamma.data_ptr(), eps, op, ldo, hp, ldh, cp, ldq, sp, _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)


def gelo_rope_table(ctx, rot_dim: int, n_pos: int, base: float = 10000.0, factor: float = 1.0, trained: float = 0.0, low: float = 1.0,
                    high: float = 4.0, first_pos: int = 0, stream=None) -> torch.Tensor:
    """(n_pos x rot_dim / 2 x 2) float32 cosines and sines for gelo_rope_append."""
    table = torch.empty((n_pos, rot_dim // 2, 2), dtype=torch.float32, device="cuda")
    _check(ctx, load_library().gelo_rope_table(ctx, rot_dim, first_pos, n_pos, base, factor, trained, low, high, table.data_ptr(), _stream(stream)))
    return table


def gelo_rope_append(ctx, QKV: torch.Tensor, n_q_heads: int, cache: KvCache, batch: SeqBatch, Q: torch.Tensor | None = None,
                     table: torch.Tensor | None = None, rot_dim: int = 0, layout: int = GELO_ROPE_HALF, stream=None):
    """Rotates the queries and keys of QKV's rows by their positions; queries into Q, keys and values into the cache."""
    zp, ld = _matrix(QKV, "QKV")
    rows, width = QKV.shape
    if QKV.dtype != cache.torch_dtype:
        raise GeloError(3, "QKV and the cache differ in type")
    if width != (n_q_heads + 2 * cache.n_kv_heads) * cache.head_dim:
        raise GeloError(2, f"a row of {width} values is not {n_q_heads} + 2 x {cache.n_kv_heads} heads of {cache.head_dim}")
    qp, ldq = None, 0
    if Q is not None:
        if Q.dtype != cache.torch_dtype or Q.shape != (rows, n_q_heads * cache.head_dim):
            raise ValueError("Q must be of QKV's dtype, a row of all query heads for each of its rows")
        qp, ldq = _matrix(Q, "Q")
    tp, n_table = None, 0
    if table is not None:
        n_table = table.shape[0]
        if table.dtype != torch.float32 or not table.is_cuda or not table.is_contiguous() or table.numel() != n_table * rot_dim:
            raise ValueError("table must be a contiguous float32 GPU tensor of positions x rot_dim")
        tp = table.data_ptr()
    described = _described(batch, rows, cache)
    status = load_library().gelo_rope_append(ctx, cache.dtype, n_q_heads, zp, ld, cache.address, described[2], layout, rot_dim, tp, n_table, qp, ldq,
                                             _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)


def gelo_rope_append_fp4(ctx, QKV: torch.Tensor, n_q_heads: int, cache: KvCacheFp4, batch: SeqBatch, Q: torch.Tensor | None = None,
                         table: torch.Tensor | None = None, rot_dim: int = 0, layout: int = GELO_ROPE_HALF, stream=None):
    """gelo_rope_append into a cache of 4 bits."""
    _of_4_bits(cache)
    zp, ld = _matrix(QKV, "QKV")
    rows, width = QKV.shape
    if width != (n_q_heads + 2 * cache.n_kv_heads) * cache.head_dim:
        raise GeloError(2, f"a row of {width} values is not {n_q_heads} + 2 x {cache.n_kv_heads} heads of {cache.head_dim}")
    qp, ldq = None, 0
    if Q is not None:
        if Q.dtype != QKV.dtype or Q.shape != (rows, n_q_heads * cache.head_dim):
            raise ValueError("Q must be of QKV's dtype, a row of all query heads for each of its rows")
        qp, ldq = _matrix(Q, "Q")
    tp, n_table = None, 0
    if table is not None:
        n_table = table.shape[0]
        if table.dtype != torch.float32 or not table.is_cuda or not table.is_contiguous() or table.numel() != n_table * rot_dim:
            raise ValueError("table must be a contiguous float32 GPU tensor of positions x rot_dim")
        tp = table.data_ptr()
    described = _described(batch, rows, cache)
    status = load_library().gelo_rope_append_fp4(ctx, _dtype_code(QKV), n_q_heads, zp, ld, cache.address, described[2], layout, rot_dim, tp, n_table, qp,
                                                 ldq, _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)


def gelo_cache_rows_fp4(ctx, cache: KvCacheFp4, batch: SeqBatch, K: torch.Tensor | None = None, V: torch.Tensor | None = None, stream=None):
    """The values that the batch's rows are held as, a row of all key heads to each, into K and V (either may be None)."""
    _of_4_bits(cache)
    some = V if K is None else K
    if some is None:
        raise ValueError("K and V are both None: nothing to write")
    shape, dtype = some.shape, some.dtype
    if len(shape) != 2 or shape[1] != cache.n_kv_heads * cache.head_dim:
        raise ValueError(f"K and V must have a row of {cache.n_kv_heads} heads of {cache.head_dim} for each row of the batch")
    kp = vp = None
    ldk = ldv = 0
    if K is not None:
        kp, ldk = _matrix(K, "K")
    if V is not None:
        if V.dtype != dtype or V.shape != shape:
            raise ValueError("K and V must be of one type and shape")
        vp, ldv = _matrix(V, "V")
    described = _described(batch, shape[0], cache)
    status = load_library().gelo_cache_rows_fp4(ctx, _dtype_code(some), cache.address, described[2], kp, ldk, vp, ldv, _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)


def gelo_attention(ctx, Q: torch.Tensor, O: torch.Tensor, n_q_heads: int, cache: KvCache, batch: SeqBatch, scale: float, causal: bool = True,
                   stream=None) -> torch.Tensor:
    """softmax(scale Q K^T) V over the rows of the cache that each row of Q sees, into O."""
    qp, ldq = _matrix(Q, "Q")
    op, ldo = _matrix(O, "O")
    shape = Q.shape
    if Q.dtype != cache.torch_dtype or O.dtype != cache.torch_dtype:
        raise GeloError(3, "Q, O and the cache differ in type")
    if shape[1] != n_q_heads * cache.head_dim or O.shape != shape:
        raise GeloError(2, f"Q and O must have {n_q_heads} heads of {cache.head_dim} values in a row")
    described = _described(batch, shape[0], cache)
    status = load_library().gelo_attention(ctx, cache.dtype, n_q_heads, qp, ldq, cache.address, described[2], scale, causal, op, ldo, _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)
    return O


def gelo_attention_fp4(ctx, Q: torch.Tensor, O: torch.Tensor, n_q_heads: int, cache: KvCacheFp4, batch: SeqBatch, scale: float, causal: bool = True,
                       stream=None) -> torch.Tensor:
    """gelo_attention over a cache of 4 bits."""
    _of_4_bits(cache)
    qp, ldq = _matrix(Q, "Q")
    op, ldo = _matrix(O, "O")
    shape = Q.shape
    if O.dtype != Q.dtype:
        raise GeloError(3, "Q and O differ in type")
    if shape[1] != n_q_heads * cache.head_dim or O.shape != shape:
        raise GeloError(2, f"Q and O must have {n_q_heads} heads of {cache.head_dim} values in a row")
    described = _described(batch, shape[0], cache)
    status = load_library().gelo_attention_fp4(ctx, _dtype_code(Q), n_q_heads, qp, ldq, cache.address, described[2], scale, causal, op, ldo, _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)
    return O


def gelo_reserve_attention(ctx, head_dim: int) -> None:
    _check(ctx, load_library().gelo_reserve_attention(ctx, head_dim))


def gelo_adapt(ctx, H: torch.Tensor, adapters: Adapters, which: torch.Tensor, Z: torch.Tensor, base: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Z = base + what the adapter of each row adds (base None: Z's own values).  which: int32, the adapter of every row; a number that is none's: base alone."""
    shape, out, dtype = H.shape, Z.shape, adapters.torch_dtype
    hp, ldh = _matrix(H, "H")
    zp, ldz = bp, ldb = _matrix(Z, "Z")
    if base is not None:
        bp, ldb = _matrix(base, "base")
        if base.dtype != dtype:
            raise GeloError(3, "base and the adapters differ in type")
        if base.shape != out:
            raise GeloError(2, f"base must be of Z's shape, {tuple(out)}")
    if H.dtype != dtype or Z.dtype != dtype:
        raise GeloError(3, "H, Z and the adapters differ in type")
    if shape[1] != adapters.d or out != (shape[0], adapters.p):
        raise GeloError(2, f"H must have rows of {adapters.d} values, Z as many of {adapters.p}")
    _vector(which, "which", torch.int32, shape[0])
    status = load_library().gelo_adapt(ctx, adapters.dtype, shape[0], adapters.d, adapters.p, hp, ldh, adapters.address, which.data_ptr(), bp, ldb, zp, ldz,
                                       _stream(stream))
    if status != GELO_OK:
        _check(ctx, status)
    return Z


def gelo_reserve_adapt(ctx, n: int, rank: int, n_parts: int, n_adapters: int) -> None:
    _check(ctx, load_library().gelo_reserve_adapt(ctx, n, rank, n_parts, n_adapters))


def gelo_debug_quantize_rows_fp8(ctx, U: torch.Tensor, stream=None):
    """Test hook: (codes n x d uint8, scales n float32) of the row quantisation of U."""
    up, ldu = _matrix(U, "U")
    n, d = U.shape
    codes = torch.empty((n, d), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n,), dtype=torch.float32, device="cuda")
    _check(ctx, load_library().gelo_debug_quantize_rows_fp8(ctx, n, d, up, ldu, c_void_p(codes.data_ptr()),
                                                            c_void_p(scales.data_ptr()), _stream(stream)))
    return codes, scales


def gelo_measure_matrix_rate(ctx, fp8: bool, iters: int = 2000, launches: int = 5, stream=None):
    """(seconds per launch, FLOP per launch) of the matrix-instruction-only kernel; waits for it."""
    sec, flop = c_double(0.0), c_double(0.0)
    _check(ctx, load_library().gelo_measure_matrix_rate(ctx, 1 if fp8 else 0, iters, launches, byref(sec), byref(flop),
                                                        _stream(stream)))
    return sec.value, flop.value


def gelo_debug_philox_words(ctx, stream_id: int, attempt: int, batch_id: int, first_block: int, blocks: int,
                            stream=None) -> torch.Tensor:
    """Test hook: blocks x 4 raw Philox words (int32 tensor holding the uint32 bit patterns)."""
    words = torch.empty((blocks, 4), dtype=torch.int32, device="cuda")
    _check(ctx, load_library().gelo_debug_philox_words(ctx, stream_id, attempt, batch_id, first_block, blocks,
                                                       c_void_p(words.data_ptr()), _stream(stream)))
    return words


def gelo_mixing_export_table(ctx, mixing, n: int, rounds: int = 3, stream=None) -> torch.Tensor:
    """Test hook: the (rounds + 1) x n table words of a structured mixing object (int32 bit patterns)."""
    table = torch.empty((rounds + 1, n), dtype=torch.int32, device="cuda")
    _check(ctx, load_library().gelo_mixing_export_table(ctx, mixing, c_void_p(table.data_ptr()), _stream(stream)))
    return table


def gelo_mixing_export(ctx, mixing, n: int, k_shield: int, d: int, want_shields: bool = True,
                       want_matrices: bool = True, stream=None):
    """Test hook: (A, A_inv, S, attempt, kappa) with A, A_inv, S float32 GPU tensors (None where not asked for)."""
    A = torch.empty((n, n), dtype=torch.float32, device="cuda") if want_matrices else None
    A_inv = torch.empty((n, n), dtype=torch.float32, device="cuda") if want_matrices else None
    S = torch.empty((k_shield, d), dtype=torch.float32, device="cuda") if (want_shields and k_shield > 0) else None
    attempt, kappa = c_int(-1), c_float(0.0)
    _check(ctx, load_library().gelo_mixing_export(
        ctx, mixing, c_void_p(A.data_ptr()) if A is not None else None,
        c_void_p(A_inv.data_ptr()) if A_inv is not None else None,
        c_void_p(S.data_ptr()) if S is not None else None, byref(attempt), byref(kappa), _stream(stream)))
    return A, A_inv, S, attempt.value, kappa.value
