"""Thin ctypes binding of libtucker_attn.so: argument marshalling only.

Same names as the C ABI (include/tucker_attn.h).  PyTorch supplies device memory and the
HIP stream; every step of the forward and backward passes runs in the library's kernels.  There is no
fallback: if the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
# TUCKER_ATTN_LIB names another build of the same library (comparing two builds in one session)
LIB_PATH = os.environ.get("TUCKER_ATTN_LIB") or os.path.join(_HERE, "libtucker_attn.so")

TUCKER_ATTN_F32 = 0
TUCKER_ATTN_BF16 = 1

EXPORTED = [
    "tucker_attn_create", "tucker_attn_destroy", "tucker_attn_parameter_count", "tucker_attn_cache_bytes",
    "tucker_attn_workspace_bytes",
    "tucker_attn_decode_workspace_bytes", "tucker_attn_forward", "tucker_attn_decode", "tucker_attn_decode_static",
    "tucker_attn_backward_workspace_bytes", "tucker_attn_backward",
    "tucker_attn_prepared_weights_bytes", "tucker_attn_prepare_weights", "tucker_attn_release_weights",
    "tucker_attn_append_paged", "tucker_attn_attend_workspace_bytes", "tucker_attn_attend_paged", "tucker_attn_attend_prefix",
    "tucker_attn_forward_paged_workspace_bytes", "tucker_attn_forward_paged",
    "tucker_attn_profile_enable", "tucker_attn_profile_read", "tucker_attn_measure_mfma_ceiling",
    "tucker_attn_status_string",
]
EXPORTED_CONVERT = [
    "tucker_convert_from_gqa", "tucker_convert_from_mla", "tucker_convert_hosvd_workspace_bytes",
    "tucker_convert_from_mha_hosvd",
]


class TuckerAttnError(RuntimeError):
    pass


class tucker_attn_config(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_head", C.c_int32),
                ("r1", C.c_int32), ("r2", C.c_int32), ("r3", C.c_int32),
                ("rt1", C.c_int32), ("rt2", C.c_int32), ("rt3", C.c_int32),
                ("causal", C.c_int32), ("use_rope", C.c_int32), ("rope_base", C.c_float),
                ("dtype", C.c_int32), ("max_positions", C.c_int32), ("shared_kv", C.c_int32),
                ("save_for_backward", C.c_int32)]


class tucker_attn_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")]


GRAD_KEYS = ("dC", "dU1", "dU2", "dU3", "dCt", "dUt1", "dUt2", "dUt3")


class tucker_attn_grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in GRAD_KEYS]


class tucker_attn_pages(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_size", C.c_int32)]

    @classmethod
    def of(cls, K, V=None) -> "tucker_attn_pages":
        """One layer's pool.  K: device tensor [pages, rows of a page, r3], V: [pages, rows of a page, rt3] (None with a shared
        key-value latent); pages may lie apart (any stride of the first dimension), rows may not.  The structure holds the tensors."""
        for t in (K, V):
            if t is not None and (t.dim() != 3 or t.stride(2) != 1 or t.stride(1) != t.shape[2]):
                raise TuckerAttnError("a pool is [pages, rows of a page, r] with contiguous pages")
        if V is not None and (V.shape[:2] != K.shape[:2] or V.dtype != K.dtype or V.device != K.device):
            raise TuckerAttnError("key and value pools have the same pages, storage type and device")
        # (0 says that pages lie one behind the other: an expanded tensor, whose stride that is, would be read behind its end)
        if K.shape[0] > 1 and any(t is not None and t.stride(0) < t.shape[1] * t.shape[2] for t in (K, V)):
            raise TuckerAttnError("pages of a pool lie apart: no expanded or overlapping tensor")
        strides = [0 if t is None or t.shape[0] == 1 else t.stride(0) for t in (K, V)]
        s = cls(K.data_ptr(), _ptr(V), *strides, K.shape[0], K.shape[1])
        s.tensors = (K, V)
        s.r3, s.rt3, s.dtype = K.shape[2], K.shape[2] if V is None else V.shape[2], K.dtype
        s.device = K.get_device()                                   # its index; -1: host memory
        s.kind = (s.r3, s.rt3, {"torch.float32": "f32", "torch.bfloat16": "bf16"}.get(str(K.dtype)))
        return s


class tucker_attn_batch(C.Structure):
    _fields_ = [("q_start", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("B", C.c_int32), ("T", C.c_int32),
                ("max_pages", C.c_int32), ("max_new", C.c_int32), ("max_len", C.c_int32)]

    @classmethod
    def of(cls, q_start, kv_len, page_table, *, tokens: int, max_new: int, max_len: int) -> "tucker_attn_batch":
        """The sequences of a step, for all layers.  q_start [B+1], kv_len [B], page_table [B, max_pages]: contiguous int32 device
        tensors, whose values may change between calls; tokens, max_new, max_len: rows of the token arrays and the bounds.
        The structure holds the tensors."""
        B = int(kv_len.shape[0])
        if tuple(q_start.shape) != (B + 1,) or page_table.dim() != 2 or page_table.shape[0] != B:
            raise TuckerAttnError("q_start is [B + 1], kv_len [B], page_table [B, max_pages]")
        for t in (q_start, kv_len, page_table):
            if str(t.dtype) != "torch.int32" or not t.is_contiguous() or t.device != kv_len.device:
                raise TuckerAttnError("the arrays of a batch are contiguous int32 tensors on one device")
        if not all(0 <= v < 2 ** 31 for v in (tokens, max_new, max_len, page_table.shape[1])):
            raise TuckerAttnError("tokens, max_new, max_len and the pages of a sequence are counted in 31 bits")   # (not cut to their low ones)
        s = cls(q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), B, int(tokens), int(page_table.shape[1]),
                int(max_new), int(max_len))
        s.tensors, s.device = (q_start, kv_len, page_table), kv_len.get_device()
        return s


WEIGHT_KEYS = ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")


class tucker_convert_weights_out(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_KEYS]


class tucker_convert_hosvd_info(C.Structure):
    _fields_ = [("sweeps", C.c_int32 * 6), ("jacobi_launches", C.c_int64), ("jacobi_ms", C.c_double),
                ("jacobi_bytes", C.c_double)]


_lib = None
# what the calls over pages hold their arrays against, by context handle: heads, model width, (r3, rt3, storage type)
_contexts: Dict[int, Tuple[int, int, Tuple[int, int, str]]] = {}


def load_library() -> C.CDLL:
    """Load the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise TuckerAttnError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2603_30033_amd.build` "
            "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    ctx_p = C.c_void_p
    lib.tucker_attn_create.argtypes = [C.POINTER(tucker_attn_config), C.POINTER(ctx_p)]
    lib.tucker_attn_create.restype = C.c_int
    lib.tucker_attn_destroy.argtypes = [ctx_p]
    lib.tucker_attn_destroy.restype = None
    lib.tucker_attn_parameter_count.argtypes = [C.POINTER(tucker_attn_config)]
    lib.tucker_attn_parameter_count.restype = C.c_size_t
    lib.tucker_attn_cache_bytes.argtypes = [ctx_p, C.c_int32, C.c_int32]
    lib.tucker_attn_cache_bytes.restype = C.c_size_t
    lib.tucker_attn_workspace_bytes.argtypes = [ctx_p, C.c_int32, C.c_int32]
    lib.tucker_attn_workspace_bytes.restype = C.c_size_t
    lib.tucker_attn_decode_workspace_bytes.argtypes = [ctx_p, C.c_int32]
    lib.tucker_attn_decode_workspace_bytes.restype = C.c_size_t
    lib.tucker_attn_forward.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_void_p,
                                        C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32,
                                        C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_forward.restype = C.c_int
    lib.tucker_attn_decode.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int32,
                                       C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_decode.restype = C.c_int
    lib.tucker_attn_decode_static.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int32,
                                              C.c_void_p]
    lib.tucker_attn_decode_static.restype = C.c_int
    lib.tucker_attn_backward_workspace_bytes.argtypes = [ctx_p, C.c_int32, C.c_int32]
    lib.tucker_attn_backward_workspace_bytes.restype = C.c_size_t
    lib.tucker_attn_backward.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.POINTER(tucker_attn_grads), C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                         C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_backward.restype = C.c_int
    lib.tucker_attn_prepared_weights_bytes.argtypes = [ctx_p]
    lib.tucker_attn_prepared_weights_bytes.restype = C.c_size_t
    lib.tucker_attn_prepare_weights.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_prepare_weights.restype = C.c_int
    lib.tucker_attn_release_weights.argtypes = [ctx_p]
    lib.tucker_attn_release_weights.restype = C.c_int
    pages_p, batch_p = C.POINTER(tucker_attn_pages), C.POINTER(tucker_attn_batch)
    lib.tucker_attn_append_paged.argtypes = [ctx_p, pages_p, batch_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                             C.c_void_p, C.c_int32, C.c_void_p]
    lib.tucker_attn_append_paged.restype = C.c_int
    lib.tucker_attn_attend_workspace_bytes.argtypes = [ctx_p, batch_p, C.c_int32]
    lib.tucker_attn_attend_workspace_bytes.restype = C.c_size_t
    lib.tucker_attn_attend_paged.argtypes = [ctx_p, pages_p, batch_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                             C.c_void_p]
    lib.tucker_attn_attend_paged.restype = C.c_int
    lib.tucker_attn_attend_prefix.argtypes = [ctx_p, pages_p, batch_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_attend_prefix.restype = C.c_int
    lib.tucker_attn_forward_paged_workspace_bytes.argtypes = [ctx_p, batch_p, C.c_int32]
    lib.tucker_attn_forward_paged_workspace_bytes.restype = C.c_size_t
    lib.tucker_attn_forward_paged.argtypes = [ctx_p, C.POINTER(tucker_attn_weights), C.c_void_p, C.c_void_p, pages_p, batch_p,
                                              C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_attn_forward_paged.restype = C.c_int
    lib.tucker_attn_profile_enable.argtypes = [ctx_p, C.c_int32]
    lib.tucker_attn_profile_enable.restype = C.c_int
    lib.tucker_attn_profile_read.argtypes = [ctx_p, C.POINTER(C.c_char_p), C.POINTER(C.c_float), C.c_int32]
    lib.tucker_attn_profile_read.restype = C.c_int
    lib.tucker_attn_measure_mfma_ceiling.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_float)]
    lib.tucker_attn_measure_mfma_ceiling.restype = C.c_int
    lib.tucker_attn_status_string.argtypes = [C.c_int]
    lib.tucker_attn_status_string.restype = C.c_char_p
    out_p = C.POINTER(tucker_convert_weights_out)
    lib.tucker_convert_from_gqa.argtypes = [C.c_int32] * 5 + [C.c_void_p] * 4 + [out_p, C.c_void_p]
    lib.tucker_convert_from_gqa.restype = C.c_int
    lib.tucker_convert_from_mla.argtypes = [C.c_int32] * 6 + [C.c_void_p] * 7 + [out_p, C.c_void_p]
    lib.tucker_convert_from_mla.restype = C.c_int
    lib.tucker_convert_hosvd_workspace_bytes.argtypes = [C.c_int32] * 3
    lib.tucker_convert_hosvd_workspace_bytes.restype = C.c_size_t
    lib.tucker_convert_from_mha_hosvd.argtypes = [C.c_int32] * 4 + [C.c_void_p] * 4 + [C.c_int32] * 7 + [
        out_p, C.POINTER(C.c_double), C.POINTER(tucker_convert_hosvd_info), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tucker_convert_from_mha_hosvd.restype = C.c_int
    _lib = lib
    return lib


def tucker_attn_status_string(status: int) -> str:
    return load_library().tucker_attn_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != 0:
        raise TuckerAttnError(f"{what}: status {status} ({tucker_attn_status_string(status)})")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream or None
    import torch
    # the handle alone: torch.cuda.current_stream() makes a Stream object first (3.0 us of a decode call's 23, this 0.4)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None


def tucker_attn_create(*, d_model, n_heads, d_head, r1, r2, r3, rt1=None, rt2=None, rt3=None, causal=True,
                       rope_base=None, dtype="bf16", max_positions=1, shared_kv=False,
                       save_for_backward=False) -> int:
    """Returns an opaque context handle (int).  Needs a current HIP device when rope_base is set."""
    cfg = tucker_attn_config(d_model, n_heads, d_head, r1, r2, r3, rt1 or r1, rt2 or r2, rt3 or r3,
                             int(bool(causal)), int(rope_base is not None), float(rope_base or 0.0),
                             {"f32": TUCKER_ATTN_F32, "bf16": TUCKER_ATTN_BF16}[dtype], int(max_positions),
                             int(bool(shared_kv)), int(bool(save_for_backward)))
    ctx = C.c_void_p()
    _check(load_library().tucker_attn_create(C.byref(cfg), C.byref(ctx)), "tucker_attn_create")
    _contexts[ctx.value] = (cfg.n_heads, cfg.d_model, (cfg.r3, cfg.rt3, dtype))
    return ctx.value


def tucker_attn_destroy(ctx: int) -> None:
    _contexts.pop(ctx, None)
    load_library().tucker_attn_destroy(ctx)


def tucker_attn_parameter_count(*, d_model, n_heads, r1, r2, r3, rt1=None, rt2=None, rt3=None, shared_kv=False) -> int:
    cfg = tucker_attn_config(d_model, n_heads, 1, r1, r2, r3, rt1 or r1, rt2 or r2, rt3 or r3, 0, 0, 0.0, TUCKER_ATTN_BF16,
                             1, int(bool(shared_kv)), 0)
    return int(load_library().tucker_attn_parameter_count(C.byref(cfg)))


def tucker_attn_cache_bytes(ctx: int, B: int, Lmax: int) -> int:
    return int(load_library().tucker_attn_cache_bytes(ctx, B, Lmax))


def tucker_attn_workspace_bytes(ctx: int, B: int, N: int) -> int:
    return int(load_library().tucker_attn_workspace_bytes(ctx, B, N))


def tucker_attn_decode_workspace_bytes(ctx: int, B: int) -> int:
    return int(load_library().tucker_attn_decode_workspace_bytes(ctx, B))


def _weights_struct(w: Dict[str, "object"]) -> tucker_attn_weights:
    return tucker_attn_weights(*[_ptr(w.get(k)) for k in ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")])


def tucker_attn_forward(ctx: int, weights: Dict, X, Y, pos0: int = 0, Kcache_out=None, Vcache_out=None,
                        workspace=None, stream=None, check: bool = True) -> int:
    """X, Y: contiguous device tensors [B, N, d]; weights: dict of contiguous device tensors;
    workspace: device uint8 tensor of at least tucker_attn_workspace_bytes bytes."""
    B, N = int(X.shape[0]), int(X.shape[1])
    Lmax = int(Kcache_out.shape[1]) if Kcache_out is not None else 0
    ws = _weights_struct(weights)
    st = load_library().tucker_attn_forward(ctx, C.byref(ws), X.data_ptr(), Y.data_ptr(), B, N, int(pos0),
                                            _ptr(Kcache_out), _ptr(Vcache_out), Lmax,
                                            _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                            _stream_ptr(stream))
    if check:
        _check(st, "tucker_attn_forward")
    return st


def tucker_attn_decode(ctx: int, weights: Dict, x, y, Kcache, Vcache, kv_len: List[int], workspace=None,
                       stream=None, check: bool = True) -> int:
    """x, y: [B, d]; Kcache/Vcache: [B, Lmax, r3]/[B, Lmax, rt3] (updated in place; with a shared
    key-value projection Vcache is None and Kcache is the one cache of unrotated latent rows);
    kv_len: host ints, cache length including the new token."""
    B = int(x.shape[0])
    Lmax = int(Kcache.shape[1])
    lens = (C.c_int32 * B)(*[int(v) for v in kv_len])
    ws = _weights_struct(weights)
    st = load_library().tucker_attn_decode(ctx, C.byref(ws), x.data_ptr(), y.data_ptr(), Kcache.data_ptr(),
                                           _ptr(Vcache), Lmax, lens, B,
                                           _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                           _stream_ptr(stream))
    if check:
        _check(st, "tucker_attn_decode")
    return st


def tucker_attn_decode_static(ctx: int, weights: Dict, x, y, Kcache, Vcache, kv_len: List[int], stream=None,
                              check: bool = True) -> int:
    """tucker_attn_decode on the library's own static scratch array (no workspace, no allocation)."""
    B = int(x.shape[0])
    Lmax = int(Kcache.shape[1])
    lens = (C.c_int32 * B)(*[int(v) for v in kv_len])
    ws = _weights_struct(weights)
    st = load_library().tucker_attn_decode_static(ctx, C.byref(ws), x.data_ptr(), y.data_ptr(), Kcache.data_ptr(),
                                                  _ptr(Vcache), Lmax, lens, B, _stream_ptr(stream))
    if check:
        _check(st, "tucker_attn_decode_static")
    return st


def tucker_attn_backward_workspace_bytes(ctx: int, B: int, N: int) -> int:
    return int(load_library().tucker_attn_backward_workspace_bytes(ctx, B, N))


def tucker_attn_backward(ctx: int, weights: Dict, X, dY, dX, grads: Dict, pos0: int = 0, workspace=None,
                         stream=None, check: bool = True, forward_state: bool = False) -> int:
    """X, dY, dX: contiguous device tensors [B, N, d] of the storage type; grads: dict of contiguous fp32
    device tensors keyed dC, dU1, dU2, dU3, dCt, dUt1, dUt2 and (unless the latent is shared) dUt3,
    shaped like the weights; all are overwritten.  forward_state: the workspace is the one the
    forward call of a save_for_backward context just used with the same inputs."""
    B, N = int(X.shape[0]), int(X.shape[1])
    ws = _weights_struct(weights)
    gs = tucker_attn_grads(*[_ptr(grads.get(k)) for k in GRAD_KEYS])
    st = load_library().tucker_attn_backward(ctx, C.byref(ws), X.data_ptr(), dY.data_ptr(), dX.data_ptr(),
                                             C.byref(gs), B, N, int(pos0), int(bool(forward_state)),
                                             _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                             _stream_ptr(stream))
    if check:
        _check(st, "tucker_attn_backward")
    return st


def tucker_attn_prepared_weights_bytes(ctx: int) -> int:
    return int(load_library().tucker_attn_prepared_weights_bytes(ctx))


def tucker_attn_prepare_weights(ctx: int, weights: Dict, prepared, stream=None, check: bool = True) -> int:
    """prepared: device uint8 tensor of at least tucker_attn_prepared_weights_bytes bytes; the caller keeps it
    (and the weight tensors) alive until tucker_attn_release_weights."""
    ws = _weights_struct(weights)
    st = load_library().tucker_attn_prepare_weights(ctx, C.byref(ws), _ptr(prepared),
                                                    0 if prepared is None else prepared.numel(), _stream_ptr(stream))
    if check:
        _check(st, "tucker_attn_prepare_weights")
    return st


def tucker_attn_release_weights(ctx: int) -> None:
    _check(load_library().tucker_attn_release_weights(ctx), "tucker_attn_release_weights")


# ---- paged latent cache ---------------------------------------------------------------------------------------

def _layer_of(ctx, pages: tucker_attn_pages) -> Tuple[int, int]:
    """Heads and model width of a context, whose cached rows `pages` hold."""
    if ctx not in _contexts:
        raise TuckerAttnError("no context of tucker_attn_create")
    heads, d_model, kind = _contexts[ctx]
    if pages.kind != kind:
        raise TuckerAttnError(f"pages of rows (r3, rt3, storage type) {pages.kind} where the context has {kind}")
    return heads, d_model


_ONE_GPU = "pools, batches, arrays and workspace of a call over pages are on one GPU"


def _rows(name: str, t, shape: Tuple[int, ...], pages: tucker_attn_pages) -> None:
    if t.shape != shape or t.dtype != pages.dtype:
        raise TuckerAttnError(f"{name}: {tuple(t.shape)} {t.dtype} where {shape} {pages.dtype} is expected")
    if t.get_device() != pages.device:
        raise TuckerAttnError(f"{name}: {_ONE_GPU}")


def _whole_rows(name: str, t, shape: Tuple[int, ...], pages: tucker_attn_pages) -> None:
    _rows(name, t, shape, pages)
    if not t.is_contiguous():
        raise TuckerAttnError(f"{name} is contiguous")


def _paged_stream_ptr(stream, pages: tucker_attn_pages, batch: tucker_attn_batch) -> Optional[int]:
    """The stream's handle, of the GPU that holds pool and batch and is the current one."""
    import torch
    device = pages.device
    if device < 0 or batch.device != device:
        raise TuckerAttnError(_ONE_GPU)
    if device != torch.cuda.current_device() or (stream is not None and stream.device_index != device):
        raise TuckerAttnError(f"a pool on GPU {device}: the calls over pages run on the current GPU, on a stream of it")
    if stream is not None:
        return stream.cuda_stream or None
    return torch._C._cuda_getCurrentRawStream(device) or None


def _paged_workspace(workspace, pages: tucker_attn_pages) -> Tuple[Optional[int], int]:
    if workspace is None:
        return None, 0
    if workspace.get_device() != pages.device:
        raise TuckerAttnError(f"workspace: {_ONE_GPU}")
    return workspace.data_ptr(), workspace.numel()


def tucker_attn_append_paged(ctx: int, pages: tucker_attn_pages, batch: tucker_attn_batch, K, V=None, Q=None, Qrot=None,
                             rotate: bool = True, stream=None, check: bool = True) -> int:
    """K: [T, r3], V: [T, rt3] (None with a shared latent), rows may lie apart (columns of a wider array); Q, Qrot: contiguous
    [T, n_heads, r3], or neither."""
    heads, _ = _layer_of(ctx, pages)
    T = batch.T
    _rows("K", K, (T, pages.r3), pages)
    ldk, channel = K.stride()
    ldv = 0
    if V is not None:
        _rows("V", V, (T, pages.rt3), pages)
        ldv, channel_v = V.stride()
        channel = channel if channel_v == 1 else 0
    if channel != 1:
        raise TuckerAttnError("the channels of a K or V row are contiguous")
    if T == 1:                                                      # one row has no distance
        ldk, ldv = pages.r3, pages.rt3
    if Q is not None:
        _whole_rows("Q", Q, (T, heads, pages.r3), pages)
    if Qrot is not None:
        _whole_rows("Qrot", Qrot, (T, heads, pages.r3), pages)
    st = load_library().tucker_attn_append_paged(ctx, C.byref(pages), C.byref(batch), K.data_ptr(), ldk, _ptr(V), ldv, _ptr(Q),
                                                 _ptr(Qrot), int(bool(rotate)), _paged_stream_ptr(stream, pages, batch))
    if check:
        _check(st, "tucker_attn_append_paged")
    return st


def tucker_attn_attend_workspace_bytes(ctx: int, batch: tucker_attn_batch, prefix_len: int = 0) -> int:
    return int(load_library().tucker_attn_attend_workspace_bytes(ctx, C.byref(batch), int(prefix_len)))


def _attend_rows(ctx, pages, batch, Q, O, lse) -> None:
    heads, _ = _layer_of(ctx, pages)
    T = batch.T
    _whole_rows("Q", Q, (T, heads, pages.r3), pages)
    _whole_rows("O", O, (T, heads, pages.rt3), pages)
    if lse is None:
        return
    if lse.shape != (T, heads) or lse.element_size() != 4 or not lse.is_floating_point() or not lse.is_contiguous():
        raise TuckerAttnError(f"lse: {tuple(lse.shape)} {lse.dtype} where contiguous ({T}, {heads}) torch.float32 is expected")
    if lse.get_device() != pages.device:
        raise TuckerAttnError(f"lse: {_ONE_GPU}")


def tucker_attn_attend_paged(ctx: int, pages: tucker_attn_pages, batch: tucker_attn_batch, Q, O, lse=None, workspace=None,
                             stream=None, check: bool = True) -> int:
    """Q: [T, n_heads, r3], O: [T, n_heads, rt3], lse: fp32 [T, n_heads] or None; workspace: device uint8 tensor of at least
    tucker_attn_attend_workspace_bytes bytes."""
    _attend_rows(ctx, pages, batch, Q, O, lse)
    st = load_library().tucker_attn_attend_paged(ctx, C.byref(pages), C.byref(batch), Q.data_ptr(), O.data_ptr(), _ptr(lse),
                                                 *_paged_workspace(workspace, pages), _paged_stream_ptr(stream, pages, batch))
    if check:
        _check(st, "tucker_attn_attend_paged")
    return st


def _prefix(pages, prefix_table, prefix_len) -> None:
    if prefix_table is None:
        return
    if prefix_len > 0 and (str(prefix_table.dtype) != "torch.int32" or not prefix_table.is_contiguous() or
                           prefix_table.numel() * pages.page_size < prefix_len):
        raise TuckerAttnError("prefix_table: int32, a page for every page_size rows of the prefix")
    if prefix_table.get_device() != pages.device:
        raise TuckerAttnError(f"prefix_table: {_ONE_GPU}")


def tucker_attn_attend_prefix(ctx: int, pages: tucker_attn_pages, batch: tucker_attn_batch, prefix_table, prefix_len: int, Q, O,
                              lse=None, workspace=None, stream=None, check: bool = True) -> int:
    """tucker_attn_attend_paged behind a common prefix; prefix_table: int32 device tensor with the pages of its rows."""
    _attend_rows(ctx, pages, batch, Q, O, lse)
    _prefix(pages, prefix_table, prefix_len)
    st = load_library().tucker_attn_attend_prefix(ctx, C.byref(pages), C.byref(batch), _ptr(prefix_table), int(prefix_len),
                                                  Q.data_ptr(), O.data_ptr(), _ptr(lse), *_paged_workspace(workspace, pages),
                                                  _paged_stream_ptr(stream, pages, batch))
    if check:
        _check(st, "tucker_attn_attend_prefix")
    return st


def tucker_attn_forward_paged_workspace_bytes(ctx: int, batch: tucker_attn_batch, prefix_len: int = 0) -> int:
    return int(load_library().tucker_attn_forward_paged_workspace_bytes(ctx, C.byref(batch), int(prefix_len)))


def tucker_attn_forward_paged(ctx: int, weights: Dict, X, Y, pages: tucker_attn_pages, batch: tucker_attn_batch, prefix_table=None,
                              prefix_len: int = 0, workspace=None, stream=None, check: bool = True) -> int:
    """X, Y: contiguous [T, d_model], the tokens of all sequences one sequence behind the other; weights: dict of contiguous device
    tensors; workspace: device uint8 tensor of at least tucker_attn_forward_paged_workspace_bytes bytes."""
    _, d_model = _layer_of(ctx, pages)
    for name, t in (("X", X), ("Y", Y)):
        _whole_rows(name, t, (batch.T, d_model), pages)
    _prefix(pages, prefix_table, prefix_len)
    if any(t is not None and t.get_device() != pages.device for t in weights.values()):
        raise TuckerAttnError(f"weights: {_ONE_GPU}")
    ws = _weights_struct(weights)
    st = load_library().tucker_attn_forward_paged(ctx, C.byref(ws), X.data_ptr(), Y.data_ptr(), C.byref(pages), C.byref(batch),
                                                  _ptr(prefix_table), int(prefix_len), *_paged_workspace(workspace, pages),
                                                  _paged_stream_ptr(stream, pages, batch))
    if check:
        _check(st, "tucker_attn_forward_paged")
    return st


def tucker_attn_profile_enable(ctx: int, on: bool) -> None:
    _check(load_library().tucker_attn_profile_enable(ctx, int(bool(on))), "tucker_attn_profile_enable")


def tucker_attn_profile_read(ctx: int) -> List[Tuple[str, float]]:
    names = (C.c_char_p * 41)()
    ms = (C.c_float * 41)()
    n = load_library().tucker_attn_profile_read(ctx, names, ms, 41)
    if n < 0:
        _check(n, "tucker_attn_profile_read")
    return [(names[i].decode(), float(ms[i])) for i in range(n)]


def tucker_attn_measure_mfma_ceiling(from_lds: bool, iters: int = 20000) -> float:
    """TFLOP/s of a bf16 MFMA loop on the current device (operands in registers, or one re-read from LDS)."""
    out = C.c_float()
    _check(load_library().tucker_attn_measure_mfma_ceiling(int(bool(from_lds)), int(iters), C.byref(out)),
           "tucker_attn_measure_mfma_ceiling")
    return float(out.value)


# ---- weight front-ends (include/tucker_convert.h) ------------------------------------------------

def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return TUCKER_ATTN_F32
    if t.dtype == torch.bfloat16:
        return TUCKER_ATTN_BF16
    raise TuckerAttnError(f"unsupported storage type {t.dtype}")


def _out_struct(out: Dict) -> tucker_convert_weights_out:
    return tucker_convert_weights_out(*[_ptr(out.get(k)) for k in WEIGHT_KEYS])


def tucker_convert_from_gqa(WQ, WK, WV, WO, n_heads: int, n_groups: int, out: Dict, stream=None,
                            check: bool = True) -> int:
    """out: dict of preallocated device tensors C, U1, U2, U3, Ct, Ut1, Ut2, Ut3."""
    d, n = WQ.shape
    st = load_library().tucker_convert_from_gqa(_dtype_code(WQ), d, n_heads, n // n_heads, n_groups, _ptr(WQ), _ptr(WK),
                                                _ptr(WV), _ptr(WO), C.byref(_out_struct(out)), _stream_ptr(stream))
    if check:
        _check(st, "tucker_convert_from_gqa")
    return st


def tucker_convert_from_mla(WDQ, WUQ, WDKV, WUK, WDV, WUV, WO, n_heads: int, out: Dict, stream=None,
                            check: bool = True) -> int:
    d, dcq = WDQ.shape
    dck, n = WUK.shape
    st = load_library().tucker_convert_from_mla(_dtype_code(WDQ), d, n_heads, n // n_heads, dcq, dck, _ptr(WDQ), _ptr(WUQ),
                                                _ptr(WDKV), _ptr(WUK), _ptr(WDV), _ptr(WUV), _ptr(WO),
                                                C.byref(_out_struct(out)), _stream_ptr(stream))
    if check:
        _check(st, "tucker_convert_from_mla")
    return st


def tucker_convert_hosvd_workspace_bytes(d: int, n_heads: int, d_head: int) -> int:
    return int(load_library().tucker_convert_hosvd_workspace_bytes(d, n_heads, d_head))


def tucker_convert_from_mha_hosvd(WQ, WK, WV, WO, n_heads: int, ranks, ranks_t, shared_kv: bool, out: Dict,
                                  workspace, want_singular_values: bool = False, stream=None, check: bool = True):
    """Returns (status, singular values as a list of 2*(nH+2d) floats or None, info dict)."""
    d, n = WQ.shape
    sv = (C.c_double * (2 * (n_heads + 2 * d)))() if want_singular_values else None
    info = tucker_convert_hosvd_info()
    st = load_library().tucker_convert_from_mha_hosvd(
        _dtype_code(WQ), d, n_heads, n // n_heads, _ptr(WQ), _ptr(WK), _ptr(WV), _ptr(WO), *[int(r) for r in ranks],
        *[int(r) for r in ranks_t], int(bool(shared_kv)), C.byref(_out_struct(out)), sv, C.byref(info), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream_ptr(stream))
    if check:
        _check(st, "tucker_convert_from_mha_hosvd")
    return st, (list(sv) if sv is not None else None), dict(
        sweeps=list(info.sweeps), jacobi_launches=int(info.jacobi_launches), jacobi_ms=float(info.jacobi_ms),
        jacobi_bytes=float(info.jacobi_bytes))
