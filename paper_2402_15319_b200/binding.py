"""ctypes binding with the same names as include/vq.h.  Argument marshalling only: every step
of the computation runs in the CUDA library.  Tensors are torch CUDA tensors (device memory and
streams are torch's); there is no CPU fallback — a missing library is an error."""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass, fields

VQ_CB_FP16, VQ_CB_INT8_SCALED, VQ_CB_INT4_G128 = 0, 1, 2
VQ_IMPL_AUTO, VQ_IMPL_GENERIC, VQ_IMPL_TUNED, VQ_IMPL_STREAM, VQ_IMPL_TILE = 0, 1, 2, 3, 4

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libvq_b200.so")
_lib = None


class VQError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {vq_status_string(code)}")


class _CFormat(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_rows", "k_cols", "vq_dim", "index_bits", "block_rows", "block_cols", "cb_type")]


class _CPackInfo(ctypes.Structure):
    _fields_ = [("entries", ctypes.c_int32), ("codebook_bits", ctypes.c_int32),
                ("indices_per_row", ctypes.c_int64), ("row_stride_bytes", ctypes.c_int64),
                ("index_bytes", ctypes.c_int64), ("n_blocks", ctypes.c_int64),
                ("codebook_bytes_per_block", ctypes.c_int64), ("codebook_bytes", ctypes.c_int64),
                ("scale_bytes", ctypes.c_int64), ("total_bytes", ctypes.c_int64),
                ("bpv_paper", ctypes.c_double), ("bpv_stored", ctypes.c_double)]


@dataclass(frozen=True)
class VQFormat:
    n_rows: int
    k_cols: int
    vq_dim: int
    index_bits: int
    block_rows: int
    block_cols: int
    cb_type: int

    def c(self) -> _CFormat:
        return _c_format(self)


@functools.lru_cache(maxsize=4096)
def _c_format(f: "VQFormat") -> _CFormat:
    # one struct per distinct format, reused by every call (the library only reads it)
    return _CFormat(f.n_rows, f.k_cols, f.vq_dim, f.index_bits, f.block_rows, f.block_cols, f.cb_type)


@dataclass(frozen=True)
class PackInfo:
    entries: int
    codebook_bits: int
    indices_per_row: int
    row_stride_bytes: int
    index_bytes: int
    n_blocks: int
    codebook_bytes_per_block: int
    codebook_bytes: int
    scale_bytes: int
    total_bytes: int
    bpv_paper: float
    bpv_stored: float


_SIGNATURES = {
    "vq_pack_info": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]),
    "vq_workspace_bytes": (ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_int]),
    "vq_workspace_bytes_host": (ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_int]),
    "vq_decode_weights": (ctypes.c_int, [ctypes.c_void_p] * 6),
    "vq_norm_info": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]),
    "vq_decode_weights_normalized": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]),
    "vq_gemm_small_batch_normalized": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                                       ctypes.c_int, ctypes.c_void_p]),
    "vq_gemv": (ctypes.c_int, [ctypes.c_void_p] * 7 + [ctypes.c_size_t, ctypes.c_void_p]),
    "vq_gemm_small_batch": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_gemm_small_batch_impl": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int]),
    "vq_gemm_small_batch_grouped": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                                   ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_grouped_kernel_launches": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]),
    "vq_gemm_small_batch_grouped_host": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                                        ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_workspace_bytes_grouped_host": (ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]),
    "vq_gemm_small_batch_host": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_gemm_small_batch_host_static": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_void_p]),
    "vq_static_scratch_bytes": (ctypes.c_size_t, []),
    "vq_int4g128_gemm_small_batch": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32] + [ctypes.c_void_p] * 4 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_int4g128_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int]),
    "vq_assign_indices": (ctypes.c_int, [ctypes.c_void_p] * 7),
    "vq_unpack_uniform": (ctypes.c_int, [ctypes.c_int, ctypes.c_int32, ctypes.c_int32] + [ctypes.c_void_p] * 4),
    "vq_device_wait_failures": (ctypes.c_int, [ctypes.c_void_p]),
    "vq_probe_decode_loop": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "vq_probe_read": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    "vq_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "vq_kv_info": (ctypes.c_int, [ctypes.c_void_p] * 2),
    "vq_kv_attention_workspace_bytes": (ctypes.c_size_t, [ctypes.c_void_p]),
    "vq_kv_attention": (ctypes.c_int, [ctypes.c_void_p] * 3 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                       ctypes.c_void_p, ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "vq_kv_append": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                    ctypes.c_void_p, ctypes.c_void_p]),
    "vq_kv_pages_workspace_bytes": (ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_int]),
    "vq_kv_reserve": (ctypes.c_int, [ctypes.c_void_p] * 6 + [ctypes.c_size_t, ctypes.c_void_p]),
    "vq_kv_fork": (ctypes.c_int, [ctypes.c_void_p] * 2 + [ctypes.c_int] + [ctypes.c_void_p] * 3 + [ctypes.c_int] + [ctypes.c_void_p] * 2 +
                   [ctypes.c_size_t, ctypes.c_void_p]),
    "vq_kv_free": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_int, ctypes.c_void_p]),
    "vq_kv_compact": (ctypes.c_int, [ctypes.c_void_p] * 2 + [ctypes.c_int] + [ctypes.c_void_p] * 4 + [ctypes.c_size_t, ctypes.c_void_p]),
    "vq_kv_copy_pages": (ctypes.c_int, [ctypes.c_void_p] * 2 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]),
    "vq_residual_norm": (ctypes.c_int, [ctypes.c_void_p] * 11),
}


def lib_path() -> str:
    return _LIB_PATH


def exported_symbols():
    return sorted(_SIGNATURES)


def load():
    """Load libvq_b200.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2402_15319_b200.build`")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def vq_status_string(code: int) -> str:
    return load().vq_status_string(int(code)).decode()


def _check(code: int, where: str):
    if code != 0:
        raise VQError(code, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


_current_raw_stream = None


def _stream(stream):
    """cudaStream_t of `stream`, or of torch's current stream on the current device (its handle directly: a Stream
    object per call is a microsecond of host time)."""
    if stream is not None:
        return stream.cuda_stream
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
        _current_raw_stream = (lambda: raw(device())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
    return _current_raw_stream()


def vq_pack_info(fmt: VQFormat) -> PackInfo:
    c, out = fmt.c(), _CPackInfo()
    _check(load().vq_pack_info(ctypes.byref(c), ctypes.byref(out)), "vq_pack_info")
    return PackInfo(*[getattr(out, n) for n, _ in _CPackInfo._fields_])


def vq_workspace_bytes(fmt: VQFormat, batch: int) -> int:
    c = fmt.c()
    return load().vq_workspace_bytes(ctypes.byref(c), int(batch))


def vq_workspace_bytes_host(fmt: VQFormat, batch: int) -> int:
    c = fmt.c()
    return load().vq_workspace_bytes_host(ctypes.byref(c), int(batch))


def vq_decode_weights(fmt: VQFormat, d_idx, d_cb, d_scale, d_W, stream=None) -> None:
    c = fmt.c()
    _check(load().vq_decode_weights(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_W),
                                    _stream(stream)), "vq_decode_weights")


class _CNormInfo(ctypes.Structure):
    _fields_ = [("code_row_bytes", ctypes.c_size_t), ("codes_bytes", ctypes.c_size_t), ("lut_bytes", ctypes.c_size_t)]


def vq_norm_info(fmt: VQFormat, norm_block_cols: int):
    """(code_row_bytes, codes_bytes, lut_bytes) of the block-wise normalisation buffers."""
    c = fmt.c()
    out = _CNormInfo()
    _check(load().vq_norm_info(ctypes.byref(c), int(norm_block_cols), ctypes.byref(out)), "vq_norm_info")
    return int(out.code_row_bytes), int(out.codes_bytes), int(out.lut_bytes)


def vq_decode_weights_normalized(fmt: VQFormat, d_idx, d_cb, d_scale, d_norm_codes, d_norm_lut, norm_block_cols: int, d_W,
                                 stream=None) -> None:
    c = fmt.c()
    _check(load().vq_decode_weights_normalized(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_norm_codes),
                                               _ptr(d_norm_lut), int(norm_block_cols), _ptr(d_W), _stream(stream)),
           "vq_decode_weights_normalized")


def vq_gemm_small_batch_normalized(fmt: VQFormat, d_idx, d_cb, d_scale, d_norm_codes, d_norm_lut, norm_block_cols: int, d_X, d_Y,
                                   batch: int, stream=None) -> None:
    c = fmt.c()
    _check(load().vq_gemm_small_batch_normalized(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_norm_codes),
                                                 _ptr(d_norm_lut), int(norm_block_cols), _ptr(d_X), _ptr(d_Y), int(batch),
                                                 _stream(stream)), "vq_gemm_small_batch_normalized")


def vq_gemv(fmt: VQFormat, d_idx, d_cb, d_scale, d_x, d_y, d_ws, stream=None) -> None:
    c = fmt.c()
    _check(load().vq_gemv(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_x), _ptr(d_y),
                          _ptr(d_ws), d_ws.numel() * d_ws.element_size(), _stream(stream)), "vq_gemv")


def vq_gemm_small_batch(fmt: VQFormat, d_idx, d_cb, d_scale, d_X, d_Y, batch: int, d_ws, stream=None) -> None:
    c = fmt.c()
    _check(load().vq_gemm_small_batch(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_X),
                                      _ptr(d_Y), int(batch), _ptr(d_ws), d_ws.numel() * d_ws.element_size(),
                                      _stream(stream)), "vq_gemm_small_batch")


class _CGroupMember(ctypes.Structure):
    _fields_ = [("d_idx", ctypes.c_void_p), ("d_cb", ctypes.c_void_p), ("d_scale", ctypes.c_void_p),
                ("d_Y", ctypes.c_void_p), ("n_rows", ctypes.c_int32)]


def vq_gemm_small_batch_grouped(fmt: VQFormat, members, d_X, batch: int, d_ws, stream=None) -> None:
    """members: sequence of (d_idx, d_cb, d_scale, d_Y, n_rows); fmt.n_rows = the sum of the members' rows."""
    arr = (_CGroupMember * len(members))(*[(_ptr(idx), _ptr(cb), _ptr(sc), _ptr(Y), int(n)) for idx, cb, sc, Y, n in members])
    c = fmt.c()
    _check(load().vq_gemm_small_batch_grouped(ctypes.byref(c), arr, len(members), _ptr(d_X), int(batch), _ptr(d_ws),
                                              d_ws.numel() * d_ws.element_size(), _stream(stream)),
           "vq_gemm_small_batch_grouped")


def vq_gemm_small_batch_grouped_host(fmt: VQFormat, members, h_X, batch: int, d_ws, stream=None) -> None:
    """members: sequence of (d_idx, d_cb, d_scale, h_Y, n_rows) with HOST outputs; h_X a host tensor (pinned for
    the direct path).  Synchronise before reading the outputs."""
    arr = (_CGroupMember * len(members))(*[(_ptr(idx), _ptr(cb), _ptr(sc), _ptr(Y), int(n)) for idx, cb, sc, Y, n in members])
    c = fmt.c()
    _check(load().vq_gemm_small_batch_grouped_host(ctypes.byref(c), arr, len(members), _ptr(h_X), int(batch), _ptr(d_ws),
                                                   d_ws.numel() * d_ws.element_size(), _stream(stream)),
           "vq_gemm_small_batch_grouped_host")


def vq_workspace_bytes_grouped_host(fmt: VQFormat, n_members: int, batch: int) -> int:
    c = fmt.c()
    return load().vq_workspace_bytes_grouped_host(ctypes.byref(c), int(n_members), int(batch))


def vq_grouped_kernel_launches(fmt: VQFormat, n_members: int, batch: int) -> int:
    c = fmt.c()
    return load().vq_grouped_kernel_launches(ctypes.byref(c), int(n_members), int(batch))


def vq_gemm_small_batch_impl(fmt: VQFormat, d_idx, d_cb, d_scale, d_X, d_Y, batch: int, d_ws, impl: int,
                             stream=None) -> None:
    c = fmt.c()
    _check(load().vq_gemm_small_batch_impl(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(d_X),
                                           _ptr(d_Y), int(batch), _ptr(d_ws),
                                           d_ws.numel() * d_ws.element_size(), _stream(stream), int(impl)),
           "vq_gemm_small_batch_impl")


def vq_gemm_small_batch_host(fmt: VQFormat, d_idx, d_cb, d_scale, h_X, h_Y, batch: int, d_ws, stream=None) -> None:
    """h_X / h_Y are host tensors (pinned for asynchronous copies); synchronise before reading h_Y."""
    c = fmt.c()
    _check(load().vq_gemm_small_batch_host(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale), _ptr(h_X),
                                           _ptr(h_Y), int(batch), _ptr(d_ws),
                                           d_ws.numel() * d_ws.element_size(), _stream(stream)),
           "vq_gemm_small_batch_host")


def vq_gemm_small_batch_host_static(fmt: VQFormat, d_idx, d_cb, d_scale, h_X, h_Y, batch: int, stream=None) -> None:
    """Host-buffer skinny GEMM that allocates nothing: the device copies of X and Y live in a
    fixed 2 MiB array inside the library (vq_static_scratch_bytes()).  For callers that may not
    call cudaMalloc.  Calls on one device share that array: keep them ordered on the GPU.
    Synchronise before reading h_Y."""
    c = fmt.c()
    _check(load().vq_gemm_small_batch_host_static(ctypes.byref(c), _ptr(d_idx), _ptr(d_cb), _ptr(d_scale),
                                                  _ptr(h_X), _ptr(h_Y), int(batch), _stream(stream)),
           "vq_gemm_small_batch_host_static")


def vq_static_scratch_bytes() -> int:
    return load().vq_static_scratch_bytes()


def vq_probe_decode_loop(policy: int, warps: int, batch: int, iters: int, d_scratch, stream=None):
    """(clocks per pass, weights decoded per pass and SM) of one policy's decode loop on resident data."""
    clocks, weights = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(load().vq_probe_decode_loop(int(policy), int(warps), int(batch), int(iters), _ptr(d_scratch),
                                       d_scratch.numel() * d_scratch.element_size(), ctypes.byref(clocks), ctypes.byref(weights),
                                       _stream(stream)), "vq_probe_decode_loop")
    return clocks.value, weights.value


def vq_probe_read(d_buf, d_out4, stream=None) -> None:
    _check(load().vq_probe_read(_ptr(d_buf), d_buf.numel() * d_buf.element_size(), _ptr(d_out4), _stream(stream)), "vq_probe_read")


def vq_device_wait_failures() -> int:
    """Bounded in-kernel waits that ran out on the current device (0 in a healthy run); synchronises."""
    out = ctypes.c_int(-1)
    _check(load().vq_device_wait_failures(ctypes.byref(out)), "vq_device_wait_failures")
    return out.value


def vq_int4g128_workspace_bytes(n_rows: int, batch: int) -> int:
    return load().vq_int4g128_workspace_bytes(int(n_rows), int(batch))


def vq_int4g128_gemm_small_batch(n_rows: int, k_cols: int, d_q, d_scale, d_X, d_Y, batch: int, d_ws, stream=None) -> None:
    _check(load().vq_int4g128_gemm_small_batch(int(n_rows), int(k_cols), _ptr(d_q), _ptr(d_scale), _ptr(d_X),
                                               _ptr(d_Y), int(batch), _ptr(d_ws), d_ws.numel() * d_ws.element_size(),
                                               _stream(stream)),
           "vq_int4g128_gemm_small_batch")


VQ_UNPACK_FP16, VQ_UNPACK_INT8_ROW, VQ_UNPACK_INT4_G128 = 0, 1, 2


def vq_unpack_uniform(kind: int, n_rows: int, k_cols: int, d_src, d_scale, d_W, stream=None) -> None:
    _check(load().vq_unpack_uniform(int(kind), int(n_rows), int(k_cols), _ptr(d_src), _ptr(d_scale), _ptr(d_W),
                                    _stream(stream)), "vq_unpack_uniform")


def vq_assign_indices(fmt: "VQFormat", d_W, d_cb, d_scale, d_hdiag, d_idx, stream=None) -> None:
    """E-step (Eq. 5): nearest centroid under diagonal weights; writes the packed index stream d_idx."""
    c = fmt.c()
    _check(load().vq_assign_indices(ctypes.byref(c), _ptr(d_W), _ptr(d_cb), _ptr(d_scale), _ptr(d_hdiag), _ptr(d_idx),
                                    _stream(stream)), "vq_assign_indices")



# ---- the cache, its attention, the residual stream ------------------------------------------------------------------

VQ_KV_FP16, VQ_KV_INT8 = 0, 1
VQ_KV_MAX_LAYERS = 120
VQ_NORM_RMS, VQ_NORM_LAYER = 0, 1
VQ_RESIDUAL_FP16, VQ_RESIDUAL_FP32 = 0, 1
VQ_GATE_NONE, VQ_GATE_CHANNEL, VQ_GATE_ELEMENT = 0, 1, 2


class _CKVFormat(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_tokens", "n_kv_heads", "head_dim", "kv_type")]


class _CKVPool(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("d_k", "d_v", "d_k_scale", "d_v_scale")]


class _CKVSeqs(ctypes.Structure):
    _fields_ = [("d_table", ctypes.c_void_p), ("d_len", ctypes.c_void_p), ("n_seqs", ctypes.c_int32), ("table_stride", ctypes.c_int32)]


class _CKVInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("pool_bytes", "scale_bytes", "page_bytes")]


class _CKVRotary(ctypes.Structure):
    _fields_ = [("d_cos_sin", ctypes.c_void_p), ("n_positions", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("d_q", ctypes.c_void_p), ("d_q_out", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("q_out_stride", ctypes.c_int64)]


class _CNormBlock(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("n_rows", "n_cols", "kind", "residual_type", "gate")] +
                [("eps", ctypes.c_float), ("residual_scale", ctypes.c_float)] +
                [(n, ctypes.c_int64) for n in ("x_stride", "y_stride", "gate_stride", "x_out_stride", "h_stride")])


# Formats and handles hold their C struct (the library only reads it): a call passes its address.

class _Held:
    __slots__ = ("_c", "_p", "device", "_size")   # (not among the fields; _size: values and rows of a pool)

    def _hold(self, struct, device=None, size=None) -> None:
        object.__setattr__(self, "_c", struct)
        object.__setattr__(self, "_p", ctypes.addressof(struct))
        object.__setattr__(self, "device", device)
        object.__setattr__(self, "_size", size)

    def __reduce__(self):   # (a copy gets a struct of its own: an address is this object's)
        return type(self), tuple(getattr(self, f.name) for f in fields(self))


@dataclass(frozen=True)
class VQKVFormat(_Held):
    n_pages: int
    page_tokens: int
    n_kv_heads: int
    head_dim: int
    kv_type: int

    def __post_init__(self):
        rows = self.n_pages * self.n_kv_heads * self.page_tokens
        self._hold(_CKVFormat(self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim, self.kv_type), None, (rows * self.head_dim, rows))

    def c(self) -> _CKVFormat:
        return self._c


@dataclass(frozen=True)
class KVInfo:
    pool_bytes: int
    scale_bytes: int
    page_bytes: int


def _device_of(*tensors):
    """Device index that all tensors share (-1: the host; None without tensors)."""
    devices = {t.get_device() for t in tensors if t is not None} or {None}
    if len(devices) != 1:
        raise ValueError(f"tensors on different devices: {sorted(devices)}")
    return devices.pop()


@dataclass(frozen=True, eq=False)
class KVPool(_Held):
    """One layer's pool: keys and values, and their scales for VQ_KV_INT8.  Holds the tensors; their memory has to stay where
    it is while the handle is used."""
    k: object
    v: object
    k_scale: object = None
    v_scale: object = None

    def __post_init__(self):
        import torch
        kinds = (torch.float16,) * 2 if self.k_scale is None and self.v_scale is None else (torch.int8, torch.int8, torch.float32, torch.float32)
        for t, kind in zip(self, kinds):
            if t is not None and (t.dtype != kind or not t.is_contiguous()):
                raise ValueError("KVPool: contiguous float16 keys and values, or int8 ones and float32 scales")
        # (what is missing is the library's to refuse)
        size = [min([t.numel() for t in pair if t is not None], default=1 << 62) for pair in ((self.k, self.v), (self.k_scale, self.v_scale))]
        self._hold(_CKVPool(*[_ptr(t) for t in self]), _device_of(*self), tuple(size))

    def __iter__(self):
        return iter((self.k, self.v, self.k_scale, self.v_scale))


@dataclass(frozen=True, eq=False)
class KVSeqs(_Held):
    """Page table (int32, a row per sequence) and lengths (int32).  Holds the tensors, as KVPool does."""
    table: object
    length: object

    def __post_init__(self):
        table, length = self.table, self.length
        import torch
        if table.dtype != torch.int32 or length.dtype != torch.int32:
            raise ValueError("KVSeqs: an int32 table and int32 lengths")
        if table.dim() != 2 or not table.is_contiguous() or length.dim() != 1 or not length.is_contiguous() or length.shape[0] != table.shape[0]:
            raise ValueError("KVSeqs: a contiguous table, and a length for each of its rows")
        self._hold(_CKVSeqs(table.data_ptr(), length.data_ptr(), table.shape[0], table.shape[1]), _device_of(table, length))


@dataclass(frozen=True, eq=False)
class KVRotary(_Held):
    """Cosines and sines, and the new tokens' queries (None: keys only).  Holds the tensors, as KVPool does."""
    d_cos_sin: object
    n_positions: int
    rot_dim: int
    interleaved: int
    n_q_heads: int = 0
    d_q: object = None
    q_stride: int = 0
    d_q_out: object = None
    q_out_stride: int = 0

    def __post_init__(self):
        import torch
        t = self.d_cos_sin
        if t is not None and (t.dtype != torch.float32 or not t.is_contiguous() or t.numel() < self.n_positions * self.rot_dim):
            raise ValueError("KVRotary: contiguous float32 cosines and sines, rot_dim of them for every position")
        for t in (self.d_q, self.d_q_out):
            if t is not None and t.dtype != torch.float16:
                raise ValueError("KVRotary: float16 queries")
        self._hold(_CKVRotary(_ptr(self.d_cos_sin), int(self.n_positions), int(self.rot_dim), int(self.interleaved), int(self.n_q_heads),
                              _ptr(self.d_q), _ptr(self.d_q_out), int(self.q_stride), int(self.q_out_stride)),
                   _device_of(self.d_cos_sin, self.d_q, self.d_q_out))


@dataclass(frozen=True)
class VQNorm(_Held):
    n_rows: int
    n_cols: int
    kind: int
    residual_type: int
    gate: int
    eps: float
    residual_scale: float
    x_stride: int
    y_stride: int = 0
    gate_stride: int = 0
    x_out_stride: int = 0
    h_stride: int = 0

    def __post_init__(self):
        self._hold(_CNormBlock(self.n_rows, self.n_cols, self.kind, self.residual_type, self.gate, self.eps, self.residual_scale, self.x_stride,
                               self.y_stride, self.gate_stride, self.x_out_stride, self.h_stride))

    def c(self) -> _CNormBlock:
        return self._c


class KVPools:
    """The pools of a cache's layers, in order (a list of KVPool does as well: it is laid out at every call)."""

    def __init__(self, pools):
        self.pools = tuple(pools)
        devices = {p.device for p in self.pools}
        if len(devices) > 1:
            raise ValueError(f"pools on different devices: {sorted(devices)}")
        self.device = devices.pop() if devices else None
        self._c = (_CKVPool * len(self.pools))(*[p._c for p in self.pools])
        self._p = ctypes.addressof(self._c)


def _pools(pools, fmt) -> KVPools:
    pools = pools if isinstance(pools, KVPools) else KVPools(pools)
    for p in pools.pools:
        _room(p, fmt)
    return pools


def _room(pool: KVPool, fmt: VQKVFormat) -> None:
    if pool._size[0] < fmt._size[0] or pool._size[1] < fmt._size[1]:
        raise ValueError("KVPool: tensors smaller than the pool that the format describes")


_current_device = None


def _device_now() -> int:
    global _current_device
    if _current_device is None:
        import torch
        _current_device = torch.cuda.current_device if torch.cuda.is_available() else lambda: 0
    return _current_device()


def _elsewhere(now, *operands):
    for t in operands:
        if t is not None:
            dev = t.get_device() if hasattr(t, "get_device") else t.device
            if dev is not None and dev != now:
                raise ValueError(f"operand on device {dev}, the current device is cuda:{now}")


_int32 = _float16 = _float32 = None


def _here(handles, *tensors) -> int:
    """The calls below launch on the current device, which is returned: operands of another one (or of the host) are refused."""
    if _int32 is None:
        _types()
    now = _device_now()
    for h in handles:
        if h.device != now:
            _elsewhere(now, *handles)
    for t in tensors:
        if t is not None and t.get_device() != now:
            _elsewhere(now, t)
    return now


def _types() -> None:
    global _int32, _float16, _float32
    import torch
    _int32, _float16, _float32 = torch.int32, torch.float16, torch.float32


def _of_type(now, dtype, *operands) -> None:
    for t in operands:
        if t is not None and (t.dtype is not dtype or t.get_device() != now):
            _elsewhere(now, t)
            raise ValueError(f"a {dtype} tensor is wanted, not {t.dtype}")


def _list(now, t, n: int) -> None:
    """A list of the books: contiguous int32, with the n entries that the call reads or writes.  What is missing is the library's to
    refuse."""
    if t is not None and (t.dtype is not _int32 or t.get_device() != now or t.numel() < n or not t.is_contiguous()):
        _elsewhere(now, t)
        raise ValueError(f"a contiguous int32 tensor of {n} entries or more is wanted, not {t.dtype} of {tuple(t.shape)}")


def _bytes(t) -> int:
    return t.numel() * t.element_size()


def vq_kv_info(fmt: VQKVFormat) -> KVInfo:
    out = _CKVInfo()
    _check(load().vq_kv_info(fmt._p, ctypes.byref(out)), "vq_kv_info")
    return KVInfo(int(out.pool_bytes), int(out.scale_bytes), int(out.page_bytes))


def vq_kv_attention_workspace_bytes(fmt: VQKVFormat) -> int:
    return load().vq_kv_attention_workspace_bytes(fmt._p)


def vq_kv_attention(fmt: VQKVFormat, pool: KVPool, seqs: KVSeqs, n_q_heads: int, d_q, q_stride: int, d_out, out_stride: int, d_lse, scale: float,
                    window: int, d_ws, stream=None) -> None:
    """One new token per sequence over the paged cache; window 0: all of it.  d_lse may be None."""
    now = _here((pool, seqs), d_ws)
    _of_type(now, _float16, d_q, d_out)
    _of_type(now, _float32, d_lse)
    _room(pool, fmt)
    _check(load().vq_kv_attention(fmt._p, pool._p, seqs._p, n_q_heads, _ptr(d_q), q_stride, _ptr(d_out), out_stride, _ptr(d_lse), scale,
                                  window, d_ws.data_ptr(), _bytes(d_ws), _stream(stream)), "vq_kv_attention")


def vq_kv_append(fmt: VQKVFormat, pool: KVPool, seqs: KVSeqs, d_starts, n_tokens: int, d_k, k_stride: int, d_v, v_stride: int,
                 rotary: KVRotary | None = None, stream=None) -> None:
    """New tokens into the cache.  d_starts None: one token per sequence."""
    now = _here((pool, seqs) if rotary is None else (pool, seqs, rotary))
    _list(now, d_starts, seqs._c.n_seqs + 1)
    _of_type(now, _float16, d_k, d_v)
    _room(pool, fmt)
    _check(load().vq_kv_append(fmt._p, pool._p, seqs._p, _ptr(d_starts), n_tokens, _ptr(d_k), k_stride, _ptr(d_v), v_stride,
                               None if rotary is None else rotary._p, _stream(stream)), "vq_kv_append")


def vq_kv_pages_workspace_bytes(fmt: VQKVFormat, n_seqs: int) -> int:
    return load().vq_kv_pages_workspace_bytes(fmt._p, n_seqs)


def vq_kv_reserve(fmt: VQKVFormat, seqs: KVSeqs, d_refs, d_new, d_status, d_ws, stream=None) -> None:
    """Room for d_new tokens per sequence (None: one each); d_status: pages missing, sequences too long."""
    now = _here((seqs,), d_ws)
    _list(now, d_refs, fmt.n_pages)
    _list(now, d_new, seqs._c.n_seqs)
    _list(now, d_status, 2)
    _check(load().vq_kv_reserve(fmt._p, seqs._p, _ptr(d_refs), _ptr(d_new), _ptr(d_status), d_ws.data_ptr(), _bytes(d_ws),
                                _stream(stream)), "vq_kv_reserve")


def vq_kv_fork(fmt: VQKVFormat, pools, seqs: KVSeqs, d_refs, d_pairs, n_pairs: int, d_status, d_ws, stream=None) -> None:
    """pools: a KVPool per layer (KVPools).  d_pairs: (parent, child) rows; d_status: pages missing, entries left out."""
    pools = _pools(pools, fmt)
    now = _here((pools, seqs), d_ws)
    _list(now, d_refs, fmt.n_pages)
    _list(now, d_pairs, 2 * n_pairs)
    _list(now, d_status, 2)
    _check(load().vq_kv_fork(fmt._p, pools._p, len(pools.pools), seqs._p, _ptr(d_refs), _ptr(d_pairs), n_pairs, _ptr(d_status),
                             d_ws.data_ptr(), _bytes(d_ws), _stream(stream)), "vq_kv_fork")


def vq_kv_free(fmt: VQKVFormat, seqs: KVSeqs, d_refs, d_slots, n_slots: int, stream=None) -> None:
    now = _here((seqs,))
    _list(now, d_refs, fmt.n_pages)
    _list(now, d_slots, n_slots)
    _check(load().vq_kv_free(fmt._p, seqs._p, _ptr(d_refs), _ptr(d_slots), n_slots, _stream(stream)), "vq_kv_free")


def vq_kv_compact(fmt: VQKVFormat, pools, seqs: KVSeqs, d_refs, d_status, d_ws, stream=None) -> None:
    """d_status: pages in use, pages moved."""
    pools = _pools(pools, fmt)
    now = _here((pools, seqs), d_ws)
    _list(now, d_refs, fmt.n_pages)
    _list(now, d_status, 2)
    _check(load().vq_kv_compact(fmt._p, pools._p, len(pools.pools), seqs._p, _ptr(d_refs), _ptr(d_status), d_ws.data_ptr(), _bytes(d_ws),
                                _stream(stream)), "vq_kv_compact")


def vq_kv_copy_pages(fmt: VQKVFormat, pools, d_pairs, n_pairs: int, stream=None) -> None:
    pools = _pools(pools, fmt)
    _list(_here((pools,)), d_pairs, 2 * n_pairs)
    _check(load().vq_kv_copy_pages(fmt._p, pools._p, len(pools.pools), _ptr(d_pairs), n_pairs, _stream(stream)), "vq_kv_copy_pages")


def vq_residual_norm(norm: VQNorm, d_x, d_y, d_gate, d_post_w, d_post_b, d_pre_w, d_pre_b, d_x_out, d_h, stream=None) -> None:
    """x' = x + residual_scale * gate * post(y), h = pre(x'); absent operands are None."""
    now = _here(())
    _of_type(now, _float16, d_y, d_gate, d_post_w, d_post_b, d_pre_w, d_pre_b, d_h)
    _of_type(now, _float32 if norm.residual_type == VQ_RESIDUAL_FP32 else _float16, d_x, d_x_out)
    _check(load().vq_residual_norm(norm._p, _ptr(d_x), _ptr(d_y), _ptr(d_gate), _ptr(d_post_w), _ptr(d_post_b), _ptr(d_pre_w), _ptr(d_pre_b),
                                   _ptr(d_x_out), _ptr(d_h), _stream(stream)), "vq_residual_norm")
