"""MI355X-native QK4PV8 FlashAttention (MpFA): thin Python binding of libmpfa.so.

Argument marshalling only: torch tensors provide device memory and the current
stream; every step of the attention path runs in the library's HIP kernels.
The binding raises if the compiled library is missing — there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
DEBUG_LIB_PATH = os.path.join(PKG_DIR, "libmpfa_debug.so")
# MPFA_DEBUG=1 loads the twin library whose entry points also check the data
# they are handed (index ranges, non-finite inputs) before launching
LIB_PATH = DEBUG_LIB_PATH if os.environ.get("MPFA_DEBUG") == "1" else os.path.join(PKG_DIR, "libmpfa.so")

(MPFA_OK, MPFA_ERR_INVALID, MPFA_ERR_UNSUPPORTED, MPFA_ERR_WORKSPACE, MPFA_ERR_HIP,
 MPFA_ERR_DATA) = range(6)
SMOOTH, COMPUTE_STATS, TSCALE_UNIT, SEED_MFMA, MXFP4, SEED_ELEMWISE = 1, 2, 4, 8, 16, 32
PV_BF16, PV_NVFP4 = 64, 128
KV4_IN_PLACE, KV4_WEIGHTS = 256, 512
HEAD_DIM, PAGE, TILE = 128, 64, 128
STATIC_SCRATCH_BYTES = 64 << 20   # MPFA_STATIC_SCRATCH_BYTES

EXPORTED = ("mpfa_quantize_qk", "mpfa_prefill", "mpfa_decode_workspace_size",
            "mpfa_decode_choose_partition", "mpfa_decode_paged", "mpfa_decode_paged_static",
            "mpfa_mixed_workspace_size",
            "mpfa_mixed_step", "mpfa_convert", "mpfa_status_string", "mpfa_version",
            "mpfa_kv4_write_workspace_size", "mpfa_kv4_write", "mpfa_kv4_prefill_plan", "mpfa_kv4_prefill",
            "mpfa_kv4_decode_plan", "mpfa_kv4_decode", "mpfa_kv4_evict",
            "mpfa_linear_prefill_workspace_size", "mpfa_linear_prefill", "mpfa_linear_decode", "mpfa_rms_norm")


class MpfaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


class QuantArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_tokens", C.c_int32), ("max_seqlen", C.c_int32),
                ("h_q", C.c_int32), ("h_kv", C.c_int32), ("head_dim", C.c_int32),
                ("flags", C.c_uint32), ("num_pages", C.c_int64),
                ("cu_seqlens", C.c_void_p), ("q", C.c_void_p), ("k", C.c_void_p),
                ("v", C.c_void_p), ("slot_mapping", C.c_void_p), ("q_mean", C.c_void_p),
                ("k_mean", C.c_void_p), ("k_tscale", C.c_void_p), ("q_codes", C.c_void_p),
                ("q_scales", C.c_void_p), ("q_tscale", C.c_void_p), ("k_codes", C.c_void_p),
                ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("ds", C.c_void_p),
                ("v_aux", C.c_void_p)]


class PrefillArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("h_q", C.c_int32), ("h_kv", C.c_int32),
                ("head_dim", C.c_int32), ("max_seqlen_q", C.c_int32), ("max_pages", C.c_int32),
                ("flags", C.c_uint32), ("cu_seqlens_q", C.c_void_p), ("q_start", C.c_void_p),
                ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("q_codes", C.c_void_p),
                ("q_scales", C.c_void_p), ("q_tscale", C.c_void_p), ("k_codes", C.c_void_p),
                ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("ds", C.c_void_p),
                ("k_tscale", C.c_void_p), ("out", C.c_void_p), ("v_aux", C.c_void_p),
                ("num_pages", C.c_int64)]


class DecodeArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("h_q", C.c_int32), ("h_kv", C.c_int32),
                ("head_dim", C.c_int32), ("max_pages", C.c_int32),
                ("partition_tokens", C.c_int32), ("max_partitions", C.c_int32),
                ("flags", C.c_uint32), ("kv_len", C.c_void_p), ("page_table", C.c_void_p),
                ("q_codes", C.c_void_p), ("q_scales", C.c_void_p), ("q_tscale", C.c_void_p),
                ("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p),
                ("ds", C.c_void_p), ("k_tscale", C.c_void_p), ("out", C.c_void_p),
                ("num_pages", C.c_int64)]


class Kv4Cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p),
                ("v_scales", C.c_void_p), ("weights", C.c_void_p), ("num_pages", C.c_int64)]


class Kv4Item(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("seq", "row", "first", "last", "state", "parts")]


class Kv4WriteArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_tokens", C.c_int32), ("max_seqlen", C.c_int32),
                ("h_kv", C.c_int32), ("head_dim", C.c_int32), ("flags", C.c_uint32),
                ("k_stride", C.c_int64), ("v_stride", C.c_int64), ("cu_seqlens", C.c_void_p),
                ("k", C.c_void_p), ("v", C.c_void_p), ("slot_mapping", C.c_void_p), ("k_mean", C.c_void_p),
                ("k_tscale", C.c_void_p), ("v_tscale", C.c_void_p), ("cache", Kv4Cache),
                ("k_out", C.c_void_p), ("v_out", C.c_void_p)]


class Kv4AttnArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("h_q", C.c_int32), ("h_kv", C.c_int32), ("head_dim", C.c_int32),
                ("max_pages", C.c_int32), ("total_tokens", C.c_int32), ("max_seqlen_q", C.c_int32),
                ("q_tokens", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32),
                ("partition_tokens", C.c_int32), ("max_partitions", C.c_int32), ("n_items", C.c_int32),
                ("n_merges", C.c_int32), ("n_states", C.c_int32), ("half", C.c_int32), ("flags", C.c_uint32),
                ("q_stride", C.c_int64), ("cu_seqlens_q", C.c_void_p), ("q_start", C.c_void_p), ("items", C.c_void_p),
                ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("q", C.c_void_p), ("cache", Kv4Cache),
                ("k_tscale", C.c_void_p), ("v_tscale", C.c_void_p), ("out", C.c_void_p)]


class Kv4EvictArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("h_kv", C.c_int32), ("max_pages", C.c_int32),
                ("dst_max_pages", C.c_int32), ("budget", C.c_int32), ("sinks", C.c_int32),
                ("recent", C.c_int32), ("flags", C.c_uint32), ("kv_len", C.c_void_p),
                ("page_table", C.c_void_p), ("dst_page_table", C.c_void_p), ("cache", Kv4Cache),
                ("kept", C.c_void_p), ("new_len", C.c_void_p)]


class LinearArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_tokens", C.c_int32), ("max_seqlen", C.c_int32), ("q_tokens", C.c_int32),
                ("h_q", C.c_int32), ("h_kv", C.c_int32), ("head_dim", C.c_int32), ("flags", C.c_uint32), ("scale", C.c_float),
                ("num_states", C.c_int32), ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("decay_stride", C.c_int64), ("cu_seqlens", C.c_void_p), ("q", C.c_void_p), ("k", C.c_void_p),
                ("v", C.c_void_p), ("log_decay", C.c_void_p), ("state_src", C.c_void_p), ("state_dst", C.c_void_p),
                ("states", C.c_void_p), ("out", C.c_void_p)]


class RmsNormArgs(C.Structure):
    _fields_ = [("rows", C.c_int32), ("width", C.c_int32), ("group", C.c_int32), ("eps", C.c_float), ("x_stride", C.c_int64),
                ("x", C.c_void_p), ("weight", C.c_void_p), ("residual", C.c_void_p), ("residual_out", C.c_void_p),
                ("out", C.c_void_p), ("scales", C.c_void_p)]


_libs: dict = {}


def lib():
    """Load libmpfa.so (built in-tree by build.py); raise if it is missing."""
    return _load(LIB_PATH)


def debug_lib():
    """Load libmpfa_debug.so: the same kernels behind entry points that also
    check the data (index ranges, non-finite inputs) and return MPFA_ERR_DATA."""
    return _load(DEBUG_LIB_PATH)


def _load(path):
    if path not in _libs:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built; run paper_2609_33135_amd/build.py")
        L = C.CDLL(path)
        L.mpfa_quantize_qk.restype = C.c_int
        L.mpfa_quantize_qk.argtypes = [C.POINTER(QuantArgs), C.c_void_p]
        L.mpfa_prefill.restype = C.c_int
        L.mpfa_prefill.argtypes = [C.POINTER(PrefillArgs), C.c_void_p]
        L.mpfa_decode_workspace_size.restype = C.c_int
        L.mpfa_decode_workspace_size.argtypes = [C.c_int32, C.c_int32, C.c_int32,
                                                 C.POINTER(C.c_size_t)]
        L.mpfa_decode_choose_partition.restype = C.c_int
        L.mpfa_decode_choose_partition.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_int32,
                                                   C.POINTER(C.c_int32)]
        L.mpfa_decode_paged.restype = C.c_int
        L.mpfa_decode_paged.argtypes = [C.POINTER(DecodeArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        L.mpfa_decode_paged_static.restype = C.c_int
        L.mpfa_decode_paged_static.argtypes = [C.POINTER(DecodeArgs), C.c_void_p]
        L.mpfa_mixed_workspace_size.restype = C.c_int
        L.mpfa_mixed_workspace_size.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                                C.POINTER(C.c_size_t)]
        L.mpfa_mixed_step.restype = C.c_int
        L.mpfa_mixed_step.argtypes = [C.POINTER(PrefillArgs), C.POINTER(DecodeArgs), C.c_void_p,
                                      C.c_size_t, C.c_void_p]
        L.mpfa_convert.restype = C.c_int
        L.mpfa_convert.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        i32, out, size = C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_size_t)
        for name, args in (
                ("mpfa_kv4_write_workspace_size", [i32, i32, i32, size]),
                ("mpfa_kv4_write", [C.POINTER(Kv4WriteArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
                ("mpfa_kv4_prefill_plan", [i32, C.c_void_p, C.c_void_p, i32, i32, i32, i32, i32, C.c_void_p, i32,
                                           out, out, out, out, size]),
                ("mpfa_kv4_prefill", [C.POINTER(Kv4AttnArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
                ("mpfa_kv4_decode_plan", [i32, C.c_void_p, i32, i32, i32, i32, i32, C.c_uint32, i32, out, out, size]),
                ("mpfa_kv4_decode", [C.POINTER(Kv4AttnArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
                ("mpfa_kv4_evict", [C.POINTER(Kv4EvictArgs), C.c_void_p]),
                ("mpfa_linear_prefill_workspace_size", [i32, i32, i32, i32, i32, size]),
                ("mpfa_linear_prefill", [C.POINTER(LinearArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
                ("mpfa_linear_decode", [C.POINTER(LinearArgs), C.c_void_p]),
                ("mpfa_rms_norm", [C.POINTER(RmsNormArgs), C.c_void_p])):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = args
        L.mpfa_status_string.restype = C.c_char_p
        L.mpfa_status_string.argtypes = [C.c_int]
        L.mpfa_version.restype = C.c_char_p
        _libs[path] = L
    return _libs[path]


def status_string(s: int) -> str:
    return lib().mpfa_status_string(s).decode()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    """Handle of the stream, by default torch's current one.  The Stream object that
    torch.cuda.current_stream() builds for it takes 2.7 us, the handle alone 0.2 us,
    of 9.6 us that a call of a few tokens took; positional arguments of the structures
    below save 0.7 us more."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(rc: int, what: str):
    if rc != MPFA_OK:
        raise MpfaError(rc, what)


class PagedCache:
    """Device buffers of the paged NVFP4/FP8 KV cache and the Delta_S side cache."""

    def __init__(self, num_pages: int, h_q: int, h_kv: int, device="cuda", smooth=True, pv=0):
        """pv: 0, PV_BF16 or PV_NVFP4 (adds the V copy of that precision, v_aux)."""
        import torch
        self.num_pages, self.h_q, self.h_kv = num_pages, h_q, h_kv
        u8 = dict(dtype=torch.uint8, device=device)
        self.k_codes = torch.zeros((num_pages, h_kv, PAGE, 64), **u8)
        self.k_scales = torch.zeros((num_pages, h_kv, PAGE, 8), **u8)
        self.v_codes = torch.zeros((num_pages, h_kv, HEAD_DIM, PAGE), **u8)
        self.ds = torch.zeros((num_pages, h_q, PAGE), dtype=torch.bfloat16, device=device) \
            if smooth else None
        self.v_aux = None
        if pv == PV_BF16:
            self.v_aux = torch.zeros((num_pages, h_kv, HEAD_DIM, PAGE), dtype=torch.bfloat16,
                                     device=device)
        elif pv == PV_NVFP4:   # code plane [P][H][128][32], then scale plane [P][H][128][4]
            self.v_aux = torch.zeros(num_pages * h_kv * HEAD_DIM * 36, **u8)


class SeqStats:
    """Per-sequence statistics frozen after the first prefill (means, K tensor scale)."""

    def __init__(self, batch: int, h_q: int, h_kv: int, device="cuda"):
        import torch
        self.q_mean = torch.zeros((batch, h_q, HEAD_DIM), dtype=torch.bfloat16, device=device)
        self.k_mean = torch.zeros((batch, h_kv, HEAD_DIM), dtype=torch.bfloat16, device=device)
        self.k_tscale = torch.ones((batch, h_kv), dtype=torch.float32, device=device)


class QuantQ:
    """NVFP4 queries of one call: codes [T][H][64], scales [T][H][8], tensor scale [B][H]."""

    def __init__(self, total: int, batch: int, h_q: int, device="cuda"):
        import torch
        self.codes = torch.zeros((total, h_q, 64), dtype=torch.uint8, device=device)
        self.scales = torch.zeros((total, h_q, 8), dtype=torch.uint8, device=device)
        self.tscale = torch.zeros((batch, h_q), dtype=torch.float32, device=device)


def quantize_qk(q, k, v, cu_seqlens, slot_mapping, cache: PagedCache, stats: SeqStats,
                qout: QuantQ, flags: int, max_seqlen: int, stream=None):
    """mpfa_quantize_qk: q bf16 [T][Hq][128], k/v bf16 [T][Hkv][128] on the device."""
    T, h_q, d = q.shape
    a = QuantArgs(cu_seqlens.numel() - 1, T, max_seqlen, h_q, k.shape[1], d, flags, cache.num_pages,
                  _ptr(cu_seqlens), _ptr(q), _ptr(k), _ptr(v), _ptr(slot_mapping), _ptr(stats.q_mean),
                  _ptr(stats.k_mean), _ptr(stats.k_tscale), _ptr(qout.codes), _ptr(qout.scales),
                  _ptr(qout.tscale), _ptr(cache.k_codes), _ptr(cache.k_scales), _ptr(cache.v_codes),
                  _ptr(cache.ds), _ptr(cache.v_aux))
    _check(lib().mpfa_quantize_qk(C.byref(a), _stream(stream)), "mpfa_quantize_qk")


def _prefill_args(qq, cache, stats, cu_seqlens_q, q_start, kv_len, page_table, out, max_seqlen_q, flags, v_aux):
    return PrefillArgs(cu_seqlens_q.numel() - 1, qq.codes.shape[1], cache.h_kv, HEAD_DIM, max_seqlen_q,
                       page_table.shape[1], flags, _ptr(cu_seqlens_q), _ptr(q_start), _ptr(kv_len),
                       _ptr(page_table), _ptr(qq.codes), _ptr(qq.scales), _ptr(qq.tscale),
                       _ptr(cache.k_codes), _ptr(cache.k_scales), _ptr(cache.v_codes), _ptr(cache.ds),
                       _ptr(stats.k_tscale), _ptr(out), _ptr(v_aux), cache.num_pages)


def prefill(qq: QuantQ, cache: PagedCache, stats: SeqStats, cu_seqlens_q, q_start, kv_len,
            page_table, out, max_seqlen_q: int, flags: int, stream=None):
    """mpfa_prefill: causal attention of the quantized queries over the paged cache."""
    a = _prefill_args(qq, cache, stats, cu_seqlens_q, q_start, kv_len, page_table, out, max_seqlen_q, flags,
                      cache.v_aux)
    _check(lib().mpfa_prefill(C.byref(a), _stream(stream)), "mpfa_prefill")


def decode_workspace_size(batch: int, h_q: int, max_partitions: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mpfa_decode_workspace_size(batch, h_q, max_partitions, C.byref(n)),
           "mpfa_decode_workspace_size")
    return n.value


def decode_choose_partition(kv_len_host, h_kv: int, num_cus: int) -> int:
    import numpy as np
    kl = np.ascontiguousarray(kv_len_host, dtype=np.int32)
    out = C.c_int32(0)
    _check(lib().mpfa_decode_choose_partition(kl.size, kl.ctypes.data, h_kv, num_cus,
                                              C.byref(out)), "mpfa_decode_choose_partition")
    return out.value


def decode_paged(qq: QuantQ, cache: PagedCache, stats: SeqStats, kv_len, page_table, out,
                 partition_tokens: int, max_partitions: int, workspace, flags: int, stream=None):
    """mpfa_decode_paged: one query per sequence (qq rows indexed by sequence)."""
    a = _decode_args(qq, cache, stats, kv_len, page_table, out, partition_tokens, max_partitions, flags)
    _check(lib().mpfa_decode_paged(C.byref(a), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)),
           "mpfa_decode_paged")


def _decode_args(qq, cache, stats, kv_len, page_table, out, partition_tokens, max_partitions, flags):
    return DecodeArgs(kv_len.numel(), qq.codes.shape[1], cache.h_kv, HEAD_DIM, page_table.shape[1],
                      partition_tokens, max_partitions, flags, _ptr(kv_len), _ptr(page_table),
                      _ptr(qq.codes), _ptr(qq.scales), _ptr(qq.tscale), _ptr(cache.k_codes),
                      _ptr(cache.k_scales), _ptr(cache.v_codes), _ptr(cache.ds), _ptr(stats.k_tscale),
                      _ptr(out), cache.num_pages)


def decode_paged_static(qq: QuantQ, cache: PagedCache, stats: SeqStats, kv_len, page_table, out,
                        partition_tokens: int, max_partitions: int, flags: int, stream=None):
    """mpfa_decode_paged_static: decode_paged with the partition states in the
    library's per-GPU scratch array instead of a caller workspace (for callers
    that cannot allocate; calls on one GPU must not overlap)."""
    a = _decode_args(qq, cache, stats, kv_len, page_table, out, partition_tokens, max_partitions, flags)
    _check(lib().mpfa_decode_paged_static(C.byref(a), _stream(stream)), "mpfa_decode_paged_static")


def mixed_workspace_size(batch: int, h_q: int, h_kv: int, max_partitions: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mpfa_mixed_workspace_size(batch, h_q, h_kv, max_partitions, C.byref(n)),
           "mpfa_mixed_workspace_size")
    return n.value


def mixed_step(pre: dict, dec: dict, workspace, flags: int, stream=None):
    """mpfa_mixed_step: one launch for a prefill (keyword arguments of prefill())
    and a decode (keyword arguments of decode_paged() without the workspace and
    flags); the workspace must start zeroed (torch.zeros) and stays zeroed."""
    pa = _prefill_args(pre["qq"], pre["cache"], pre["stats"], pre["cu_seqlens_q"], pre["q_start"],
                       pre["kv_len"], pre["page_table"], pre["out"], pre["max_seqlen_q"], flags, None)
    da = _decode_args(dec["qq"], dec["cache"], dec["stats"], dec["kv_len"], dec["page_table"], dec["out"],
                      dec["partition_tokens"], dec["max_partitions"], flags)
    _check(lib().mpfa_mixed_step(C.byref(pa), C.byref(da), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)),
           "mpfa_mixed_step")


def convert(fmt: int, x, out, stream=None):
    """mpfa_convert: fmt 0 FP32 -> E4M3, fmt 1 FP32 -> E2M1 (one code per byte),
    written from the format definitions; fmt 2 / 3 the same through the hardware
    converters the quantization pass uses; 0x100 + c: E2M1 of x / e4m3(c) by the
    NVFP4 quantizer's division; 0x200 + b: E2M1 of x / 2^(b-127) (MXFP4);
    0x300 + c / 0x400 + b: the same quotients from their definitions (IEEE
    division, exact scaling) through the fmt 1 encoder."""
    _check(lib().mpfa_convert(fmt, _ptr(x), x.numel(), _ptr(out), _stream(stream)), "mpfa_convert")


# ---- the 4-bit cache: writer, windowed attention, eviction ------------------------------

def _same(what, dtype, dev, *tensors):
    """Contiguous tensors of one type on one device, or ValueError."""
    for t in tensors:
        if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"{what}: a tensor is {t.dtype}, device {t.get_device()}, "
                             f"{'' if t.is_contiguous() else 'not '}contiguous; "
                             f"wanted contiguous {dtype} on device {dev}")


def _rows(what, t, heads, dev):
    """Token stride of a bf16 [T][heads][128] tensor whose tokens may lie apart (a slice of a
    fused projection), or ValueError."""
    import torch
    shape, stride = t.shape, t.stride()
    if (t.dtype is not torch.bfloat16 or t.get_device() != dev or len(shape) != 3 or shape[1] != heads or
            shape[2] != HEAD_DIM or stride[2] != 1 or (heads > 1 and stride[1] != HEAD_DIM)):
        raise ValueError(f"{what}: bf16 [T][{heads}][{HEAD_DIM}] on device {dev} with contiguous heads is wanted, got "
                         f"{t.dtype} {tuple(shape)} strides {stride} on device {t.get_device()}")
    return stride[0] if shape[0] > 1 else heads * HEAD_DIM   # of one token any stride will do


def _want(ok, what):
    if not ok:
        raise ValueError(what)


def _call(name, dev, stream, *args):
    """The library call on the tensors' device (made current for it) and its current stream, or the
    given one; returns the stream's handle."""
    import torch
    if dev < 0:
        raise ValueError(f"{name}: tensors on a GPU are wanted")
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            return _call(name, dev, stream, *args)
    on = _stream(stream)
    rc = getattr(lib(), name)(*args, on)
    if rc:
        _check(rc, name)
    return on


class _Tensors:
    """Tensors named once: they are read as attributes, and their addresses are taken when the
    object is made (a call of a few tokens takes 2 us less so)."""

    def __init__(self, tensors):
        object.__setattr__(self, "_at", {n: _ptr(t) for n, t in tensors.items()})
        self.__dict__.update(tensors)

    def __setattr__(self, name, value):
        if name in self._at:
            raise AttributeError(f"{name} belongs to the object: make a new one for other tensors")
        object.__setattr__(self, name, value)


class PagedCache4(_Tensors):
    """Planes of the paged 4-bit cache (NVFP4 K and V); weights: with the FP32 weight per
    token that decode accumulates and eviction reads.  planes: existing tensors by plane
    name instead of new zeroed ones."""

    def __init__(self, num_pages: int, h_kv: int, device="cuda", weights=False, planes=None):
        import torch
        shapes = dict(k_codes=(PAGE, 64), k_scales=(PAGE, 8), v_codes=(PAGE, 64), v_scales=(8, PAGE), weights=(PAGE,))
        if planes is None:
            planes = {n: torch.zeros((num_pages, h_kv, *s), device=device,
                                     dtype=torch.float32 if n == "weights" else torch.uint8)
                      for n, s in shapes.items() if weights or n != "weights"}
        found = {n: planes.get(n) for n in shapes}
        _want(all(t is not None or n == "weights" for n, t in found.items()), "PagedCache4: a plane is missing")
        dev = found["k_codes"].get_device()
        for n, t in found.items():
            if t is not None:
                _same("PagedCache4", torch.float32 if n == "weights" else torch.uint8, dev, t)
                _want(tuple(t.shape) == (num_pages, h_kv, *shapes[n]), f"PagedCache4: {n} has shape {tuple(t.shape)}")
        super().__init__(found)
        self.num_pages, self.h_kv, self.device = num_pages, h_kv, dev
        self._c = Kv4Cache(*self._at.values(), num_pages)


class SeqStats4(_Tensors):
    """Per-sequence statistics of the 4-bit cache, frozen after a sequence's first write: K mean
    and the tensor scales of K and V (existing tensors may be given)."""

    def __init__(self, batch: int, h_kv: int, device="cuda", k_mean=None, k_tscale=None, v_tscale=None):
        import torch
        new = dict(dtype=torch.float32, device=device)
        kt = torch.ones((batch, h_kv), **new) if k_tscale is None else k_tscale
        vt = torch.ones((batch, h_kv), **new) if v_tscale is None else v_tscale
        mean = torch.zeros((batch, h_kv, HEAD_DIM), dtype=torch.bfloat16, device=kt.device) if k_mean is None else k_mean
        dev = kt.get_device()
        _same("SeqStats4", torch.float32, dev, kt, vt)
        _same("SeqStats4", torch.bfloat16, dev, mean)
        _want(tuple(kt.shape) == tuple(vt.shape) == (batch, h_kv) and tuple(mean.shape) == (batch, h_kv, HEAD_DIM),
              "SeqStats4: shapes")
        super().__init__(dict(k_mean=mean, k_tscale=kt, v_tscale=vt))
        self.batch, self.h_kv, self.device = batch, h_kv, dev


class Kv4Plan:
    """How a prefill or decode call is cut, and its workspace.  A plan serves one call at a time.
    A decode plan holds for every length up to those it was made for, a prefill plan for its
    row counts and lengths alone.

    Its workspace and items are made on the current stream.  A call on another stream waits for
    that one first, as for any tensor (Stream.wait_stream); the plan may be dropped as soon as
    the call returns, whichever stream it is on.  The plan of a captured call lives as long as
    the graph."""

    def __init__(self, what, workspace, home=None, **kw):
        self.what, self.workspace = what, workspace
        self.home = home   # handle of the stream that the workspace and the items were made on
        self.partition_tokens = self.max_partitions = self.n_items = self.n_merges = self.n_states = self.half = 0
        self.q_tokens = self.flags = self.max_rows = self.rows = 0
        self.items = None
        self.__dict__.update(kw)

    def cut(self):
        """The fields of Kv4AttnArgs that the plan sets: q_tokens, then partition_tokens .. flags."""
        return (self.q_tokens, self.partition_tokens, self.max_partitions, self.n_items, self.n_merges, self.n_states,
                self.half, self.flags)


def _host_ints(x):
    import numpy as np
    return np.ascontiguousarray(x, dtype=np.int32)


def _units(device):
    import torch
    dev = torch.device(device)
    return dev, torch.cuda.get_device_properties(dev).multi_processor_count


def _workspace(size, dev):
    import torch
    return torch.empty(size, dtype=torch.uint8, device=dev) if size else None


def _home(dev):
    """Handle of the stream that tensors of the device are made on now."""
    import torch
    return torch.cuda.current_stream(dev).cuda_stream


def kv4_prefill_plan(rows_host, kv_len_host, h_q: int, h_kv: int, window=0, sinks=0, device="cuda") -> Kv4Plan:
    """mpfa_kv4_prefill_plan, its items on the device and its workspace: rows and keys (the call's
    rows included) per sequence."""
    import numpy as np
    import torch
    rows, kv = _host_ints(rows_host), _host_ints(kv_len_host)
    _want(rows.size == kv.size, "kv4_prefill_plan: as many row counts as lengths are wanted")
    dev, cus = _units(device)
    n, merges, states, half, size = C.c_int32(0), C.c_int32(0), C.c_int32(0), C.c_int32(0), C.c_size_t(0)
    room = 256
    while True:
        items = np.empty((room, 6), np.int32)
        rc = lib().mpfa_kv4_prefill_plan(rows.size, rows.ctypes.data, kv.ctypes.data, h_q, h_kv, window, sinks, cus,
                                         items.ctypes.data, room, C.byref(n), C.byref(merges), C.byref(states), C.byref(half),
                                         C.byref(size))
        if rc != MPFA_ERR_WORKSPACE or n.value + merges.value <= room:
            break
        room = n.value + merges.value
    _check(rc, "mpfa_kv4_prefill_plan")
    used = items[:n.value + merges.value]
    return Kv4Plan(("prefill", rows.size, h_q, h_kv, window, sinks), _workspace(size.value, dev), _home(dev), n_items=n.value,
                   n_merges=merges.value, n_states=states.value, half=half.value, max_rows=int(rows.max()), rows=int(rows.sum()),
                   items=torch.from_numpy(used).to(dev) if n.value else None)


def kv4_decode_plan(kv_len_host, h_q: int, h_kv: int, q_tokens=1, window=0, sinks=0, weights=False,
                    device="cuda") -> Kv4Plan:
    """mpfa_kv4_decode_plan with its workspace; weights: the calls accumulate attention weights."""
    kv, flags = _host_ints(kv_len_host), KV4_WEIGHTS if weights else 0
    dev, cus = _units(device)
    part, maxp, size = C.c_int32(0), C.c_int32(0), C.c_size_t(0)
    _check(lib().mpfa_kv4_decode_plan(kv.size, kv.ctypes.data, h_q, h_kv, q_tokens, window, sinks, flags, cus, C.byref(part),
                                      C.byref(maxp), C.byref(size)), "mpfa_kv4_decode_plan")
    return Kv4Plan(("decode", kv.size, h_q, h_kv, window, sinks), _workspace(size.value, dev), _home(dev), partition_tokens=part.value,
                   max_partitions=maxp.value, q_tokens=q_tokens, flags=flags)


def kv4_write_workspace_size(batch: int, total_tokens: int, h_kv: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mpfa_kv4_write_workspace_size(batch, total_tokens, h_kv, C.byref(n)), "mpfa_kv4_write_workspace_size")
    return n.value


def kv4_write(k, v, cu_seqlens, slot_mapping, cache: PagedCache4, stats: SeqStats4, flags: int, max_seqlen: int,
              workspace=None, k_out=None, v_out=None, stream=None):
    """mpfa_kv4_write: k, v bf16 [T][Hkv][128] (tokens may lie apart) into the 4-bit cache; workspace:
    kv4_write_workspace_size bytes, with COMPUTE_STATS."""
    import torch
    dev, h_kv, T, batch = cache.device, cache.h_kv, k.shape[0], cu_seqlens.numel() - 1
    ks, vs = _rows("kv4_write: k", k, h_kv, dev), _rows("kv4_write: v", v, h_kv, dev)
    _same("kv4_write", torch.int32, dev, cu_seqlens)
    _same("kv4_write", torch.int64, dev, slot_mapping)
    if v.shape[0] != T or slot_mapping.numel() != T:
        raise ValueError("kv4_write: as many V rows and slots as K rows are wanted")
    if stats.batch != batch or stats.h_kv != h_kv or stats.device != dev:
        raise ValueError("kv4_write: stats of another batch")
    out, size = [None, None], 0
    for i, t in enumerate((k_out, v_out)):
        if t is not None:
            _same("kv4_write", torch.bfloat16, dev, t)
            _want(t.numel() == k.numel(), "kv4_write: k_out and v_out have the shape of k")
            out[i] = t.data_ptr()
    if workspace is not None:
        _same("kv4_write: workspace", workspace.dtype, dev, workspace)
        size = workspace.numel() * workspace.element_size()
    at = stats._at
    a = Kv4WriteArgs(batch, T, max_seqlen, h_kv, HEAD_DIM, flags, ks, vs, cu_seqlens.data_ptr(), k.data_ptr(), v.data_ptr(),
                     slot_mapping.data_ptr(), at["k_mean"], at["k_tscale"], at["v_tscale"], cache._c, *out)
    _call("mpfa_kv4_write", dev, stream, C.byref(a), _ptr(workspace), size)


def _kv4_attn(what, kind, q, cache, stats, cu, q_start, kv_len, page_table, out, plan, max_seqlen_q, window, sinks, stream):
    import torch
    dev, h_kv, batch, shape = cache.device, cache.h_kv, kv_len.numel(), q.shape
    h_q = shape[1] if len(shape) == 3 else 0
    stride = _rows(what, q, h_q, dev)
    _same(what, torch.int32, dev, kv_len, page_table)
    _same(what, torch.bfloat16, dev, out)
    if out.numel() != q.numel() or page_table.dim() != 2 or page_table.shape[0] != batch:
        raise ValueError(f"{what}: shapes")
    if stats.batch != batch or stats.h_kv != h_kv or stats.device != dev:
        raise ValueError(f"{what}: stats of another batch")
    ws, items, cut = None, None, (0,) * 8
    if plan is not None:
        if plan.what != (kind, batch, h_q, h_kv, window, sinks):
            raise ValueError(f"{what}: the plan was made for another call: {plan.what}")
        cut, ws, items = plan.cut(), plan.workspace, _ptr(plan.items)
        for t in (ws, plan.items):
            if t is not None and t.get_device() != dev:
                raise ValueError(f"{what}: the plan is of another device")
    a = Kv4AttnArgs(batch, h_q, h_kv, HEAD_DIM, page_table.shape[1], shape[0], max_seqlen_q, cut[0], window, sinks, *cut[1:],
                    stride, cu, q_start, items, kv_len.data_ptr(), page_table.data_ptr(), q.data_ptr(), cache._c,
                    stats._at["k_tscale"], stats._at["v_tscale"], out.data_ptr())
    on = _call("mpfa_kv4_" + kind, dev, stream, C.byref(a), _ptr(ws), 0 if ws is None else ws.numel())
    if plan is not None and on != plan.home:   # the plan's memory is not reused before this stream has passed the call
        for t in (ws, plan.items):
            if t is not None:
                t.record_stream(torch.cuda.ExternalStream(on, device=dev))


def kv4_prefill(q, cache: PagedCache4, stats: SeqStats4, cu_seqlens_q, q_start, kv_len, page_table, out, plan=None,
                window=0, sinks=0, max_seqlen_q=None, stream=None):
    """mpfa_kv4_prefill: causal attention of bf16 queries [T][Hq][128] (tokens may lie apart) over the
    4-bit cache; plan: kv4_prefill_plan of the same window and sinks (None: one pass), whose rows are computed
    and what q has more is padding.  max_seqlen_q: the most rows of one sequence (by default the plan's, or T
    without one)."""
    import torch
    if max_seqlen_q is None:
        max_seqlen_q = q.shape[0] if plan is None else plan.max_rows
    if plan is not None and q.shape[0] < plan.rows:
        raise ValueError(f"kv4_prefill: q has {q.shape[0]} rows, the plan was made for {plan.rows}")
    _same("kv4_prefill", torch.int32, cache.device, cu_seqlens_q, q_start)
    if cu_seqlens_q.numel() != kv_len.numel() + 1 or q_start.numel() != kv_len.numel():
        raise ValueError("kv4_prefill: shapes")
    _kv4_attn("kv4_prefill", "prefill", q, cache, stats, cu_seqlens_q.data_ptr(), q_start.data_ptr(), kv_len, page_table, out,
              plan, max_seqlen_q, window, sinks, stream)


def kv4_decode(q, cache: PagedCache4, stats: SeqStats4, kv_len, page_table, out, plan: Kv4Plan, window=0, sinks=0,
               stream=None):
    """mpfa_kv4_decode: the plan's q_tokens rows per sequence, the last ones of its kv_len keys; with a
    plan made for weights the attention weights are added to cache.weights."""
    if q.shape[0] != kv_len.numel() * plan.q_tokens:
        raise ValueError("kv4_decode: q has q_tokens rows per sequence")
    _kv4_attn("kv4_decode", "decode", q, cache, stats, None, None, kv_len, page_table, out, plan, 0, window, sinks, stream)


def kv4_evict(cache: PagedCache4, kv_len, page_table, dst_page_table, budget: int, kept, new_len, sinks=0, recent=0,
              in_place=False, stream=None):
    """mpfa_kv4_evict: cuts every sequence to the `budget` tokens of the largest cache.weights (per KV head;
    the first `sinks` and last `recent` always stay); kept int32 [B][Hkv][budget] and new_len [B] are written."""
    import torch
    dev, h_kv, batch, src, dst = cache.device, cache.h_kv, kv_len.numel(), page_table.shape, dst_page_table.shape
    _same("kv4_evict", torch.int32, dev, kv_len, page_table, dst_page_table, kept, new_len)
    if (len(src) != 2 or len(dst) != 2 or src[0] != batch or dst[0] != batch or kept.shape != (batch, h_kv, budget) or
            new_len.numel() != batch):
        raise ValueError("kv4_evict: shapes")
    a = Kv4EvictArgs(batch, h_kv, src[1], dst[1], budget, sinks, recent, KV4_IN_PLACE if in_place else 0, kv_len.data_ptr(),
                     page_table.data_ptr(), dst_page_table.data_ptr(), cache._c, kept.data_ptr(), new_len.data_ptr())
    _call("mpfa_kv4_evict", dev, stream, C.byref(a))


# ---- linear attention with a decay, the norm around attention ---------------------------

LINEAR_SCALE = HEAD_DIM ** -0.5
_INT32 = 1 << 31   # ctypes drops the bits of a larger number without a word


def _fits(what, *numbers):
    for n in numbers:
        if not -_INT32 <= n < _INT32:
            raise ValueError(f"{what}: {n} is not a 32-bit number")


def linear_prefill_workspace_size(batch: int, total_tokens: int, max_seqlen: int, h_q: int, h_kv: int) -> int:
    """Bytes that linear_prefill needs for these sizes and for every smaller batch, total_tokens and max_seqlen of the
    same heads."""
    n = C.c_size_t(0)
    _fits("linear_prefill_workspace_size", batch, total_tokens, max_seqlen, h_q, h_kv)
    _check(lib().mpfa_linear_prefill_workspace_size(batch, total_tokens, max_seqlen, h_q, h_kv, C.byref(n)),
           "mpfa_linear_prefill_workspace_size")
    return n.value


def _linear_args(what, q, k, v, log_decay, states, state_src, state_dst, out, batch, max_seqlen, q_tokens, cu, scale):
    import torch
    shape, slots, dev = q.shape, states.shape, states.get_device()
    if len(shape) != 3 or len(slots) != 4 or slots[2] != HEAD_DIM or slots[3] != HEAD_DIM:
        raise ValueError(f"{what}: q [T][Hq][{HEAD_DIM}] and states [slots][Hkv][{HEAD_DIM}][{HEAD_DIM}] are wanted")
    T, h_q, h_kv = shape[0], shape[1], slots[1]
    qs, ks, vs = _rows(what, q, h_q, dev), _rows(what, k, h_kv, dev), _rows(what, v, h_kv, dev)
    _same(what, torch.float32, dev, states)
    _same(what, torch.int32, dev, state_src, state_dst)
    _same(what, torch.bfloat16, dev, out)
    if k.shape[0] != T or v.shape[0] != T or out.numel() != q.numel() or state_src.numel() != batch or state_dst.numel() != batch:
        raise ValueError(f"{what}: shapes")
    gs, at = log_decay.shape, log_decay.stride()
    if (log_decay.dtype is not torch.float32 or log_decay.get_device() != dev or len(gs) not in (1, 2) or gs[-1] != h_kv or
            (h_kv > 1 and at[-1] != 1) or (len(gs) == 2 and gs[0] != T)):
        raise ValueError(f"{what}: log_decay is float32 [Hkv] or [T][Hkv]")
    decay_stride = 0 if len(gs) == 1 else at[0] if T > 1 else h_kv
    return dev, LinearArgs(batch, T, max_seqlen, q_tokens, h_q, h_kv, HEAD_DIM, 0, LINEAR_SCALE if scale is None else scale,
                           slots[0], qs, ks, vs, decay_stride, cu, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
                           state_src.data_ptr(), state_dst.data_ptr(), states.data_ptr(), out.data_ptr())


def linear_prefill(q, k, v, log_decay, cu_seqlens, states, state_src, state_dst, out, max_seqlen: int, workspace=None,
                   scale=None, stream=None):
    """mpfa_linear_prefill: linear attention with a decay over packed prompts.  q bf16 [T][Hq][128], k, v bf16
    [T][Hkv][128] (tokens may lie apart), log_decay f32 [Hkv] or [T][Hkv], states f32 [slots][Hkv][128][128] from
    whose slots state_src (negative: zeros) the sequences start and in whose slots state_dst (negative: nowhere) they
    end; workspace: linear_prefill_workspace_size bytes; scale: 1 / sqrt(128) by default."""
    import torch
    batch = cu_seqlens.numel() - 1
    if batch >= _INT32 or not -_INT32 <= max_seqlen < _INT32:
        _fits("linear_prefill", batch, max_seqlen)
    dev, a = _linear_args("linear_prefill", q, k, v, log_decay, states, state_src, state_dst, out, batch, max_seqlen, 0, cu_seqlens.data_ptr(), scale)
    _same("linear_prefill", torch.int32, dev, cu_seqlens)
    size = 0
    if workspace is not None:
        _same("linear_prefill: workspace", workspace.dtype, dev, workspace)
        size = workspace.numel() * workspace.element_size()
    _call("mpfa_linear_prefill", dev, stream, C.byref(a), _ptr(workspace), size)


def linear_decode(q, k, v, log_decay, states, state_src, state_dst, out, q_tokens: int = 1, scale=None, stream=None):
    """mpfa_linear_decode: q_tokens new tokens of each sequence (rows b * q_tokens + i) from the states in state_src,
    which lead to those in state_dst; tensors as for linear_prefill."""
    batch = state_src.numel()
    if q.shape[0] != batch * q_tokens:
        raise ValueError("linear_decode: q has q_tokens rows per sequence")
    dev, a = _linear_args("linear_decode", q, k, v, log_decay, states, state_src, state_dst, out, batch, 0, q_tokens, None, scale)
    _call("mpfa_linear_decode", dev, stream, C.byref(a))


def rms_norm(x, weight, out, eps: float = 1e-6, residual=None, residual_out=None, scales=None, group: int = 0, stream=None):
    """mpfa_rms_norm over the last dimension of x (bf16; contiguous, or rows of a matrix that lie apart): out bf16, or
    with scales (f32 [rows][groups]) float8_e4m3fn codes, a scale per `group` channels (0: per row).  residual:
    x + residual is normalised, and goes to residual_out (by default to residual).  weight: bf16 [width] or None.
    A bf16 out may be x, where that is contiguous."""
    import torch
    dev, shape = x.get_device(), x.shape
    if x.dtype is not torch.bfloat16 or not shape or shape[-1] == 0:
        raise ValueError("rms_norm: x is bf16 [..][width]")
    width = shape[-1]
    values = x.numel()
    rows = values // width
    if values >= _INT32 or group >> 31:
        _fits("rms_norm", rows, width, group)
    if x.is_contiguous():
        stride = width
    elif len(shape) == 2 and x.stride(1) == 1:
        stride = x.stride(0) if rows > 1 else width
    else:
        raise ValueError(f"rms_norm: x is contiguous or rows of a matrix, got strides {x.stride()}")
    if residual is None:
        _want(residual_out is None, "rms_norm: residual_out goes with a residual")
    else:
        residual_out = residual if residual_out is None else residual_out
        _same("rms_norm", torch.bfloat16, dev, residual, residual_out)
        _want(residual.numel() == residual_out.numel() == rows * width, "rms_norm: residual has the shape of x")
    if weight is not None:
        _same("rms_norm", torch.bfloat16, dev, weight)
        _want(weight.numel() == width, "rms_norm: weight is [width]")
    _same("rms_norm", torch.bfloat16 if scales is None else torch.float8_e4m3fn, dev, out)
    _want(out.numel() == rows * width, "rms_norm: out has the shape of x")
    if scales is not None:
        _same("rms_norm", torch.float32, dev, scales)
        _want(group >= 0 and scales.numel() == rows * -(-width // (group or width)), "rms_norm: scales are [rows][groups]")
    a = RmsNormArgs(rows, width, group, eps, stride, x.data_ptr(), _ptr(weight), _ptr(residual), _ptr(residual_out),
                    out.data_ptr(), _ptr(scales))
    _call("mpfa_rms_norm", dev, stream, C.byref(a))
