"""ctypes binding of libkeep_hip.so: argument marshalling only.

Every step of the path runs inside the library's HIP kernels; this module turns
torch tensors (device memory, streams) and Python lists into the plain pointers
and sizes of include/keep.h and raises KeepError on a non-zero status.  There is
no CPU fallback: loading fails loudly when the library has not been built.
"""
import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkeep_hip.so")

KEEP_OK = 0
KEEP_ERR_INVALID_ARG, KEEP_ERR_SHAPE, KEEP_ERR_STATE, KEEP_ERR_WORKSPACE, KEEP_ERR_HIP, KEEP_ERR_UNSUPPORTED = range(1, 7)
KEEP_F32, KEEP_BF16 = 0, 1
KEEP_KV_DEVICE, KEEP_KV_PINNED_HOST = 0, 1
KEEP_BUDGET_GROUP_COUNT, KEEP_BUDGET_TOKENS = 0, 1
KEEP_LOAD_SERIAL, KEEP_LOAD_NEXT_LAYER, KEEP_LOAD_LAYER_BALANCED = 0, 1, 2
KEEP_KERNELS_AUTO, KEEP_KERNELS_GENERIC = 0, 1
KEEP_REPORT_MAX_LAYERS = 128
KEEP_ROPE_HALF, KEEP_ROPE_INTERLEAVED = 0, 1
KEEP_ROPE_PLAIN, KEEP_ROPE_LINEAR, KEEP_ROPE_BASE, KEEP_ROPE_PARTS = 0, 1, 2, 3
KEEP_CACHE_F32, KEEP_CACHE_BF16, KEEP_CACHE_FP8, KEEP_CACHE_INT8 = 0, 1, 2, 3
KEEP_PAGED_MAX_SEQS = 4096
KEEP_SAMPLE_MAX_VOCAB = 1 << 20

KEEP_OPT_PROPAGATION_SOURCES = 0
KEEP_SOURCES_QUERY_AND_SET, KEEP_SOURCES_SET_ONLY = 0, 1
KEEP_STATE_ATTN_OUT, KEEP_STATE_LSE = 0, 1

EXPORTED = ("keep_init", "keep_destroy", "keep_last_error", "keep_uses_mfma", "keep_workspace_bytes", "keep_recompute_layer",
            "keep_set_option", "keep_read_layer_state", "keep_select_groups_static", "keep_prefill_tokens",
            "keep_select_tokens",
            "keep_score_groups", "keep_select_groups", "keep_prefill",
            "keep_prefill_padded", "keep_decode", "keep_precompute_group", "keep_precompute_groups",
            "keep_dequantize_int4", "keep_attach_int4",
            "keep_rope_frequencies", "keep_rope_rows", "keep_cache_write", "keep_cache_read",
            "keep_paged_attention_workspace_bytes", "keep_paged_attention", "keep_sample_workspace_bytes", "keep_sample",
            "keep_decode_sampled",
            "keep_memory_create", "keep_memory_destroy", "keep_memory_last_error",
            "keep_memory_put", "keep_memory_remove", "keep_memory_end_step", "keep_memory_unit_count",
            "keep_memory_unit_info", "keep_memory_unit_tokens", "keep_memory_mark_computed")


class KeepError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__("keep status %d: %s" % (status, text))
        self.status = status


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn_dim", "vocab")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float)] + \
               [(n, C.c_int32) for n in ("dtype", "max_tokens", "max_groups", "kernel_path")]


_W_NAMES = ("ln1", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "ln2", "wgate", "wup", "wdown")


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _W_NAMES]


_W4_NAMES = ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown")


class Int4Matrix(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scale_zero", C.c_void_p)]


class LayerWeightsInt4(C.Structure):
    _fields_ = [(n, Int4Matrix) for n in _W4_NAMES]


class Prompt(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("group_len", C.POINTER(C.c_int32)), ("group_kind", C.POINTER(C.c_uint8)),
                ("instr_len", C.c_int32), ("token_ids", C.POINTER(C.c_int32)),
                ("k_blocks", C.POINTER(C.c_void_p)), ("v_blocks", C.POINTER(C.c_void_p)), ("kv_location", C.c_int32)]


_L = KEEP_REPORT_MAX_LAYERS
_REPORT_MS = ("ms_realign", "ms_prep", "ms_qkv_gemm", "ms_rope", "ms_attn", "ms_oproj", "ms_norm2", "ms_gateup",
              "ms_down", "ms_score")


class Report(C.Structure):
    _fields_ = ([("events_in", C.c_int32), ("n_layers", C.c_int32), ("used_mfma", C.c_int32), ("ms_total", C.c_float),
                 ("rows", C.c_int32 * _L), ("set_size", C.c_int32 * _L), ("hops_run", C.c_int32 * _L),
                 ("realign_rows", C.c_int32 * _L), ("ffn_rows", C.c_int32 * _L),
                 ("attn_rows", C.c_int32 * _L), ("attn_keys", C.c_uint64 * _L)]
                + [(_n, C.c_float * _L) for _n in _REPORT_MS]
                + [("bytes_loaded", C.c_uint64 * _L)])


class RopeDesc(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32), ("theta", C.c_double), ("factor", C.c_double),
                ("trained_len", C.c_int32), ("fast", C.c_double), ("slow", C.c_double)]


class RopeRowsDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_rows", "n_q_heads", "n_kv_heads", "head_dim", "rot_dim", "layout")] + \
               [("magnitude", C.c_float)] + \
               [(n, C.c_int64) for n in ("q_in_stride", "q_out_stride", "k_in_stride", "k_out_stride")]


class PagedCacheDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("format", "n_pages", "page_size", "n_kv_heads", "head_dim")] + \
               [(n, C.c_int64) for n in ("page_stride", "head_stride", "token_stride")] + \
               [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class PagedAttentionDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_seqs", "n_rows", "n_q_heads", "max_pages", "window")] + \
               [("scale", C.c_float), ("q_stride", C.c_int64), ("out_stride", C.c_int64)]


class SampleDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_rows", "vocab")] + [("row_stride", C.c_int64)]


class Sampling(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float),
                ("uniform", C.POINTER(C.c_float))]


_lib = None


class MemoryUnit(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "id", "group", "n_segments", "n_tokens", "dirty")]


class MemoryStepReport(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("step", "n_static", "n_dynamic", "n_to_dynamic", "n_to_static",
                                         "dirty_units")] + [("dirty_tokens", C.c_int64)]


def load_library() -> C.CDLL:
    """dlopen the HIP library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libkeep_hip.so is missing: build it with `python -m paper_2602_23592_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
    pi32 = C.POINTER(C.c_int32)
    lib.keep_init.restype = i32
    lib.keep_init.argtypes = [C.POINTER(ModelDesc), C.POINTER(LayerWeights), vp, vp, vp, vp, C.POINTER(vp)]
    lib.keep_destroy.restype = i32
    lib.keep_destroy.argtypes = [vp]
    lib.keep_last_error.restype = C.c_char_p
    lib.keep_last_error.argtypes = [vp]
    lib.keep_uses_mfma.restype = i32
    lib.keep_uses_mfma.argtypes = [vp]
    lib.keep_workspace_bytes.restype = C.c_uint64
    lib.keep_workspace_bytes.argtypes = [C.POINTER(ModelDesc)]
    lib.keep_set_option.restype = i32
    lib.keep_set_option.argtypes = [vp, i32, i32]
    lib.keep_read_layer_state.restype = i32
    lib.keep_read_layer_state.argtypes = [vp, i32, vp, C.c_uint64]
    lib.keep_recompute_layer.restype = i32
    lib.keep_recompute_layer.argtypes = [vp, C.POINTER(Prompt), i32, pi32, i32, vp, vp, vp, vp]
    lib.keep_score_groups.restype = i32
    lib.keep_score_groups.argtypes = [vp, C.POINTER(Prompt), i32, pi32, i32, f32, i32, i32, C.POINTER(f32), pi32, pi32, pi32]
    lib.keep_select_groups.restype = i32
    lib.keep_select_groups.argtypes = [vp, C.POINTER(f32), pi32, i32, pi32, i32, f32, i32, i32, pi32, pi32, pi32]
    lib.keep_select_groups_static.restype = i32
    lib.keep_select_groups_static.argtypes = [vp, vp, i32, vp, i32, i32, f32, i32, i32, i32, vp, vp]
    lib.keep_prefill_tokens.restype = i32
    lib.keep_prefill_tokens.argtypes = [vp, C.POINTER(Prompt), C.POINTER(f32), i32, vp, vp, vp, pi32, pi32,
                                        C.POINTER(f32), C.POINTER(Report)]
    lib.keep_select_tokens.restype = i32
    lib.keep_select_tokens.argtypes = [vp, C.POINTER(f32), i32, i32, pi32]
    lib.keep_prefill.restype = i32
    lib.keep_prefill.argtypes = [vp, C.POINTER(Prompt), C.POINTER(f32), i32, i32, i32, vp, vp, vp, pi32, pi32,
                                 C.POINTER(Report)]
    lib.keep_prefill_padded.restype = i32
    lib.keep_prefill_padded.argtypes = [vp, C.POINTER(Prompt), C.POINTER(f32), i32, i32, i32, vp, vp, i32, vp, pi32, pi32,
                                        C.POINTER(Report)]
    lib.keep_decode.restype = i32
    lib.keep_decode.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, pi32, vp, pi32]
    lib.keep_dequantize_int4.restype = i32
    lib.keep_dequantize_int4.argtypes = [vp, vp, i32, i32, vp, vp]
    lib.keep_attach_int4.restype = i32
    lib.keep_attach_int4.argtypes = [vp, C.POINTER(LayerWeightsInt4)]
    lib.keep_rope_frequencies.restype = i32
    lib.keep_rope_frequencies.argtypes = [C.POINTER(RopeDesc), C.POINTER(C.c_double), C.POINTER(f32)]
    lib.keep_rope_rows.restype = i32
    lib.keep_rope_rows.argtypes = [C.POINTER(RopeRowsDesc), vp, vp, vp, vp, vp, vp, vp]
    for name in ("keep_cache_write", "keep_cache_read"):
        getattr(lib, name).restype = i32
        getattr(lib, name).argtypes = [C.POINTER(PagedCacheDesc), i32, vp, vp, i32, C.c_int64, vp, vp]
    lib.keep_paged_attention_workspace_bytes.restype = C.c_uint64
    lib.keep_paged_attention_workspace_bytes.argtypes = [C.POINTER(PagedCacheDesc), i32, i32]
    lib.keep_paged_attention.restype = i32
    lib.keep_paged_attention.argtypes = [C.POINTER(PagedAttentionDesc), C.POINTER(PagedCacheDesc), vp, vp, vp, vp, vp, vp, vp,
                                         C.c_uint64, vp]
    lib.keep_sample_workspace_bytes.restype = C.c_uint64
    lib.keep_sample_workspace_bytes.argtypes = [i32, i32]
    lib.keep_sample.restype = i32
    lib.keep_sample.argtypes = [C.POINTER(SampleDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_uint64, vp]
    lib.keep_decode_sampled.restype = i32
    lib.keep_decode_sampled.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, C.POINTER(Sampling), pi32, C.POINTER(f32), vp,
                                        pi32]
    lib.keep_precompute_group.restype = i32
    lib.keep_precompute_group.argtypes = [vp, pi32, i32, vp, vp, C.POINTER(Report)]
    lib.keep_precompute_groups.restype = i32
    lib.keep_precompute_groups.argtypes = [vp, i32, pi32, pi32, vp, vp, C.POINTER(Report)]
    lib.keep_memory_create.restype = i32
    lib.keep_memory_create.argtypes = [i32, C.POINTER(vp)]
    lib.keep_memory_destroy.restype = i32
    lib.keep_memory_destroy.argtypes = [vp]
    lib.keep_memory_last_error.restype = C.c_char_p
    lib.keep_memory_last_error.argtypes = [vp]
    lib.keep_memory_put.restype = i32
    lib.keep_memory_put.argtypes = [vp, i32, i32, pi32, i32, pi32]
    lib.keep_memory_remove.restype = i32
    lib.keep_memory_remove.argtypes = [vp, i32]
    lib.keep_memory_end_step.restype = i32
    lib.keep_memory_end_step.argtypes = [vp, C.POINTER(MemoryStepReport), pi32, i32, pi32, i32]
    lib.keep_memory_unit_count.restype = i32
    lib.keep_memory_unit_count.argtypes = [vp]
    lib.keep_memory_unit_info.restype = i32
    lib.keep_memory_unit_info.argtypes = [vp, i32, C.POINTER(MemoryUnit)]
    lib.keep_memory_unit_tokens.restype = i32
    lib.keep_memory_unit_tokens.argtypes = [vp, i32, pi32, i32, pi32]
    lib.keep_memory_mark_computed.restype = i32
    lib.keep_memory_mark_computed.argtypes = [vp, i32]
    _lib = lib
    return lib


def _i32_array(values: Sequence[int]):
    a = np.ascontiguousarray(np.asarray(values, dtype=np.int32))
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_handle(s) -> Optional[int]:
    if s is None:
        return None
    return s.cuda_stream if hasattr(s, "cuda_stream") else int(s)


def _forced_tokens(tokens: Optional[Sequence[int]], n_new: int):
    """(array that owns the memory, its address) of the tokens to feed: the library reads n_new - 1 of them"""
    if tokens is None:
        return None, None
    if len(tokens) < n_new - 1:
        raise KeepError(KEEP_ERR_INVALID_ARG, "forced_tokens has %d entries, %d new tokens need %d" % (len(tokens), n_new, n_new - 1))
    return _i32_array(list(tokens) if len(tokens) else [0])


class KeepPrompt:
    """Keeps the host arrays of a keep_prompt alive and exposes the C struct."""

    def __init__(self, group_len: Sequence[int], instr_len: int, token_ids: Sequence[int], k_blocks, v_blocks,
                 n_layers: int, kv_location: int = KEEP_KV_DEVICE, group_kind: Optional[Sequence[int]] = None):
        self.group_len = [int(v) for v in group_len]
        self.instr_len = int(instr_len)
        self.n_groups = len(self.group_len)
        self._gl, gl_p = _i32_array(self.group_len if self.n_groups else [0])
        self._tok, tok_p = _i32_array(token_ids)
        self._kind = None
        kind_p = None
        if group_kind is not None:
            self._kind = np.ascontiguousarray(np.asarray(group_kind, dtype=np.uint8))
            kind_p = self._kind.ctypes.data_as(C.POINTER(C.c_uint8))
        # k_blocks[l][g]: tensors (device or pinned host); flattened to layer*G + g
        self._blocks = (k_blocks, v_blocks)     # keep the tensors alive
        n = max(1, n_layers * self.n_groups)
        self._kp = (C.c_void_p * n)()
        self._vp = (C.c_void_p * n)()
        if k_blocks is not None:
            for l in range(n_layers):
                for g in range(self.n_groups):
                    self._kp[l * self.n_groups + g] = k_blocks[l][g].data_ptr()
                    self._vp[l * self.n_groups + g] = v_blocks[l][g].data_ptr()
        self.c = Prompt(self.n_groups, gl_p, kind_p, self.instr_len, tok_p,
                        C.cast(self._kp, C.POINTER(C.c_void_p)), C.cast(self._vp, C.POINTER(C.c_void_p)), kv_location)

    @property
    def n_mem(self) -> int:
        return sum(self.group_len)

    @property
    def n_tokens(self) -> int:
        return self.n_mem + self.instr_len

    def n_rows(self, groups: Sequence[int]) -> int:
        return sum(self.group_len[g] for g in groups) + self.instr_len


def dequantize_int4(codes: torch.Tensor, scale_zero: torch.Tensor, rows: int, k: int, stream=None) -> torch.Tensor:
    """keep_dequantize_int4: codes (uint8, rows * K / 2) and scale_zero (32-bit words, rows * K / 128) in the
    library's block order, on the device -> the bfloat16 weights [rows, K] (new device tensor; the allocation is
    the only thing done here)."""
    lib = load_library()
    assert codes.is_cuda and codes.is_contiguous() and codes.dtype == torch.uint8 and codes.numel() == rows * k // 2
    assert scale_zero.is_cuda and scale_zero.is_contiguous() and scale_zero.element_size() == 4
    assert scale_zero.numel() == rows * k // 128
    out = torch.empty((rows, k), dtype=torch.bfloat16, device=codes.device)
    st = lib.keep_dequantize_int4(codes.data_ptr(), scale_zero.data_ptr(), rows, k, out.data_ptr(),
                                  _stream_handle(stream if stream is not None else torch.cuda.current_stream()))
    if st != KEEP_OK:
        raise KeepError(st, lib.keep_last_error(None).decode())
    return out


def select_groups_static(S: torch.Tensor, groups: torch.Tensor, group_len: torch.Tensor, mem_tokens: int,
                         ratio_next: float, hops: int, budget_mode: int, propagation_sources: int,
                         result: torch.Tensor, stream=None):
    """keep_select_groups_static: every tensor is caller-allocated device memory (S float32 [(m+1), m], groups
    int32 [m], group_len int32 [G], result int32 [m + 2]); nothing is allocated here or in the library."""
    lib = load_library()
    m = int(groups.numel())
    for t, dt in ((S, torch.float32), (groups, torch.int32), (group_len, torch.int32), (result, torch.int32)):
        assert t.is_cuda and t.is_contiguous() and t.dtype == dt
    assert S.numel() == (m + 1) * m and result.numel() >= m + 2
    st = lib.keep_select_groups_static(S.data_ptr(), groups.data_ptr(), m, group_len.data_ptr(), int(group_len.numel()),
                                       int(mem_tokens), float(ratio_next), hops, budget_mode, propagation_sources,
                                       result.data_ptr(),
                                       _stream_handle(stream if stream is not None else torch.cuda.current_stream()))
    if st != KEEP_OK:
        raise KeepError(st, lib.keep_last_error(None).decode())


# ---- the operators of include/keep_serve.h ------------------------------------------------------------------
# `stream` of these calls: a torch stream or a hipStream_t, by default the current stream of the tensors' device.  That the
# tensors' contents are there when the stream reaches the call is the caller's; their memory may be dropped behind the call.
_DTYPES = {torch.float32: KEEP_F32, torch.bfloat16: KEEP_BF16}
_FORMATS = {torch.float32: KEEP_CACHE_F32, torch.bfloat16: KEEP_CACHE_BF16, torch.float8_e4m3fn: KEEP_CACHE_FP8,
            torch.int8: KEEP_CACHE_INT8}


def _refuse(text: str):
    raise KeepError(KEEP_ERR_INVALID_ARG, text)


def _on_gpu(device: torch.device):
    if device.type != "cuda":
        _refuse("tensors must be on the GPU, these are on %s" % device)


def _launch(device: torch.device, stream, call, *args):
    """One call on `stream`, by default the current one of the tensors' device, with that device current."""
    if stream is None:
        stream = torch.cuda.current_stream(device)
    if torch.cuda.current_device() == device.index:
        st = call(*args, _stream_handle(stream))
    else:
        with torch.cuda.device(device):
            st = call(*args, _stream_handle(stream))
    if st != KEEP_OK:
        raise KeepError(st, _lib.keep_last_error(None).decode())


def _stream_object(stream, device: torch.device) -> torch.cuda.Stream:
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = _stream_handle(stream)
    return torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)


def _empty(shape, dtype: torch.dtype, device: torch.device, stream) -> torch.Tensor:
    """New memory that belongs to the stream of the call: its next use there waits for the call, wherever the tensor is dropped"""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_stream_object(stream, device)):
        return torch.empty(shape, dtype=dtype, device=device)


def _hold(device: torch.device, stream, *tensors: Optional[torch.Tensor]):
    """Memory of a call's tensors is not handed out again before the call is done, also where they are dropped behind it and
    belong to another stream than its own"""
    if stream is None or (_stream_handle(stream) or 0) == torch.cuda.current_stream(device).cuda_stream:
        return
    on = _stream_object(stream, device)
    for t in tensors:
        if t is not None and t.is_cuda:
            t.record_stream(on)


def _array(name: str, t: Optional[torch.Tensor], dtype, numel: int, device: torch.device, optional: bool = False):
    """Address of a dense device array of `numel` elements"""
    if t is None:
        return None if optional else _refuse(name + " is missing")
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.device != device:
        _refuse("%s must be a dense %s array of %d elements on %s" % (name, dtype, numel, device))
    return t.data_ptr()


def _heads(name: str, t: torch.Tensor, device: torch.device, dtype=None) -> int:
    """Row stride of [rows, heads, head_dim] whose rows are dense"""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or t.device != device or not (t.dtype is dtype if dtype is not None else t.dtype in _DTYPES):
        _refuse("%s must be [rows, heads, head_dim] in float32 or bfloat16, of one type and on one device" % name)
    rows, h, d = shape
    if not ((d <= 1 or stride[2] == 1) and (h <= 1 or stride[1] == d)) and rows * h * d:
        _refuse("the heads of a row of %s must be adjacent" % name)
    return stride[0] if rows > 1 else h * d


def rope_frequencies(rot_dim: int, theta: float = 1.0e6, scaling: int = KEEP_ROPE_PLAIN, factor: float = 1.0,
                     trained_len: int = 1, fast: float = 32.0, slow: float = 1.0):
    """keep_rope_frequencies: (float64 numpy array [rot_dim / 2], factor on the rotated values)"""
    lib = load_library()
    freq = np.zeros(max(1, rot_dim // 2), dtype=np.float64)
    mag = C.c_float(0.0)
    desc = RopeDesc(rot_dim, scaling, theta, factor, trained_len, fast, slow)
    st = lib.keep_rope_frequencies(C.byref(desc), freq.ctypes.data_as(C.POINTER(C.c_double)), C.byref(mag))
    if st != KEEP_OK:
        raise KeepError(st, lib.keep_last_error(None).decode())
    return freq, mag.value


def rope_rows(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor, freq: torch.Tensor,
              layout: int = KEEP_ROPE_HALF, magnitude: float = 1.0, q_out: Optional[torch.Tensor] = None,
              k_out: Optional[torch.Tensor] = None, stream=None):
    """keep_rope_rows: q, k [rows, heads, head_dim] (either may be None) -> q_out, k_out, by default q and k themselves.
    rot_dim is twice the length of freq (float64, on the device)."""
    lib = load_library()
    ref = q if q is not None else k
    if ref is None:
        _refuse("neither queries nor keys")
    device, dtype = ref.device, ref.dtype
    _on_gpu(device)
    if dtype not in _DTYPES or ref.dim() != 3 or (q is None and q_out is not None) or (k is None and k_out is not None):
        _refuse("queries and keys must be [rows, heads, head_dim] in float32 or bfloat16, outputs go with inputs")
    n, _, d = ref.shape
    hq = hkv = qi = qo = ki = ko = 0
    if q is not None:
        q_out = q if q_out is None else q_out
        hq, qi, qo = q.shape[1], _heads("q", q, device, dtype), _heads("q_out", q_out, device, dtype)
        if q_out.shape != q.shape:
            _refuse("the shape of q_out differs from that of q")
    if k is not None:
        k_out = k if k_out is None else k_out
        ki, ko = _heads("k", k, device, dtype), _heads("k_out", k_out, device, dtype)
        rows, hkv, dk = k.shape
        if k_out.shape != k.shape or rows != n or dk != d:
            _refuse("rows or head_dim of keys differ from the queries', or k_out from k")
    pairs = freq.numel()
    _hold(device, stream, q, k, q_out, k_out, positions, freq)
    desc = RopeRowsDesc(_DTYPES[dtype], n, hq, hkv, d, 2 * pairs, layout, magnitude, qi, qo, ki, ko)
    _launch(device, stream, lib.keep_rope_rows, C.byref(desc), _ptr(q), _ptr(q_out), _ptr(k), _ptr(k_out),
            _array("positions", positions, torch.int32, n, device), _array("freq", freq, torch.float64, pairs, device))
    return q_out, k_out


class PagedCache:
    """keep_paged_cache over tensors k, v [n_pages, n_kv_heads, page_size, head_dim] (float32, bfloat16, float8_e4m3fn or
    int8; strides of 16-byte multiples, pages outermost, adjacent values) and, for the 8-bit types, float32 k_scale, v_scale
    [n_pages, n_kv_heads, page_size].  Keeps the tensors alive."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        self.lib = load_library()
        if k.dim() != 4 or k.dtype not in _FORMATS or v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride() \
                or v.device != k.device or not k.is_cuda:
            _refuse("k and v must be alike, [n_pages, n_kv_heads, page_size, head_dim], of a cache type, on the GPU")
        if k.stride(3) != 1:
            _refuse("a head's values must be adjacent")
        n = k.shape[0] * k.shape[1] * k.shape[2]
        scaled = k.element_size() == 1
        if not scaled and (k_scale is not None or v_scale is not None):
            _refuse("only 8-bit caches have scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = k.device
        self.c = PagedCacheDesc(_FORMATS[k.dtype], k.shape[0], k.shape[2], k.shape[1], k.shape[3], k.stride(0), k.stride(1),
                                k.stride(2), k.data_ptr(), v.data_ptr(),
                                _array("k_scale", k_scale, torch.float32, n, k.device, not scaled),
                                _array("v_scale", v_scale, torch.float32, n, k.device, not scaled))

    @classmethod
    def empty(cls, dtype: torch.dtype, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, device="cuda"):
        """A cache of new, uninitialised dense pages"""
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        ks, vs = (torch.empty(shape[:3], dtype=torch.float32, device=device) if k.element_size() == 1 else None
                  for _ in range(2))
        return cls(k, v, ks, vs)

    def _rows(self, call, k, v, slots, stream):
        stride = _heads("k", k, self.device)
        n, h, d = k.shape
        if _heads("v", v, self.device, k.dtype) != stride or v.shape != k.shape or h != self.c.n_kv_heads or d != self.c.head_dim:
            _refuse("k and v must be alike, [rows, n_kv_heads, head_dim]")
        _hold(self.device, stream, k, v, slots, self.k, self.v, self.k_scale, self.v_scale)
        _launch(self.device, stream, call, C.byref(self.c), _DTYPES[k.dtype], k.data_ptr(), v.data_ptr(), n, stride,
                _array("slots", slots, torch.int32, n, self.device))

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None):
        """keep_cache_write: rows k, v [n, n_kv_heads, head_dim] into the slots (int32 [n])"""
        self._rows(self.lib.keep_cache_write, k, v, slots, stream)

    def read(self, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None):
        """keep_cache_read: the slots' rows into k, v [n, n_kv_heads, head_dim]"""
        self._rows(self.lib.keep_cache_read, k, v, slots, stream)


def paged_attention_workspace_bytes(n_q_heads: int, cache: PagedCache, n_seqs: int) -> int:
    return int(cache.lib.keep_paged_attention_workspace_bytes(C.byref(cache.c), n_q_heads, n_seqs))


def paged_attention(q: torch.Tensor, cache: PagedCache, q_start: torch.Tensor, kv_len: torch.Tensor,
                    page_table: torch.Tensor, window: int = 0, scale: float = 0.0, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """keep_paged_attention: q [rows, n_q_heads, head_dim] of len(kv_len) sequences, rows q_start[s] .. q_start[s + 1] each,
    page_table int32 [n_seqs, max_pages].  out and workspace (uint8) are allocated where they are not given, for `stream`."""
    stride = _heads("q", q, cache.device)
    n, hq, d = q.shape
    if d != cache.c.head_dim:
        _refuse("head_dim of q differs from the cache's")
    seqs = kv_len.numel()
    if page_table.dim() != 2 or page_table.shape[0] != seqs:
        _refuse("page_table must be [n_seqs, max_pages]")
    if out is None:
        out = _empty((n, hq, d), q.dtype, q.device, stream)
    if out.shape != q.shape:
        _refuse("out must have the shape of q")
    need = paged_attention_workspace_bytes(hq, cache, seqs)
    if workspace is None:
        workspace = _empty(max(1, need), torch.uint8, q.device, stream)
    desc = PagedAttentionDesc(_DTYPES[q.dtype], seqs, n, hq, page_table.shape[1], window, scale, stride,
                              _heads("out", out, q.device, q.dtype))
    dev = cache.device
    _hold(dev, stream, q, q_start, kv_len, page_table, out, lse, workspace, cache.k, cache.v, cache.k_scale, cache.v_scale)
    _launch(dev, stream, cache.lib.keep_paged_attention, C.byref(desc), C.byref(cache.c), q.data_ptr(),
            _array("q_start", q_start, torch.int32, seqs + 1, dev), _array("kv_len", kv_len, torch.int32, seqs, dev),
            _array("page_table", page_table, torch.int32, page_table.numel(), dev), out.data_ptr(),
            _array("lse", lse, torch.float32, n * hq, dev, True),
            _array("workspace", workspace, torch.uint8, workspace.numel(), dev), workspace.numel())
    return out


def sample_workspace_bytes(n_rows: int, vocab: int) -> int:
    return int(load_library().keep_sample_workspace_bytes(n_rows, vocab))


def sample(logits: torch.Tensor, uniform: torch.Tensor, temperature: Optional[torch.Tensor] = None,
           top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
           tokens: Optional[torch.Tensor] = None, probs: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """keep_sample: one token per row of logits [rows, vocab], from uniform [rows]; the parameters are arrays [rows]."""
    lib = load_library()
    if logits.dim() != 2 or logits.dtype not in _DTYPES or (logits.numel() and logits.shape[1] > 1 and logits.stride(1) != 1):
        _refuse("logits must be [rows, vocab] in float32 or bfloat16 with adjacent values")
    n, vocab = logits.shape
    dev = logits.device
    _on_gpu(dev)
    if tokens is None:
        tokens = _empty(n, torch.int32, dev, stream)
    if workspace is None:
        workspace = _empty(max(1, sample_workspace_bytes(n, vocab)), torch.uint8, dev, stream)
    _hold(dev, stream, logits, uniform, temperature, top_k, top_p, min_p, tokens, probs, workspace)
    desc = SampleDesc(_DTYPES[logits.dtype], n, vocab, logits.stride(0) if n > 1 else vocab)
    _launch(dev, stream, lib.keep_sample, C.byref(desc), logits.data_ptr(), _array("uniform", uniform, torch.float32, n, dev),
            _array("temperature", temperature, torch.float32, n, dev, True), _array("top_k", top_k, torch.int32, n, dev, True),
            _array("top_p", top_p, torch.float32, n, dev, True), _array("min_p", min_p, torch.float32, n, dev, True),
            _array("tokens", tokens, torch.int32, n, dev), _array("probs", probs, torch.float32, n, dev, True),
            _array("workspace", workspace, torch.uint8, workspace.numel(), dev), workspace.numel())
    return tokens


class KeepContext:
    """keep_ctx handle.  Weights: list of dicts name -> device tensor (or None for absent biases)."""

    def __init__(self, shape, layers: List[dict], embed: torch.Tensor, max_tokens: int, max_groups: int,
                 kernel_path: int = KEEP_KERNELS_AUTO, stream_compute=None, stream_eval=None, stream_copy=None):
        self.lib = load_library()
        self.shape = shape
        self.dtype = KEEP_BF16 if shape.storage == "bf16" else KEEP_F32
        self.torch_dtype = torch.bfloat16 if shape.storage == "bf16" else torch.float32
        self.desc = ModelDesc(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                              shape.ffn_dim, shape.vocab, shape.rope_theta, shape.rms_eps, self.dtype,
                              int(max_tokens), int(max_groups), kernel_path)
        self._keep = (layers, embed, stream_compute, stream_eval, stream_copy)
        arr = (LayerWeights * shape.n_layers)()
        for l, w in enumerate(layers):
            for n in _W_NAMES:
                t = w.get(n)
                if t is not None:
                    assert t.is_cuda and t.is_contiguous() and t.dtype == self.torch_dtype, n
                setattr(arr[l], n, _ptr(t))
        assert embed.is_cuda and embed.is_contiguous() and embed.dtype == self.torch_dtype
        self.device = embed.device
        handle = C.c_void_p()
        st = self.lib.keep_init(C.byref(self.desc), arr, embed.data_ptr(), _stream_handle(stream_compute),
                                _stream_handle(stream_eval), _stream_handle(stream_copy), C.byref(handle))
        if st != KEEP_OK:
            raise KeepError(st, self.lib.keep_last_error(None).decode())
        self.handle = handle

    def close(self):
        if getattr(self, "handle", None):
            self.lib.keep_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def attach_int4(self, layers4: Optional[List[dict]]):
        """keep_attach_int4.  layers4: per layer a dict name -> (codes, scale_zero) device tensors for the seven
        projections, or None to detach.  The tensors are kept alive by this object."""
        if layers4 is None:
            self._check(self.lib.keep_attach_int4(self.handle, None))
            self._keep4 = None
            return
        arr = (LayerWeightsInt4 * self.shape.n_layers)()
        for l, w in enumerate(layers4):
            for n in _W4_NAMES:
                codes, sz = w[n][0], w[n][1]
                assert codes.is_cuda and codes.is_contiguous() and sz.is_cuda and sz.is_contiguous(), n
                getattr(arr[l], n).codes = codes.data_ptr()
                getattr(arr[l], n).scale_zero = sz.data_ptr()
        self._check(self.lib.keep_attach_int4(self.handle, arr))
        self._keep4 = layers4

    @property
    def uses_mfma(self) -> bool:
        return self.lib.keep_uses_mfma(self.handle) == 1

    def _check(self, st: int):
        if st != KEEP_OK:
            raise KeepError(st, self.lib.keep_last_error(self.handle).decode())

    # -- the C entry points ---------------------------------------------------
    def set_option(self, option: int, value: int):
        self._check(self.lib.keep_set_option(self.handle, option, value))

    def read_layer_state(self, what: int, n_rows: int) -> np.ndarray:
        """keep_read_layer_state: attention output [n_rows, Hq, dh] (float32 view of the stored values) or
        log-sum-exp [n_rows, Hq] of the last keep_recompute_layer, on the host."""
        s = self.shape
        if what == KEEP_STATE_LSE:
            out = np.empty((n_rows, s.n_q_heads), dtype=np.float32)
        elif self.dtype == KEEP_BF16:
            out = np.empty((n_rows, s.n_q_heads, s.head_dim), dtype=np.uint16)
        else:
            out = np.empty((n_rows, s.n_q_heads, s.head_dim), dtype=np.float32)
        self._check(self.lib.keep_read_layer_state(self.handle, what, out.ctypes.data_as(C.c_void_p), out.nbytes))
        if out.dtype == np.uint16:      # bfloat16 bit patterns -> the float32 values they stand for
            out = (out.astype(np.uint32) << np.uint32(16)).view(np.float32)
        return out

    def recompute_layer(self, prompt: KeepPrompt, layer: int, groups: Sequence[int], x_in: Optional[torch.Tensor],
                        x_out: torch.Tensor, k_cache_l: torch.Tensor, v_cache_l: torch.Tensor):
        g, gp = _i32_array(groups if len(groups) else [0])
        self._check(self.lib.keep_recompute_layer(self.handle, C.byref(prompt.c), layer, gp, len(groups), _ptr(x_in),
                                                  x_out.data_ptr(), k_cache_l.data_ptr(), v_cache_l.data_ptr()))

    def score_groups(self, prompt: KeepPrompt, layer: int, groups: Sequence[int], ratio_next: float, hops: int,
                     budget_mode: int = KEEP_BUDGET_GROUP_COUNT, want_scores: bool = True):
        m = len(groups)
        g, gp = _i32_array(groups if m else [0])
        S = np.zeros((m + 1, max(m, 1)), dtype=np.float32) if want_scores else None
        nxt = np.zeros(max(m, 1), dtype=np.int32)
        n_next, runs = C.c_int32(0), C.c_int32(0)
        self._check(self.lib.keep_score_groups(
            self.handle, C.byref(prompt.c), layer, gp, m, float(ratio_next), hops, budget_mode,
            S.ctypes.data_as(C.POINTER(C.c_float)) if want_scores else None,
            nxt.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(n_next), C.byref(runs)))
        scores = S[:, :m].reshape(m + 1, m) if want_scores else None
        return [int(v) for v in nxt[:n_next.value]], runs.value, scores

    def select_groups(self, S: np.ndarray, groups: Sequence[int], group_len: Sequence[int], ratio_next: float,
                      hops: int, budget_mode: int = KEEP_BUDGET_GROUP_COUNT):
        m = len(groups)
        S = np.ascontiguousarray(S, dtype=np.float32)
        assert S.shape == (m + 1, m)
        g, gp = _i32_array(groups if m else [0])
        gl, glp = _i32_array(group_len if len(group_len) else [0])
        nxt = np.zeros(max(m, 1), dtype=np.int32)
        n_next, runs = C.c_int32(0), C.c_int32(0)
        self._check(self.lib.keep_select_groups(
            self.handle, S.ctypes.data_as(C.POINTER(C.c_float)), gp, m, glp, len(group_len), float(ratio_next), hops,
            budget_mode, nxt.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(n_next), C.byref(runs)))
        return [int(v) for v in nxt[:n_next.value]], runs.value

    def prefill(self, prompt: KeepPrompt, ratios: Sequence[float], hops: int, k_cache: torch.Tensor,
                v_cache: torch.Tensor, x_final: torch.Tensor, budget_mode: int = KEEP_BUDGET_GROUP_COUNT,
                load_mode: int = KEEP_LOAD_LAYER_BALANCED, want_report: bool = False,
                cache_rows: Optional[int] = None, gate_up_events_only: bool = False):
        """cache_rows: rows per layer of k_cache / v_cache when they leave room for decoded tokens.
        gate_up_events_only: with a report, time only the gate/up GEMM (far fewer HIP events in the stream)."""
        L, G = self.shape.n_layers, prompt.n_groups
        r = np.ascontiguousarray(np.asarray(ratios, dtype=np.float32))
        sel = np.zeros(max(1, L * G), dtype=np.int32)
        cnt = np.zeros(L, dtype=np.int32)
        rep = Report() if want_report else None
        if want_report:
            rep.events_in = 1 if gate_up_events_only else 0
        if cache_rows is None:
            self._check(self.lib.keep_prefill(
                self.handle, C.byref(prompt.c), r.ctypes.data_as(C.POINTER(C.c_float)), hops, budget_mode, load_mode,
                k_cache.data_ptr(), v_cache.data_ptr(), x_final.data_ptr(), sel.ctypes.data_as(C.POINTER(C.c_int32)),
                cnt.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(rep) if want_report else None))
        else:
            self._check(self.lib.keep_prefill_padded(
                self.handle, C.byref(prompt.c), r.ctypes.data_as(C.POINTER(C.c_float)), hops, budget_mode, load_mode,
                k_cache.data_ptr(), v_cache.data_ptr(), cache_rows, x_final.data_ptr(),
                sel.ctypes.data_as(C.POINTER(C.c_int32)), cnt.ctypes.data_as(C.POINTER(C.c_int32)),
                C.byref(rep) if want_report else None))
        sets = [[int(v) for v in sel[l * G:l * G + cnt[l]]] for l in range(L)]
        return sets, rep

    def prefill_tokens(self, prompt: KeepPrompt, ratios: Sequence[float], k_cache: torch.Tensor, v_cache: torch.Tensor,
                       x_final: torch.Tensor, load_mode: int = KEEP_LOAD_LAYER_BALANCED, want_deviation: bool = False,
                       want_report: bool = False):
        """keep_prefill_tokens.  Returns (rows per layer, deviations per layer or None, report or None)."""
        L, nm = self.shape.n_layers, prompt.n_mem
        r = np.ascontiguousarray(np.asarray(ratios, dtype=np.float32))
        sel = np.zeros(max(1, L * nm), dtype=np.int32)
        cnt = np.zeros(L, dtype=np.int32)
        dev = np.zeros(max(1, L * nm), dtype=np.float32) if want_deviation else None
        rep = Report() if want_report else None
        self._check(self.lib.keep_prefill_tokens(
            self.handle, C.byref(prompt.c), r.ctypes.data_as(C.POINTER(C.c_float)), load_mode, k_cache.data_ptr(),
            v_cache.data_ptr(), x_final.data_ptr(), sel.ctypes.data_as(C.POINTER(C.c_int32)),
            cnt.ctypes.data_as(C.POINTER(C.c_int32)),
            dev.ctypes.data_as(C.POINTER(C.c_float)) if want_deviation else None,
            C.byref(rep) if want_report else None))
        rows = [[int(v) for v in sel[l * nm:l * nm + cnt[l]]] for l in range(L)]
        devs = [dev[l * nm:l * nm + cnt[l]].copy() for l in range(L)] if want_deviation else None
        return rows, devs, rep

    def select_tokens(self, deviation: np.ndarray, k: int) -> List[int]:
        d = np.ascontiguousarray(deviation, dtype=np.float32)
        out = np.zeros(max(1, k), dtype=np.int32)
        self._check(self.lib.keep_select_tokens(self.handle, d.ctypes.data_as(C.POINTER(C.c_float)), len(d), k,
                                                out.ctypes.data_as(C.POINTER(C.c_int32))))
        return [int(v) for v in out[:k]]

    def precompute_groups(self, unit_len: Sequence[int], token_ids: Sequence[int], k_blocks: torch.Tensor,
                          v_blocks: torch.Tensor, want_report: bool = False):
        """KV blocks [n_layers][sum(unit_len), n_kv_heads, head_dim] of several units, each computed on its own."""
        ul, ulp = _i32_array(unit_len)
        ids, ip = _i32_array(token_ids)
        rep = Report() if want_report else None
        self._check(self.lib.keep_precompute_groups(self.handle, len(ul), ulp, ip, k_blocks.data_ptr(),
                                                    v_blocks.data_ptr(), C.byref(rep) if want_report else None))
        return rep

    def decode(self, final_norm: torch.Tensor, lm_head: torch.Tensor, x_last: torch.Tensor, k_cache: torch.Tensor,
               v_cache: torch.Tensor, n_ctx: int, n_new: int, logits_out: Optional[torch.Tensor] = None,
               forced_tokens: Optional[Sequence[int]] = None):
        """Greedy tokens after a prompt of n_ctx tokens; caches are [n_layers, cache_rows, Hkv, dh]."""
        out = np.zeros(max(1, n_new), dtype=np.int32)
        f, fp = _forced_tokens(forced_tokens, n_new)
        self._check(self.lib.keep_decode(self.handle, final_norm.data_ptr(), lm_head.data_ptr(), x_last.data_ptr(),
                                         k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[1], n_ctx, n_new,
                                         out.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(logits_out), fp))
        return [int(v) for v in out[:n_new]]

    def decode_sampled(self, final_norm: torch.Tensor, lm_head: torch.Tensor, x_last: torch.Tensor, k_cache: torch.Tensor,
                       v_cache: torch.Tensor, n_ctx: int, uniform: Sequence[float], temperature: float = 1.0, top_k: int = 0,
                       top_p: float = 1.0, min_p: float = 0.0, logits_out: Optional[torch.Tensor] = None,
                       forced_tokens: Optional[Sequence[int]] = None):
        """keep_decode_sampled: one token per uniform number; returns (tokens, their probabilities)"""
        u = np.ascontiguousarray(np.asarray(uniform, dtype=np.float32))
        n_new = len(u)
        out, probs = np.zeros(max(1, n_new), dtype=np.int32), np.zeros(max(1, n_new), dtype=np.float32)
        f, fp = _forced_tokens(forced_tokens, n_new)
        how = Sampling(temperature, top_k, top_p, min_p, u.ctypes.data_as(C.POINTER(C.c_float)))
        self._check(self.lib.keep_decode_sampled(
            self.handle, final_norm.data_ptr(), lm_head.data_ptr(), x_last.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            k_cache.shape[1], n_ctx, n_new, C.byref(how), out.ctypes.data_as(C.POINTER(C.c_int32)),
            probs.ctypes.data_as(C.POINTER(C.c_float)), _ptr(logits_out), fp))
        return [int(v) for v in out[:n_new]], [float(v) for v in probs[:n_new]]

    def precompute_group(self, token_ids: Sequence[int], k_blocks: torch.Tensor, v_blocks: torch.Tensor,
                         want_report: bool = False):
        """KV blocks [n_layers][n, n_kv_heads, head_dim] of one memory unit computed on its own."""
        ids, ip = _i32_array(token_ids)
        rep = Report() if want_report else None
        self._check(self.lib.keep_precompute_group(self.handle, ip, len(ids), k_blocks.data_ptr(), v_blocks.data_ptr(),
                                                   C.byref(rep) if want_report else None))
        return rep


class KeepMemory:
    """Static-dynamic memory store of the library (host-side bookkeeping; marshalling only)."""

    def __init__(self, window_t: int):
        self.lib = load_library()
        h = C.c_void_p()
        st = self.lib.keep_memory_create(window_t, C.byref(h))
        if st != KEEP_OK:
            raise KeepError(st, "keep_memory_create failed")
        self.handle = h

    def close(self):
        if self.handle:
            self.lib.keep_memory_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != KEEP_OK:
            raise KeepError(st, self.lib.keep_memory_last_error(self.handle).decode())

    def put(self, group: int, segment: int, tokens: Sequence[int]) -> bool:
        ids, ip = _i32_array(tokens if len(tokens) else [0])
        changed = C.c_int32(0)
        self._check(self.lib.keep_memory_put(self.handle, group, segment, ip, len(tokens), C.byref(changed)))
        return bool(changed.value)

    def remove(self, segment: int):
        self._check(self.lib.keep_memory_remove(self.handle, segment))

    def end_step(self, cap: int = 4096):
        rep = MemoryStepReport()
        td = np.zeros(cap, dtype=np.int32)
        ts = np.zeros(cap, dtype=np.int32)
        p32 = C.POINTER(C.c_int32)
        self._check(self.lib.keep_memory_end_step(self.handle, C.byref(rep), td.ctypes.data_as(p32), cap,
                                                  ts.ctypes.data_as(p32), cap))
        return rep, [int(v) for v in td[:rep.n_to_dynamic]], [int(v) for v in ts[:rep.n_to_static]]

    def units(self):
        out = []
        for i in range(self.lib.keep_memory_unit_count(self.handle)):
            u = MemoryUnit()
            self._check(self.lib.keep_memory_unit_info(self.handle, i, C.byref(u)))
            out.append(u)
        return out

    def unit_tokens(self, unit: int, cap: int):
        buf = np.zeros(max(1, cap), dtype=np.int32)
        n = C.c_int32(0)
        self._check(self.lib.keep_memory_unit_tokens(self.handle, unit, buf.ctypes.data_as(C.POINTER(C.c_int32)), cap,
                                                     C.byref(n)))
        return [int(v) for v in buf[:n.value]]

    def mark_computed(self, unit: int):
        self._check(self.lib.keep_memory_mark_computed(self.handle, unit))
