"""GB300 (sm_103a) Llama-family decoder forward behind a C ABI.

This module is the thin Python binding of `libaxon_gb300.so` (see
`include/axon.h`): functions with the C names that marshal torch tensors
into pointers and raise on a non-zero status. Every step of the forward pass
runs in the library's CUDA kernels; torch only provides device memory and
streams. There is no CPU fallback: if the library was not built, the first
call raises.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaxon_gb300.so")

AXON_OK = 0
AXON_ERR_INVALID_ARG = 1
AXON_ERR_SHAPE_MISMATCH = 2
AXON_ERR_MISSING_WEIGHT = 3
AXON_ERR_UNSUPPORTED = 4
AXON_ERR_OOM = 5
AXON_ERR_CUDA = 6
AXON_ERR_TIMEOUT = 7
AXON_ERR_DEVICE_CHECK = 8
AXON_KV_CONTIGUOUS, AXON_KV_PAGED = 0, 1
AXON_BF16, AXON_FP32_DEBUG, AXON_FP16 = 0, 1, 2
AXON_DTYPE_BF16, AXON_DTYPE_F32 = 0, 1
AXON_LOGITS_LAST, AXON_LOGITS_ALL = 0, 1
AXON_ACT_SILU, AXON_ACT_GELU_TANH = 0, 1
AXON_ROPE_HALF, AXON_ROPE_INTERLEAVED = 0, 1

EXPORTED = ["axon_model_create", "axon_prefill", "axon_prefill_varlen", "axon_decode_step", "axon_reset",
            "axon_check_device", "axon_kv_view_get", "axon_profile_decode_step", "axon_profile_prefill",
            "axon_decode_step_noalloc", "axon_moe_routing_record", "axon_kv_cache_get", "axon_attn_decode",
            "axon_attn_decode_workspace", "axon_attn_prefill", "axon_attn_shared", "axon_attn_shared_workspace",
            "axon_rope_table", "axon_kv_append", "axon_sample", "axon_kv_copy_blocks", "axon_kv_fork",
            "axon_kv_release", "axon_kv_reserve", "axon_kv_compact", "axon_kv_workspace", "axon_check_error",
            "axon_free", "axon_status_string"]


class axon_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_hidden_layers", "hidden_size", "num_attention_heads", "num_key_value_heads", "head_dim",
        "intermediate_size", "vocab_size", "tie_word_embeddings", "attention_bias")] + [
        ("rope_theta", ctypes.c_float), ("rms_norm_eps", ctypes.c_float)] + [
        (n, ctypes.c_int32) for n in ("max_batch", "max_context", "max_prefill_tokens", "kv_layout",
                                      "kv_block_size", "kv_num_blocks", "precision", "sliding_window")] + [
        (n, ctypes.c_float) for n in ("rope_scaling_factor", "rope_low_freq_factor", "rope_high_freq_factor")] + [
        ("rope_original_max_position", ctypes.c_int32), ("hidden_act", ctypes.c_int32), ("qk_norm", ctypes.c_int32)] + [
        (n, ctypes.c_int32) for n in ("n_routed_experts", "num_experts_per_tok", "moe_intermediate_size",
                                      "n_shared_experts", "first_k_dense_replace", "norm_topk_prob", "sink_tokens")]


class axon_tensor(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("data", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("ndim", ctypes.c_int32), ("shape", ctypes.c_int64 * 4)]


class axon_kv_view(ctypes.Structure):
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("num_blocks", ctypes.c_int64),
                ("blocks_per_seq", ctypes.c_int32), ("block_size", ctypes.c_int32), ("elem_bytes", ctypes.c_int32)]


class axon_kernel_time(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_float),
                ("bytes", ctypes.c_double), ("flops", ctypes.c_double)]


class axon_kv_cache(ctypes.Structure):
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p)] + [
        (n, ctypes.c_int32) for n in ("num_layers", "num_blocks", "num_kv_heads", "block_size", "head_dim", "precision")]


class axon_kv_seqs(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("context_lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("max_seqs", ctypes.c_int32), ("blocks_per_seq", ctypes.c_int32)]


class AxonError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn} failed: {status} ({axon_status_string(status)})")


_lib = None
_torch = None  # imported with the library
_raw_stream = None  # (device index) -> the current stream's handle
_current_device = None  # () -> index of the device that launches go to


def lib() -> ctypes.CDLL:
    """Load the CUDA library (raises if it has not been built)."""
    global _lib, _torch, _raw_stream, _current_device
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2608_19889_gb300.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, p_i32 = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)
        L.axon_model_create.argtypes = [ctypes.POINTER(axon_config), ctypes.POINTER(axon_tensor), i32, vp,
                                        ctypes.POINTER(vp)]
        L.axon_prefill.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp]
        L.axon_prefill_varlen.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, i32, vp, vp, vp]
        L.axon_decode_step.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
        L.axon_decode_step_noalloc.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
        L.axon_moe_routing_record.argtypes = [vp, vp, i32]
        L.axon_reset.argtypes = [vp]
        L.axon_check_device.argtypes = [vp, vp, p_i32]
        L.axon_kv_view_get.argtypes = [vp, ctypes.POINTER(axon_kv_view)]
        L.axon_profile_decode_step.argtypes = [vp, vp, i32, vp, vp, vp, vp, ctypes.POINTER(axon_kernel_time), i32,
                                               p_i32]
        L.axon_profile_prefill.argtypes = [vp, vp, i32, i32, vp, vp, vp, ctypes.POINTER(axon_kernel_time), i32, p_i32]
        i64, f32, p_i64 = ctypes.c_int64, ctypes.c_float, ctypes.POINTER(ctypes.c_int64)
        L.axon_kv_cache_get.argtypes = [vp, ctypes.POINTER(axon_kv_cache)]
        L.axon_attn_decode.argtypes = [vp, i32, vp, i64, i64, i32, i32, vp, vp, i32, i32, i32, f32, vp, i64, i64, vp, vp,
                                       i64, vp, vp]
        L.axon_attn_decode_workspace.argtypes = [vp, i32, i32, p_i64]
        L.axon_attn_prefill.argtypes = [vp, i32, vp, i64, i64, i32, i32, i32, vp, vp, i32, vp, i32, i32, i32, f32, vp,
                                        i64, i64, vp, vp]
        L.axon_attn_shared.argtypes = [vp, i32, vp, i64, i64, i32, i32, vp, vp, i32, vp, vp, i32, i32, i32, f32, vp, i64, i64,
                                       vp, vp, i64, vp, vp]
        L.axon_attn_shared_workspace.argtypes = [vp, i32, i32, p_i64]
        L.axon_rope_table.argtypes = [vp, i32, i32, f32, f32, f32, f32, i32, vp]
        L.axon_kv_append.argtypes = [vp, i32] + [vp, i64, i64] * 3 + [i32, i32, i32, vp, vp, vp, i32, vp, i32, i32, i32, vp,
                                                                      i64, i64, vp, vp]
        L.axon_sample.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.axon_kv_copy_blocks.argtypes = [vp, vp, vp, i32, vp, vp]
        L.axon_kv_fork.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp, vp]
        L.axon_kv_release.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp]
        L.axon_kv_reserve.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp, vp]
        L.axon_kv_compact.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp]
        L.axon_kv_workspace.argtypes = [vp, vp, p_i64]
        L.axon_check_error.argtypes = [vp, vp, p_i32]
        L.axon_free.argtypes = [vp]
        L.axon_free.restype = None
        L.axon_status_string.argtypes = [ctypes.c_int]
        L.axon_status_string.restype = ctypes.c_char_p
        for n in ("axon_model_create", "axon_prefill", "axon_prefill_varlen", "axon_decode_step", "axon_reset",
                  "axon_check_device", "axon_kv_view_get", "axon_profile_decode_step", "axon_profile_prefill",
                  "axon_decode_step_noalloc", "axon_moe_routing_record", "axon_kv_cache_get", "axon_attn_decode",
                  "axon_attn_decode_workspace", "axon_attn_prefill", "axon_kv_copy_blocks", "axon_kv_fork",
                  "axon_kv_release", "axon_kv_reserve", "axon_kv_compact", "axon_kv_workspace", "axon_check_error",
                  "axon_rope_table", "axon_kv_append", "axon_sample", "axon_attn_shared",
                  "axon_attn_shared_workspace"):
            getattr(L, n).restype = ctypes.c_int
        import torch
        _torch = torch
        # a handle without the Stream object around it (0.1 us against 3 us), where this torch has the call
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        lib()
        if _raw_stream is not None:
            return _raw_stream(_torch.cuda.current_device())
        stream = _torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(fn, rc):
    if rc != AXON_OK:
        raise AxonError(fn, rc)


def axon_status_string(status: int) -> str:
    return lib().axon_status_string(status).decode()


def make_config(m: dict, max_batch: int, max_context: int, kv_layout=AXON_KV_CONTIGUOUS, kv_num_blocks=0,
                precision=AXON_BF16, max_prefill_tokens=0) -> axon_config:
    """axon_config from a shape dict with keys L, D, H, G, d, F, V, tie, bias, theta, eps (and optionally
    window, the sliding window, sinks, the first tokens that stay visible under it, rope_factor / rope_low / rope_high / rope_orig, the RoPE frequency
    scaling, 0 or absent = none; act, "silu" (default) or "gelu_tanh"; qk_norm, per-head RMSNorm of q and k;
    n_experts, top_k, moe_F, n_shared, first_dense, norm_topk: the mixture-of-experts MLP)."""
    return axon_config(m["L"], m["D"], m["H"], m["G"], m["d"], m["F"], m["V"], int(m["tie"]), int(m["bias"]),
                       float(m["theta"]), float(m["eps"]), max_batch, max_context, max_prefill_tokens, kv_layout, 16,
                       kv_num_blocks, precision, int(m.get("window", 0)), float(m.get("rope_factor", 0.0)),
                       float(m.get("rope_low", 1.0)), float(m.get("rope_high", 4.0)), int(m.get("rope_orig", 8192)),
                       AXON_ACT_GELU_TANH if m.get("act", "silu") == "gelu_tanh" else AXON_ACT_SILU,
                       int(bool(m.get("qk_norm", False))), int(m.get("n_experts", 0)), int(m.get("top_k", 0)),
                       int(m.get("moe_F", 0)), int(m.get("n_shared", 0)), int(m.get("first_dense", 0)),
                       int(bool(m.get("norm_topk", False))), int(m.get("sinks", 0)))


def axon_model_create(cfg: axon_config, weights: dict, stream=None) -> ctypes.c_void_p:
    """Create a model from {HF name: torch tensor (bf16 or fp32, host or device)}."""
    import torch
    names = list(weights.keys())
    arr = (axon_tensor * len(names))()
    keep = []
    for i, n in enumerate(names):
        t = weights[n].contiguous()
        keep.append(t)
        if t.dtype == torch.bfloat16:
            dt = AXON_DTYPE_BF16
        elif t.dtype == torch.float32:
            dt = AXON_DTYPE_F32
        else:
            raise TypeError(f"{n}: unsupported dtype {t.dtype}")
        shape = (ctypes.c_int64 * 4)(*(list(t.shape) + [0] * (4 - t.dim())))
        arr[i] = axon_tensor(n.encode(), t.data_ptr(), dt, t.dim(), shape)
    h = ctypes.c_void_p()
    _check("axon_model_create", lib().axon_model_create(ctypes.byref(cfg), arr, len(names), _stream(stream),
                                                        ctypes.byref(h)))
    h.device = torch.cuda.current_device()
    return h


def axon_prefill(m, ids, block_table=None, logits_mode=AXON_LOGITS_LAST, logits=None, next_tokens=None,
                 stream=None):
    """ids: int32 [B, S] on the device; outputs written into the given tensors."""
    B, S = ids.shape
    _check("axon_prefill", lib().axon_prefill(m, _ptr(ids), B, S, _ptr(block_table), logits_mode, _ptr(logits),
                                              _ptr(next_tokens), _stream(stream)))


def axon_prefill_varlen(m, ids, cu_seqlens, context_lens, max_chunk, block_table=None, logits_mode=AXON_LOGITS_LAST,
                        logits=None, next_tokens=None, stream=None):
    """ids: int32 [T] packed chunks; cu_seqlens: int32 [B+1] row offsets;
    context_lens: int32 [B] tokens cached before each chunk (advanced by the
    chunk lengths); max_chunk: host bound on the longest chunk. All device
    tensors; outputs written into the given tensors."""
    T = ids.shape[0]
    B = cu_seqlens.shape[0] - 1
    _check("axon_prefill_varlen", lib().axon_prefill_varlen(
        m, _ptr(ids), B, T, _ptr(cu_seqlens), _ptr(context_lens), int(max_chunk), _ptr(block_table), logits_mode,
        _ptr(logits), _ptr(next_tokens), _stream(stream)))


def axon_decode_step(m, tokens, context_lens, block_table=None, logits=None, next_tokens=None, stream=None):
    """tokens, context_lens: int32 [B] on the device (context_lens advances by one)."""
    B = tokens.shape[0]
    _check("axon_decode_step", lib().axon_decode_step(m, _ptr(tokens), B, _ptr(context_lens), _ptr(block_table),
                                                      _ptr(logits), _ptr(next_tokens), _stream(stream)))


def axon_moe_routing_record(m, experts=None, rows=0):
    """experts: int32 device tensor [L, rows, k] that later passes fill with
    each MoE layer's chosen experts (see include/axon.h), or None to stop."""
    _check("axon_moe_routing_record", lib().axon_moe_routing_record(m, _ptr(experts), int(rows)))


def axon_decode_step_noalloc(m, tokens, context_lens, block_table=None, logits=None, next_tokens=None, stream=None):
    """Allocation-free decode step (see include/axon.h): same contract as
    axon_decode_step, direct launches, fixed library-owned merge scratch."""
    B = tokens.shape[0]
    _check("axon_decode_step_noalloc", lib().axon_decode_step_noalloc(
        m, _ptr(tokens), B, _ptr(context_lens), _ptr(block_table), _ptr(logits), _ptr(next_tokens), _stream(stream)))


def axon_reset(m):
    _check("axon_reset", lib().axon_reset(m))


def axon_check_device(m, stream=None) -> tuple[int, int]:
    """(status, raw error bits) after synchronising the stream."""
    bits = ctypes.c_int32(0)
    rc = lib().axon_check_device(m, _stream(stream), ctypes.byref(bits))
    return rc, bits.value


def axon_kv_view_get(m) -> axon_kv_view:
    v = axon_kv_view()
    _check("axon_kv_view_get", lib().axon_kv_view_get(m, ctypes.byref(v)))
    return v


def _profile_result(arr, n):
    return [dict(name=arr[i].name.decode(), launches=arr[i].launches, total_ms=arr[i].total_ms,
                 bytes=arr[i].bytes, flops=arr[i].flops) for i in range(n.value)]


def axon_profile_decode_step(m, tokens, context_lens, block_table=None, next_tokens=None, stream=None):
    """Per-kernel-kind timing of one decode step (runs the step)."""
    arr = (axon_kernel_time * 16)()
    n = ctypes.c_int32(0)
    B = tokens.shape[0]
    _check("axon_profile_decode_step", lib().axon_profile_decode_step(
        m, _ptr(tokens), B, _ptr(context_lens), _ptr(block_table), _ptr(next_tokens), _stream(stream), arr, 16,
        ctypes.byref(n)))
    return _profile_result(arr, n)


def axon_profile_prefill(m, ids, block_table=None, next_tokens=None, stream=None):
    """Per-kernel-kind timing of one prefill (LAST-position logits not stored)."""
    arr = (axon_kernel_time * 16)()
    n = ctypes.c_int32(0)
    B, S = ids.shape
    _check("axon_profile_prefill", lib().axon_profile_prefill(
        m, _ptr(ids), B, S, _ptr(block_table), _ptr(next_tokens), _stream(stream), arr, 16, ctypes.byref(n)))
    return _profile_result(arr, n)


def axon_free(m):
    lib().axon_free(m)


# ------------------------------------------------- operators on a paged cache
# Small calls are bound by the host: what a wrapper reads of a tensor costs 0.05 to 0.15 us apiece.


def _want(t, dtype, what, n, device):
    """Address of a dense tensor of n elements on the device; refuse what the C call could not tell from one."""
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.numel() == n:
        return t.data_ptr()
    raise TypeError(f"{what}: a dense {dtype} tensor of {n} elements on cuda:{max(device, 0)} is wanted, got {t.dtype} "
                    f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _list(t, what, device):
    """Address and length of a dense int32 device vector."""
    if t.dim() != 1:
        raise TypeError(f"{what}: a vector is wanted, got {tuple(t.shape)}")
    n = t.numel()
    return _want(t, _torch.int32, what, n, device), n


def _word(err, device):
    return None if err is None else _want(err, _torch.int32, "err", 1, device)


def _space(t, device):
    """Address of a workspace."""
    if t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise TypeError(f"workspace: dense memory of cuda:{device} is wanted, got {tuple(t.shape)} with strides {t.stride()} on "
                    f"{t.device}")


def _current(device):
    """Kernels go to the current device, which has to be the operands'."""
    if _current_device() != device:
        raise ValueError(f"operands are on cuda:{device}, the current device is cuda:{_current_device()}")


def _handle(stream, device):
    """The stream's handle; None: the device's current one."""
    if stream is None and _raw_stream is not None and _current_device() == device:
        return _raw_stream(device)
    _current(device)
    if getattr(stream, "device_index", device) != device:
        raise ValueError(f"operands are on cuda:{device}, the stream is on cuda:{stream.device_index}")
    return _stream(stream)


def make_kv_cache(k, v) -> axon_kv_cache:
    """Descriptor of the pools k, v: dense device tensors [layers, blocks, kv heads, 16, head_dim] (bf16, fp16; the
    block operators also take fp32). It holds their addresses: keep the tensors."""
    lib()
    prec = {_torch.bfloat16: AXON_BF16, _torch.float16: AXON_FP16, _torch.float32: AXON_FP32_DEBUG}.get(k.dtype)
    if prec is None or k.dim() != 5 or v.shape != k.shape:
        raise TypeError(f"k, v: bf16, fp16 or fp32 tensors of the same 5 dimensions are wanted, got {k.dtype} "
                        f"{tuple(k.shape)} and {v.dtype} {tuple(v.shape)}")
    L, N, G, bs, d = k.shape
    n, dev = k.numel(), _on(k, "k")
    return _described(axon_kv_cache(_want(k, k.dtype, "k", n, dev), _want(v, k.dtype, "v", n, dev), L, N, G, bs, d, prec), dev)


def _on(t, what):
    """Index of a tensor's device."""
    if not t.is_cuda:
        raise TypeError(f"{what}: device memory is wanted, got a tensor on {t.device}")
    return t.get_device()


def _described(c, device):
    """What the wrappers read of a descriptor at every call, as plain attributes."""
    c.device = device
    c.dtype = {AXON_BF16: _torch.bfloat16, AXON_FP16: _torch.float16, AXON_FP32_DEBUG: _torch.float32}[c.precision]
    c.blocks, c.dim, c.kv_heads, c.ref = c.num_blocks, c.head_dim, c.num_kv_heads, ctypes.byref(c)
    return c


def axon_kv_cache_get(m) -> axon_kv_cache:
    """Descriptor of a model's own cache."""
    c = axon_kv_cache()
    _check("axon_kv_cache_get", lib().axon_kv_cache_get(m, ctypes.byref(c)))
    return _described(c, getattr(m, "device", _current_device()))


def make_kv_seqs(block_table, context_lens, refs) -> axon_kv_seqs:
    """Descriptor of a block table [rows, blocks per row], lengths [rows] and counts [blocks] (int32, device). It holds
    their addresses: keep the tensors."""
    lib()
    R, P = block_table.shape
    dev = _on(block_table, "block_table")
    s = axon_kv_seqs(_want(block_table, _torch.int32, "block_table", R * P, dev),
                     _want(context_lens, _torch.int32, "context_lens", R, dev), _list(refs, "refs", dev)[0], R, P)
    s.device, s.blocks, s.ref = dev, refs.numel(), ctypes.byref(s)
    return s


def make_attn_workspace(cache, rows, heads):
    """Zeroed workspace of axon_attn_decode for `heads` heads on this cache, or for any call that needs no larger one."""
    n = ctypes.c_int64(0)
    _current(cache.device)
    _check("axon_attn_decode_workspace", lib().axon_attn_decode_workspace(cache.ref, heads, rows, ctypes.byref(n)))
    return _torch.zeros(n.value, dtype=_torch.uint8, device=_torch.device("cuda", cache.device))


def make_shared_workspace(cache, rows, heads):
    """Zeroed workspace of axon_attn_shared for up to `rows` rows of `heads` heads on this cache; it serves axon_attn_decode
    too."""
    n = ctypes.c_int64(0)
    _current(cache.device)
    _check("axon_attn_shared_workspace", lib().axon_attn_shared_workspace(cache.ref, heads, rows, ctypes.byref(n)))
    return _torch.zeros(n.value, dtype=_torch.uint8, device=_torch.device("cuda", cache.device))


def make_kv_workspace(cache, seqs):
    """Workspace of axon_kv_fork, axon_kv_reserve and axon_kv_compact."""
    n = ctypes.c_int64(0)
    _check("axon_kv_workspace", lib().axon_kv_workspace(cache.ref, seqs.ref, ctypes.byref(n)))
    return _torch.empty(n.value, dtype=_torch.uint8, device=_torch.device("cuda", cache.device))


def _rows(q, out, cache):
    """(rows, heads, row stride, head stride of q, of out) of [rows, heads, head_dim] tensors of the cache's type."""
    shape, qs, os_ = q.shape, q.stride(), out.stride()
    if (len(shape) != 3 or out.shape != shape or shape[2] != cache.dim or q.dtype is not cache.dtype or
            out.dtype is not cache.dtype or qs[2] != 1 or os_[2] != 1 or q.get_device() != cache.device or
            out.get_device() != cache.device):
        raise TypeError(f"q, out: {cache.dtype} tensors [rows, heads, {cache.dim}] on cuda:{cache.device} with a dense last "
                        f"dimension are wanted, got {q.dtype} {tuple(shape)} on {q.device}, {out.dtype} {tuple(out.shape)} on {out.device}")
    return shape[0], shape[1], qs[0], qs[1], os_[0], os_[1]


def _table(block_table, blocks_per_seq, rows, device):
    if block_table is None:
        return None, blocks_per_seq
    per = block_table.shape[-1]
    return _want(block_table, _torch.int32, "block_table", rows * per, device), per


def axon_attn_decode(cache, layer, q, context_lens, out, workspace, block_table=None, blocks_per_seq=0, window=0, sinks=0,
                     scale=0.0, lse=None, err=None, stream=None):
    """Attention of one new token per row (see include/axon.h). q, out: [B, heads, head_dim], any row and head strides;
    context_lens: int32 [B]; block_table: int32 [B, blocks], or None with blocks_per_seq for contiguous rows;
    workspace: make_attn_workspace; lse: fp32 [B, heads] or None; err: int32 [1] error word or None."""
    B, H, qr, qh, orow, ohead = _rows(q, out, cache)
    dev = cache.device
    table, per = _table(block_table, blocks_per_seq, B, dev)
    rc = _lib.axon_attn_decode(
        cache.ref, layer, q.data_ptr(), qr, qh, B, H, _want(context_lens, _torch.int32, "context_lens", B, dev), table, per,
        window, sinks, scale, out.data_ptr(), orow, ohead,
        None if lse is None else _want(lse, _torch.float32, "lse", B * H, dev), _space(workspace, dev), workspace.nbytes,
        None if err is None else _word(err, dev), _handle(stream, dev))
    if rc:
        raise AxonError("axon_attn_decode", rc)


def axon_attn_shared(cache, layer, q, context_lens, group_offsets, prefix_lens, out, workspace, block_table, window=0,
                     sinks=0, scale=0.0, lse=None, err=None, stream=None):
    """axon_attn_decode for rows in groups whose first blocks are the same (see include/axon.h). group_offsets: int32
    [groups + 1], rows of the groups; prefix_lens: int32 [groups], tokens whose whole blocks they share; workspace:
    make_shared_workspace; the rest as in axon_attn_decode."""
    B, H, qr, qh, orow, ohead = _rows(q, out, cache)
    dev = cache.device
    table, per = _table(block_table, 0, B, dev)
    prefix, N = _list(prefix_lens, "prefix_lens", dev)
    rc = _lib.axon_attn_shared(
        cache.ref, layer, q.data_ptr(), qr, qh, B, H, _want(context_lens, _torch.int32, "context_lens", B, dev), table, per,
        _want(group_offsets, _torch.int32, "group_offsets", N + 1, dev), prefix, N, window, sinks, scale, out.data_ptr(), orow,
        ohead, None if lse is None else _want(lse, _torch.float32, "lse", B * H, dev), _space(workspace, dev), workspace.nbytes,
        None if err is None else _word(err, dev), _handle(stream, dev))
    if rc:
        raise AxonError("axon_attn_shared", rc)


def axon_attn_prefill(cache, layer, q, cu_seqlens, context_lens, max_chunk, out, block_table=None, blocks_per_seq=0,
                      window=0, sinks=0, scale=0.0, err=None, stream=None):
    """Attention of packed chunks (see include/axon.h). q, out: [T, heads, head_dim]; cu_seqlens: int32 [B+1];
    context_lens: int32 [B] tokens before each chunk (not advanced); the rest as in axon_attn_decode."""
    T, H, qr, qh, orow, ohead = _rows(q, out, cache)
    dev = cache.device
    past, B = _list(context_lens, "context_lens", dev)
    table, per = _table(block_table, blocks_per_seq, B, dev)
    rc = _lib.axon_attn_prefill(
        cache.ref, layer, q.data_ptr(), qr, qh, B, T, H, _want(cu_seqlens, _torch.int32, "cu_seqlens", B + 1, dev), past,
        max_chunk, table, per, window, sinks, scale, out.data_ptr(), orow, ohead, None if err is None else _word(err, dev),
        _handle(stream, dev))
    if rc:
        raise AxonError("axon_attn_prefill", rc)


def axon_rope_table(positions, rotary_dim, theta, factor=0.0, low=1.0, high=4.0, original=8192, device=None, stream=None):
    """Rotary table fp32 [positions, rotary_dim / 2, 2] of axon_kv_append (see include/axon.h); factor, low, high, original: the
    frequency scaling of make_config's rope_factor, rope_low, rope_high, rope_orig (0: none). device: where it is made; None, or
    one without a number: the current device."""
    lib()
    dev = _torch.device("cuda" if device is None else device)
    if dev.type != "cuda":
        raise TypeError(f"device: a CUDA device is wanted, got {dev}")
    dev = _torch.device("cuda", _current_device() if dev.index is None else dev.index)
    handle = _handle(stream, dev.index)
    table = _torch.empty(positions, rotary_dim // 2, 2, dtype=_torch.float32, device=dev)
    _check("axon_rope_table",
           _lib.axon_rope_table(table.data_ptr(), positions, rotary_dim, theta, factor, low, high, original, handle))
    return table


def _heads(t, what, rows, heads, cache):
    """Address, row and head strides of a tensor [rows, heads, head_dim] of the cache's type."""
    shape, s = t.shape, t.stride()
    if (len(shape) == 3 and shape[0] == rows and shape[1] == heads and shape[2] == cache.dim and t.dtype is cache.dtype and
            s[2] == 1 and t.get_device() == cache.device):
        return t.data_ptr(), s[0], s[1]
    raise TypeError(f"{what}: a {cache.dtype} tensor [{rows}, {heads}, {cache.dim}] on cuda:{cache.device} with a dense last "
                    f"dimension is wanted, got {t.dtype} {tuple(shape)} with strides {s} on {t.device}")


def axon_kv_append(cache, layer, k, v, context_lens, block_table=None, blocks_per_seq=0, cu_seqlens=None, rope=None,
                   interleaved=False, q=None, q_out=None, err=None, stream=None):
    """New tokens into a layer of the cache, keys and queries rotated (see include/axon.h). k, v: [T, kv heads, head_dim] and
    q, q_out: [T, heads, head_dim] (q_out may be q), any row and head strides; context_lens: int32 [B] tokens before the
    new ones (not advanced); cu_seqlens: int32 [B+1], or None: one token per row; rope: fp32 [positions, rotated pairs, 2]
    as axon_rope_table returns it, or None: no rotation; block_table, blocks_per_seq as in axon_attn_decode."""
    dev, T = cache.device, k.shape[0]
    past, B = _list(context_lens, "context_lens", dev)
    table, per = _table(block_table, blocks_per_seq, B, dev)
    positions = pairs = 0
    turn = None
    if rope is not None:
        positions, pairs = rope.shape[0], rope.shape[1]
        turn = _want(rope, _torch.float32, "rope", 2 * positions * pairs, dev)
    if q is None:
        if q_out is not None:
            raise TypeError("q_out: there is no q to rotate")
        heads, queries, out = 0, (None, 0, 0), (None, 0, 0)
    else:
        heads = q.shape[1]
        queries, out = _heads(q, "q", T, heads, cache), _heads(q_out, "q_out", T, heads, cache)
    rc = _lib.axon_kv_append(
        cache.ref, layer, *queries, *_heads(k, "k", T, cache.kv_heads, cache), *_heads(v, "v", T, cache.kv_heads, cache), B, T,
        heads, None if cu_seqlens is None else _want(cu_seqlens, _torch.int32, "cu_seqlens", B + 1, dev), past, table, per,
        turn, positions, 2 * pairs, AXON_ROPE_INTERLEAVED if interleaved else AXON_ROPE_HALF, *out,
        None if err is None else _word(err, dev), _handle(stream, dev))
    if rc:
        raise AxonError("axon_kv_append", rc)


def _same_pool(cache, seqs):
    if cache.blocks != seqs.blocks:
        raise TypeError(f"refs: {cache.blocks} counts are wanted, one per block, got {seqs.blocks}")
    if cache.device != seqs.device:
        raise TypeError(f"tables on cuda:{cache.device} are wanted, got cuda:{seqs.device}")
    return cache.device


def axon_kv_copy_blocks(cache, src, dst, err=None, stream=None):
    """Copy blocks src[i] to dst[i] (int32 [n]) in all layers."""
    dev = cache.device
    s, n = _list(src, "src", dev)
    _check("axon_kv_copy_blocks", _lib.axon_kv_copy_blocks(cache.ref, s, _want(dst, _torch.int32, "dst", n, dev), n,
                                                           _word(err, dev), _handle(stream, dev)))


def axon_kv_fork(cache, seqs, src, dst, workspace, err=None, stream=None):
    """Rows dst[i] take over what rows src[i] hold (int32 [n]); workspace: make_kv_workspace."""
    dev = _same_pool(cache, seqs)
    s, n = _list(src, "src", dev)
    _check("axon_kv_fork", _lib.axon_kv_fork(cache.ref, seqs.ref, s, _want(dst, _torch.int32, "dst", n, dev), n,
                                             _space(workspace, dev), workspace.nbytes, _word(err, dev), _handle(stream, dev)))


def axon_kv_release(cache, seqs, rows, window=0, sinks=0, err=None, stream=None):
    """Rows (int32 [n]) give back everything, or with a window what no later query sees."""
    dev = _same_pool(cache, seqs)
    r, n = _list(rows, "rows", dev)
    _check("axon_kv_release", _lib.axon_kv_release(cache.ref, seqs.ref, r, n, window, sinks, _word(err, dev),
                                                   _handle(stream, dev)))


def axon_kv_reserve(cache, seqs, rows, new_tokens, workspace, err=None, stream=None):
    """Rows (int32 [n]) take blocks for new_tokens (int32 [n]) more tokens; workspace: make_kv_workspace."""
    dev = _same_pool(cache, seqs)
    r, n = _list(rows, "rows", dev)
    _check("axon_kv_reserve", _lib.axon_kv_reserve(
        cache.ref, seqs.ref, r, _want(new_tokens, _torch.int32, "new_tokens", n, dev), n, _space(workspace, dev),
        workspace.nbytes, _word(err, dev), _handle(stream, dev)))


def axon_kv_compact(cache, seqs, workspace, moved=None, live=None, err=None, stream=None):
    """Move the blocks in use to the front of the pool. moved: int32 [blocks] each block's number afterwards (-1: free);
    live: int32 [1] their count; workspace: make_kv_workspace."""
    dev = _same_pool(cache, seqs)
    _check("axon_kv_compact", _lib.axon_kv_compact(
        cache.ref, seqs.ref, None if moved is None else _want(moved, _torch.int32, "moved", cache.blocks, dev),
        None if live is None else _want(live, _torch.int32, "live", 1, dev), _space(workspace, dev), workspace.nbytes,
        _word(err, dev), _handle(stream, dev)))


def axon_check_error(err, stream=None) -> tuple[int, int]:
    """(status, bits) of an operator's error word (int32 [1]) after synchronising the stream; the word is cleared."""
    bits = ctypes.c_int32(0)
    dev = _on(err, "err")
    rc = lib().axon_check_error(_word(err, dev), _handle(stream, dev), ctypes.byref(bits))
    return rc, bits.value


def axon_sample(logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, stream=None):
    """A token per row (see include/axon.h). logits: fp32, bf16 or fp16 [B, V], any row stride; u: fp32 [B] random numbers in
    [0, 1); tokens: int32 [B]; temperature, top_p, min_p: fp32 [B] and top_k: int32 [B], or None (1, 1, 0, all); prob: fp32
    [B] or None, the token's probability among those it was chosen from."""
    if _lib is None:
        lib()
    dtype = logits.dtype
    prec = (AXON_FP32_DEBUG if dtype is _torch.float32 else AXON_BF16 if dtype is _torch.bfloat16 else
            AXON_FP16 if dtype is _torch.float16 else None)
    if prec is None or logits.dim() != 2 or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits: a device tensor [rows, vocabulary] of fp32, bf16 or fp16 with dense rows is wanted, got "
                        f"{dtype} {tuple(logits.shape)} with strides {logits.stride()} on {logits.device}")
    (B, V), dev = logits.shape, logits.get_device()
    f32 = _torch.float32
    rc = _lib.axon_sample(
        logits.data_ptr(), logits.stride(0), prec, B, V,
        None if temperature is None else _want(temperature, f32, "temperature", B, dev),
        None if top_k is None else _want(top_k, _torch.int32, "top_k", B, dev),
        None if top_p is None else _want(top_p, f32, "top_p", B, dev),
        None if min_p is None else _want(min_p, f32, "min_p", B, dev),
        _want(u, f32, "u", B, dev), _want(tokens, _torch.int32, "tokens", B, dev),
        None if prob is None else _want(prob, f32, "prob", B, dev), _handle(stream, dev))
    if rc:
        raise AxonError("axon_sample", rc)
