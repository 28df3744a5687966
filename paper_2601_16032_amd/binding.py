"""ctypes binding of libsawattn.so: argument marshalling only, same names as the C ABI.

Every step of the attention forward runs inside the HIP library.  There is no fallback: if the
library has not been built, loading raises.  PyTorch is used for device memory and streams.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

from .build import LIB_PATH, PAGED_BINDING_PATH, PROBE_LIB_PATH

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_RUNTIME = 0, 1, 2, 3
SCAN_CYCLIC, SCAN_SAWTOOTH = 0, 1
F16, BF16, F32 = 0, 1, 2

LAUNCH_PERSISTENT, LAUNCH_GRID, LAUNCH_AUTO = 0, 1, 2
DECODE_DOMAIN, DECODE_LINEAR = 0, 1

_DTYPE_CODE = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
_IN_DTYPE_CODE = {torch.float16: F16, torch.bfloat16: BF16}
_current_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_SCAN_CODE = {"cyclic": SCAN_CYCLIC, "sawtooth": SCAN_SAWTOOTH, SCAN_CYCLIC: SCAN_CYCLIC,
              SCAN_SAWTOOTH: SCAN_SAWTOOTH}


class LaunchInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "tile_q", "tile_kv", "block_threads", "grid", "lds_bytes", "domains", "slots",
        "parts_per_head", "q_tiles_per_head", "max_local_tiles", "launch", "tiles_per_workgroup",
        "qo_streaming")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Variant(ctypes.Structure):
    """sawattn_variant: which launch / work decode to run (None everywhere = the default)."""
    _fields_ = [("launch", ctypes.c_int), ("decode", ctypes.c_int), ("slots_per_domain", ctypes.c_int),
                ("tiles_per_workgroup", ctypes.c_int), ("rows_per_wavefront", ctypes.c_int),
                ("align_rounds", ctypes.c_int), ("kv_halves", ctypes.c_int), ("qo_streaming", ctypes.c_int)]


_LAUNCH_CODE = {"persistent": LAUNCH_PERSISTENT, "grid": LAUNCH_GRID, "auto": LAUNCH_AUTO}
_DECODE_CODE = {"domain": DECODE_DOMAIN, "linear": DECODE_LINEAR}


def variant(launch="persistent", decode="domain", slots_per_domain=0, tiles_per_workgroup=0,
            rows_per_wavefront=0, align_rounds=0, kv_halves=0, qo_streaming=0) -> Variant:
    return Variant(_LAUNCH_CODE.get(launch, launch), _DECODE_CODE.get(decode, decode),
                   int(slots_per_domain), int(tiles_per_workgroup), int(rows_per_wavefront), int(align_rounds),
                   int(kv_halves), int(qo_streaming))


def _vptr(v):
    return ctypes.byref(v) if v is not None else None


class SawattnError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"sawattn error {code}: {text}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load libsawattn.so (built by paper_2601_16032_amd.build.build()); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is not built; run `python -m paper_2601_16032_amd.build` "
                "(or __graft_entry__.build()) first -- there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.attn_fwd.restype = ci
        L.attn_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ctypes.c_float, ci, ci, ci, ci, vp]
        pv = ctypes.POINTER(Variant)
        L.attn_fwd_variant.restype = ci
        L.attn_fwd_variant.argtypes = L.attn_fwd.argtypes + [pv, vp, vp]
        L.attn_fwd_workspace.restype = ci
        L.attn_fwd_workspace.argtypes = L.attn_fwd_variant.argtypes + [vp, ctypes.c_size_t]
        L.attn_fwd_workspace_bytes.restype = ci
        L.attn_fwd_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci, pv, ctypes.POINTER(ctypes.c_size_t),
                                               ctypes.POINTER(LaunchInfo)]
        L.attn_fwd_static.restype = ci
        L.attn_fwd_static.argtypes = L.attn_fwd.argtypes
        L.attn_fwd_launch_info.restype = ci
        L.attn_fwd_launch_info.argtypes = [ci, ci, ci, ci, ci, ci, ci, ctypes.POINTER(LaunchInfo)]
        L.attn_fwd_variant_launch_info.restype = ci
        L.attn_fwd_variant_launch_info.argtypes = [ci, ci, ci, ci, ci, ci, pv, ctypes.POINTER(LaunchInfo)]
        L.attn_fwd_plan.restype = ci
        L.attn_fwd_plan.argtypes = [ci, ci, ci, ci, ci, ci, ci, pv, vp, vp]
        L.attn_kv_pages.restype = ci
        L.attn_kv_pages.argtypes = [vp, vp, ci, vp, i64, ci, ci, vp, ci, vp, vp, vp, vp, vp, vp, vp, ci, vp]
        L.attn_qkv_prepare.restype = ci
        L.attn_qkv_prepare.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp]
        L.attn_decode.restype = ci
        L.attn_decode.argtypes = [vp, i64, i64, vp, i64, i64, ci, vp, vp, i64, ci, vp, ci, ci, ctypes.c_float, ci, vp,
                                  ctypes.c_size_t, vp]
        L.attn_decode_workspace_bytes.restype = ci
        L.attn_decode_workspace_bytes.argtypes = [vp, ci, ci, ci, ctypes.POINTER(ctypes.c_size_t)]
        for name in ("attn_last_error", "sawattn_last_error"):
            getattr(L, name).restype = ctypes.c_char_p
            getattr(L, name).argtypes = []
        for name in ("attn_version", "sawattn_version"):
            getattr(L, name).restype = ci
            getattr(L, name).argtypes = []
        _lib = L
    return _lib


_probe_lib = None


def probe_lib() -> ctypes.CDLL:
    """Load libsawattn_probe.so, the benchmark's matrix-rate probe (built with the main library)."""
    global _probe_lib
    if _probe_lib is None:
        if not os.path.exists(PROBE_LIB_PATH):
            raise FileNotFoundError(f"{PROBE_LIB_PATH} is not built; run `python -m paper_2601_16032_amd.build` first")
        L = ctypes.CDLL(PROBE_LIB_PATH)
        L.sawattn_mfma_probe.restype = ctypes.c_int
        L.sawattn_mfma_probe.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                         ctypes.POINTER(ctypes.c_double)]
        L.sawattn_probe_last_error.restype = ctypes.c_char_p
        L.sawattn_probe_last_error.argtypes = []
        _probe_lib = L
    return _probe_lib


def attn_last_error() -> str:
    return lib().attn_last_error().decode()


def attn_version() -> int:
    return int(lib().attn_version())


sawattn_last_error, sawattn_version = attn_last_error, attn_version   # older names


def _check(rc: int):
    if rc != OK:
        raise SawattnError(rc, attn_last_error())


def _in_dtype_code(dtype) -> int:
    return {"f16": F16, "bf16": BF16}.get(dtype, _DTYPE_CODE.get(dtype, dtype))


def attn_fwd_launch_info(B: int, H: int, N: int, d: int, causal: bool = False, scan_order="sawtooth",
                         dtype="f16") -> dict:
    """Launch geometry of attn_fwd."""
    info = LaunchInfo()
    _check(lib().attn_fwd_launch_info(B, H, N, d, int(bool(causal)), _SCAN_CODE[scan_order], _in_dtype_code(dtype),
                                      ctypes.byref(info)))
    return info.as_dict()


def attn_fwd_variant_launch_info(B: int, H: int, N: int, d: int, causal: bool = False, variant: Variant = None,
                                 dtype="f16") -> dict:
    """Launch geometry of attn_fwd_variant (variant None: the default, as attn_fwd_launch_info)."""
    info = LaunchInfo()
    _check(lib().attn_fwd_variant_launch_info(B, H, N, d, int(bool(causal)), _in_dtype_code(dtype), _vptr(variant),
                                              ctypes.byref(info)))
    return info.as_dict()


def attn_fwd_plan(B: int, H: int, N: int, d: int, causal: bool = False, scan_order="sawtooth",
                  variant: Variant = None, dtype="f16"):
    """Host-side schedule: returns (trace[grid, max_local, 4], count[grid]) as CPU int32 tensors."""
    info = attn_fwd_variant_launch_info(B, H, N, d, causal, variant, dtype)
    trace = torch.full((info["grid"], max(info["max_local_tiles"], 1), 4), -1, dtype=torch.int32)
    count = torch.zeros((info["grid"],), dtype=torch.int32)
    _check(lib().attn_fwd_plan(B, H, N, d, int(bool(causal)), _SCAN_CODE[scan_order], _in_dtype_code(dtype),
                               _vptr(variant), trace.data_ptr(), count.data_ptr()))
    return trace, count


def attn_fwd_workspace_bytes(B: int, H: int, N: int, d: int, causal: bool = False, variant: Variant = None,
                             dtype="bf16"):
    """(bytes of workspace attn_fwd_workspace would use -- 0 where it changes nothing --, launch geometry)."""
    n = ctypes.c_size_t(0)
    info = LaunchInfo()
    _check(lib().attn_fwd_workspace_bytes(B, H, N, d, int(bool(causal)), _in_dtype_code(dtype), _vptr(variant),
                                          ctypes.byref(n), ctypes.byref(info)))
    return int(n.value), info.as_dict()


def sawattn_mfma_probe(iters: int, mode: int, stream=None) -> float:
    """Enqueue the matrix-rate probe on the current (or given) stream; returns its flop count."""
    sink = torch.zeros(512, dtype=torch.float32, device="cuda")
    flops = ctypes.c_double(0.0)
    st = stream if stream is not None else torch.cuda.current_stream()
    L = probe_lib()
    rc = L.sawattn_mfma_probe(sink.data_ptr(), int(iters), int(mode), st.cuda_stream, ctypes.byref(flops))
    if rc != OK:
        raise SawattnError(rc, L.sawattn_probe_last_error().decode())
    return float(flops.value)


def _refuse(Q, K, V):
    """Raise what is wrong with Q, K, V (called once the checks of _marshal have found that something is)."""
    for name, t in (("Q", Q), ("K", K), ("V", V)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous [B, H, N, d] device tensor")
    if not (Q.shape == K.shape == V.shape) or not (Q.dtype == K.dtype == V.dtype):
        raise ValueError("Q, K, V must share shape and dtype")
    raise ValueError("inputs must be float16 or bfloat16")


# One attn_fwd of a short head takes about as long on the host as on the GPU (5 to 6 us), so the calls below look each
# attribute up once, raise from a function of its own, and take the stream as the number it is.  One head of
# 256 x 64 called in a row: 8.4 -> 6.7 us.
def _marshal(Q, K, V, O, o_dtype):
    """(O, shape of all four tensors, code of the input type, code of the output type)"""
    shape, dtype = Q.shape, Q.dtype
    if not (Q.is_cuda and K.is_cuda and V.is_cuda and Q.is_contiguous() and K.is_contiguous() and V.is_contiguous()
            and len(shape) == 4 and shape == K.shape and shape == V.shape and dtype == K.dtype and dtype == V.dtype
            and dtype in _IN_DTYPE_CODE):
        _refuse(Q, K, V)
    if O is None:
        O = torch.empty(shape, dtype=o_dtype or dtype, device=Q.device)
        out = _DTYPE_CODE[O.dtype]
    else:
        out = _DTYPE_CODE.get(O.dtype)
        if out is None or not O.is_cuda or not O.is_contiguous() or O.shape != shape:
            raise ValueError("O must be a contiguous device tensor shaped like Q (f16, bf16 or f32)")
    return O, shape, _IN_DTYPE_CODE[dtype], out


def _stream(Q, stream):
    """Handle of the given stream, or of the current one of Q's device."""
    return stream.cuda_stream if stream is not None else _current_raw_stream(Q.get_device())


def attn_fwd(Q, K, V, O=None, *, scale: float, causal: bool = False, scan_order="sawtooth",
             o_dtype=None, stream=None):
    """O = softmax(Q K^T * scale) V on the current (or given) stream; returns O without waiting."""
    O, (B, H, N, d), i_code, o_code = _marshal(Q, K, V, O, o_dtype)
    rc = (_lib or lib()).attn_fwd(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), B, H, N, d, float(scale),
                                  1 if causal else 0, _SCAN_CODE[scan_order], i_code, o_code, _stream(Q, stream))
    if rc != OK:
        _check(rc)
    return O


def attn_fwd_variant(Q, K, V, O=None, *, scale: float, causal: bool = False, scan_order="sawtooth",
                     o_dtype=None, stream=None, variant: Variant = None, trace: bool = False):
    """attn_fwd under a launch variant.  Returns O, or with trace=True (O, trace[grid, max_local, 4],
    count[grid]): the schedule the workgroups recorded."""
    O, (B, H, N, d), i_code, o_code = _marshal(Q, K, V, O, o_dtype)
    tr = cnt = None
    if trace:
        info = attn_fwd_variant_launch_info(B, H, N, d, causal, variant, Q.dtype)
        tr = torch.full((info["grid"], max(info["max_local_tiles"], 1), 4), -1, dtype=torch.int32,
                        device=Q.device)
        cnt = torch.zeros((info["grid"],), dtype=torch.int32, device=Q.device)
    _check(lib().attn_fwd_variant(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), B, H, N, d,
                                  float(scale), int(bool(causal)), _SCAN_CODE[scan_order],
                                  i_code, o_code, _stream(Q, stream), _vptr(variant),
                                  tr.data_ptr() if trace else None, cnt.data_ptr() if trace else None))
    return (O, tr, cnt) if trace else O


def attn_fwd_workspace(Q, K, V, O=None, *, scale: float, causal: bool = False, scan_order="sawtooth",
                       o_dtype=None, stream=None, variant: Variant = None, trace: bool = False, workspace=None):
    """attn_fwd_variant with a workspace (a uint8 CUDA tensor of at least attn_fwd_workspace_bytes bytes; allocated
    here when None and needed).  Returns like attn_fwd_variant."""
    O, (B, H, N, d), i_code, o_code = _marshal(Q, K, V, O, o_dtype)
    need, info = attn_fwd_workspace_bytes(B, H, N, d, causal, variant, Q.dtype)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
    tr = cnt = None
    if trace:
        tr = torch.full((info["grid"], max(info["max_local_tiles"], 1), 4), -1, dtype=torch.int32,
                        device=Q.device)
        cnt = torch.zeros((info["grid"],), dtype=torch.int32, device=Q.device)
    _check(lib().attn_fwd_workspace(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), B, H, N, d,
                                    float(scale), int(bool(causal)), _SCAN_CODE[scan_order],
                                    i_code, o_code, _stream(Q, stream), _vptr(variant),
                                    tr.data_ptr() if trace else None, cnt.data_ptr() if trace else None,
                                    workspace.data_ptr() if workspace is not None else None,
                                    workspace.numel() if workspace is not None else 0))
    return (O, tr, cnt) if trace else O


def attn_fwd_static(Q, K, V, O=None, *, scale: float, causal: bool = False, scan_order="sawtooth", o_dtype=None,
                    stream=None):
    """attn_fwd with the library's fixed scratch array standing in for a workspace (the C call allocates nothing;
    pass O to keep this wrapper from allocating the output)."""
    O, (B, H, N, d), i_code, o_code = _marshal(Q, K, V, O, o_dtype)
    _check(lib().attn_fwd_static(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), B, H, N, d,
                                 float(scale), int(bool(causal)), _SCAN_CODE[scan_order],
                                 i_code, o_code, _stream(Q, stream)))
    return O


# ---- decoding over a paged key-value cache

REQUEST_ENDS = -1        # in new_tokens of attn_kv_pages: the request's pages go back to the free list


class _CacheStruct(ctypes.Structure):
    """sawattn_kv_cache"""
    _fields_ = ([("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]
                + [(n, ctypes.c_int64) for n in ("k_page", "k_head", "k_row", "v_page", "v_head", "v_row")]
                + [(n, ctypes.c_int) for n in ("pages", "page_size", "heads", "d", "dtype")])


class KVCache:
    """The keys and values of one layer in pages: two device tensors [pages, heads, page_size, d] of any strides whose last
    dimension is contiguous ([pages, page_size, heads, d] as its .transpose(1, 2)).  Made once, kept with the tensors; their
    storage must not be replaced."""

    def __init__(self, k, v):
        for name, t in (("k", k), ("v", v)):
            if not t.is_cuda or t.dim() != 4 or t.stride(3) != 1:
                raise ValueError(f"{name} must be a [pages, heads, page_size, d] device tensor, contiguous in its last dimension")
        if k.shape != v.shape or k.dtype != v.dtype or k.device != v.device:
            raise ValueError("k and v must share shape, dtype and device")
        if k.dtype not in _IN_DTYPE_CODE:
            raise ValueError("a cache must be float16 or bfloat16")
        if max(k.shape) > 2 ** 31 - 1:
            raise ValueError("a cache must have fewer than 2^31 pages, heads and rows per page")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.get_device()
        self.pages, self.heads, self.page_size, self.d = k.shape
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], self.pages, self.page_size,
                                    self.heads, self.d, _IN_DTYPE_CODE[k.dtype])
        self.ptr = ctypes.addressof(self._struct)


_paged = None


def _paged_module():
    """The module that looks at tensors and calls the library for the three operators below (built with the library), bound to it."""
    global _paged
    if _paged is None:
        if not os.path.exists(PAGED_BINDING_PATH):
            raise FileNotFoundError(f"{PAGED_BINDING_PATH} is not built; run `python -m paper_2601_16032_amd.build` first")
        L = lib()
        from . import _paged as module
        module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.attn_kv_pages, L.attn_qkv_prepare, L.attn_decode, L.hipGetDevice, L.hipSetDevice)))      # (the last two of the HIP runtime it loads)
        _paged = module
    return _paged


def _stream_on(device, stream):
    """Handle of the given stream, or of the device's current one."""
    if device < 0:
        raise ValueError("the first tensor must be a device tensor")
    if stream is None:
        return _current_raw_stream(device)
    if stream.device.index != device:
        raise ValueError("the stream must be one of the tensors' device")
    return stream.cuda_stream


def _empty(shape, dtype, device, stream):
    """A new tensor out of the memory of the stream that uses it first: memory of the current stream may still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class PageStep(NamedTuple):
    """What attn_kv_pages writes."""
    lengths: torch.Tensor         # int32 [R]
    granted: torch.Tensor         # int32 [R]
    token_offsets: torch.Tensor   # int32 [R + 1]
    free_state: torch.Tensor      # int32 [2]
    slots: torch.Tensor           # int64 [tokens]
    positions: torch.Tensor       # int32 [tokens]


def attn_kv_pages(lengths, new_tokens, table, free_pages, free_state, *, page_size: int, tokens: int = None, lengths_out=None,
                  granted=None, token_offsets=None, free_state_out=None, slots=None, positions=None, stream=None) -> PageStep:
    """Pages, slots and positions of the tokens that `new_tokens` adds to requests of `lengths`; `table` and the ring `free_pages` are
    brought up to date in place, the rest is written to the tensors given or to new ones (`tokens` rows where no slots are given)."""
    if slots is None:
        if tokens is None:
            raise ValueError("either slots or the number of tokens must be given")
        slots = _empty(tokens, torch.int64, lengths.device, stream)
    elif tokens is not None and tokens != slots.numel():
        raise ValueError("slots must hold as many elements as there are tokens")
    if lengths_out is None or granted is None or token_offsets is None or free_state_out is None or positions is None:
        R = lengths.numel()
        lengths_out, granted, token_offsets, free_state_out, positions = (
            _empty(size, torch.int32, lengths.device, stream) if t is None else t for t, size in (
                (lengths_out, R), (granted, R), (token_offsets, R + 1), (free_state_out, 2), (positions, slots.numel())))
    rc = (_paged or _paged_module()).kv_pages(lengths, new_tokens, table, free_pages, free_state, lengths_out, granted, token_offsets,
                                              free_state_out, slots, positions, page_size, _stream_on(lengths.get_device(), stream))
    if rc != OK:
        _check(rc)
    return PageStep(lengths_out, granted, token_offsets, free_state_out, slots, positions)


def attn_qkv_prepare(q, k, v, *, positions, frequencies=None, interleaved: bool = False, q_weight=None, k_weight=None,
                     eps: float = 1e-6, q_out=None, k_out=None, v_out=None, cache: KVCache = None, slots=None, stream=None):
    """Norms of the heads of Q and K (where a weight is given) and rotation of their first 2 * len(frequencies) elements, K and V
    written to `slots` of the cache and / or to k_out and v_out.  q, k, v: [B, N, heads, d] or [N, heads, d], of any strides.
    Returns (q_out, k_out, v_out); q_out is made where it is not given, k_out and v_out where there is no cache either.  A token of negative
    position is padding: its rows of the outputs are left as they are, in those made here whatever the memory held."""
    if (cache is None) != (slots is None) or (k_out is None) != (v_out is None):
        raise ValueError("cache and slots, and k_out and v_out, must be given together")
    if q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    if cache is None:
        ptr, at = None, -1
        if k_out is None:
            k_out, v_out = _empty(k.shape, k.dtype, q.device, stream), _empty(k.shape, k.dtype, q.device, stream)
    else:
        ptr, at = cache.ptr, cache.device
    rc = (_paged or _paged_module()).qkv_prepare(q, k, v, q_out, k_out, v_out, ptr, at, slots, positions, q_weight, k_weight, eps, frequencies,
                                                 interleaved, _stream_on(q.get_device(), stream))
    if rc != OK:
        _check(rc)
    return q_out, k_out, v_out


def attn_decode_workspace_bytes(R: int, H: int, cache: KVCache, max_pages: int) -> int:
    """Bytes of workspace attn_decode needs for R requests of H heads, or fewer requests, and page tables of max_pages entries, or fewer."""
    n = ctypes.c_size_t(0)
    _check(lib().attn_decode_workspace_bytes(cache.ptr, R, H, max_pages, ctypes.byref(n)))
    return int(n.value)


def attn_decode(Q, cache: KVCache, table, lengths, O=None, *, scale: float, window: int = 0, o_dtype=None, workspace=None,
                stream=None):
    """O[r, h] = softmax(q . K^T * scale) V of one token per request, Q [R, H, d], over the last `window` (0: all) of the lengths[r]
    cached rows that table[r] names the pages of.  workspace: a uint8 tensor of at least attn_decode_workspace_bytes bytes, made
    here when None.  Returns O without waiting."""
    if O is None:
        O = _empty(Q.shape, o_dtype or Q.dtype, Q.device, stream)
    if workspace is None:
        workspace = _empty(attn_decode_workspace_bytes(Q.shape[0], Q.shape[1], cache, table.shape[-1]), torch.uint8, Q.device, stream)
    device = cache.device
    rc = (_paged or _paged_module()).decode(Q, O, cache.ptr, device, table, lengths, scale, window, workspace, _stream_on(device, stream))
    if rc != OK:
        _check(rc)
    return O
