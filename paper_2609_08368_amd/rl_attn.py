"""Thin ctypes binding over librlattn.so (argument marshalling only).

Every step of the attention runs in the HIP library; this module turns torch
tensors into the ABI's non-owning ``rl_tensor`` views and passes torch's
current stream. There is no fallback: if the library is missing or a call
fails, an exception is raised.
"""

from __future__ import annotations

import ctypes
import os
import re
import warnings
from typing import NamedTuple, Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# RL_ATTN_LIB selects another build of the library (A/B comparisons of builds)
LIB_PATH = os.environ.get("RL_ATTN_LIB", os.path.join(_PKG, "librlattn.so"))
INCLUDE = os.path.join(os.path.dirname(_PKG), "include")
HEADER = os.path.join(INCLUDE, "rl_attn.h")

RL_BF16, RL_F32, RL_I32, RL_FP8_E4M3, RL_I64 = 1, 2, 3, 4, 5
RL_PREFIX_AUTO, RL_PREFIX_OFF = 0, 1
STATUS = {
    0: "RL_OK", -1: "RL_ERR_INVALID_ARG", -2: "RL_ERR_SHAPE", -3: "RL_ERR_DTYPE", -4: "RL_ERR_UNSUPPORTED",
    -5: "RL_ERR_WORKSPACE", -6: "RL_ERR_HIP", -7: "RL_ERR_DEVICE",
}
CODES = {v: k for k, v in STATUS.items()}


class RlTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 4), ("strides", ctypes.c_int64 * 4)]


class RlOpts(ctypes.Structure):
    _fields_ = [("split_tokens", ctypes.c_int32), ("prefix_share", ctypes.c_int32),
                ("validate", ctypes.c_int32), ("deterministic", ctypes.c_int32), ("reserved", ctypes.c_int32 * 4)]


class RlRopeOpts(ctypes.Structure):
    _fields_ = [("interleaved", ctypes.c_int32), ("inverse", ctypes.c_int32), ("reserved", ctypes.c_int32 * 6)]


class RlAttnError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS.get(code, code)}: {message}")
        self.code = code
        self.status = STATUS.get(code, str(code))


_lib = None


def lib() -> ctypes.CDLL:
    """Load librlattn.so (built by ``python -m paper_2609_08368_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
        L = ctypes.CDLL(LIB_PATH)
        vp = ctypes.c_void_p
        P = vp                                  # rl_tensor: the bytes of one (_arg), or a reference to one
        L.rl_attn_decode.argtypes = [P, P, P, P, P, ctypes.c_float, P, vp]
        L.rl_attn_extend.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, vp]
        L.rl_attn_decode_ex.argtypes = [P, P, P, P, P, ctypes.c_float, P, P, ctypes.POINTER(RlOpts), vp]
        L.rl_attn_extend_ex.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, P, ctypes.POINTER(RlOpts), vp]
        L.rl_attn_decode_noalloc.argtypes = [P, P, P, P, P, ctypes.c_float, P, P, ctypes.POINTER(RlOpts), vp]
        L.rl_attn_decode_fp8.argtypes = [P, P, P, P, P, P, P, ctypes.c_float, P, P, ctypes.POINTER(RlOpts), vp]
        L.rl_attn_extend_fp8.argtypes = [P, P, P, P, P, P, P, P, ctypes.c_float, P, P, ctypes.POINTER(RlOpts), vp]
        L.rl_attn_append_kv.argtypes = [P, P, P, P, P, P, P, vp]
        L.rl_attn_append_kv_fp8.argtypes = [P, P, P, P, P, P, P, P, P, vp]
        L.rl_attn_map_slots.argtypes = [P, P, P, P, P, ctypes.c_int64, ctypes.c_int64, P, P, P, P, P, P, vp]
        R = ctypes.POINTER(RlRopeOpts)
        L.rl_attn_rope.argtypes = [P, P, P, P, P, R, P, P, vp]
        L.rl_attn_rope_append_kv.argtypes = [P, P, P, P, P, P, R, P, P, P, P, P, vp]
        L.rl_attn_rope_append_kv_fp8.argtypes = [P, P, P, P, P, P, R, P, P, P, P, P, P, P, vp]
        F = ctypes.c_float
        L.rl_attn_norm_rope.argtypes = [P, P, P, P, F, P, P, P, R, P, P, vp]
        L.rl_attn_norm_rope_append_kv.argtypes = [P, P, P, P, P, F, P, P, P, R, P, P, P, P, P, vp]
        L.rl_attn_norm_rope_append_kv_fp8.argtypes = [P, P, P, P, P, F, P, P, P, R, P, P, P, P, P, P, P, vp]
        L.rl_attn_norm_rope_backward.argtypes = [P, P, P, P, P, P, F, P, P, P, R, P, P, P, P, vp]
        L.rl_attn_norm_rope_backward_workspace_size.argtypes = []
        L.rl_attn_norm_rope_backward_workspace_size.restype = ctypes.c_size_t
        L.rl_attn_token_logprobs.argtypes = [P] * 8 + [vp]
        L.rl_attn_token_logprobs_backward.argtypes = [P] * 8 + [vp]
        L.rl_attn_token_logprobs_workspace_size.argtypes = [ctypes.c_int64] * 3
        L.rl_attn_token_logprobs_workspace_size.restype = ctypes.c_size_t
        L.rl_attn_fork_requests.argtypes = [P, P, P, P, P, ctypes.c_int64, ctypes.c_int64, P, P, P, P, vp]
        L.rl_attn_copy_pages.argtypes = [P, P, P, vp]
        L.rl_attn_drop_tokens.argtypes = [P, P, P, ctypes.c_int64, ctypes.c_int64, P, P, P, P, vp]
        L.rl_attn_prefill.argtypes = [P, P, P, P, ctypes.c_float, P, P, vp]
        L.rl_attn_merge.argtypes = [P, P, P, P, P, vp]
        L.rl_attn_last_error.restype = ctypes.c_char_p
        L.rl_attn_check_device_errors.argtypes = [vp]
        L.rl_attn_reserve_workspace.argtypes = [ctypes.c_size_t, vp]
        L.rl_attn_decode_workspace_size.argtypes = [ctypes.c_int64] * 6 + [ctypes.c_int32]
        L.rl_attn_decode_workspace_size.restype = ctypes.c_size_t
        L.rl_attn_extend_workspace_size.argtypes = [ctypes.c_int64] * 6
        L.rl_attn_extend_workspace_size.restype = ctypes.c_size_t
        L.rl_attn_release.restype = None
        L.rl_attn_profile_enable.argtypes = [ctypes.c_int]
        L.rl_attn_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_double)]
        dp = ctypes.POINTER(ctypes.c_double)
        L.rl_attn_diag_read_bandwidth.argtypes = [vp, ctypes.c_int64, ctypes.c_int32, dp, vp]
        L.rl_attn_diag_mfma_bf16.argtypes = [ctypes.c_int64, dp, vp]
        i64p = ctypes.POINTER(ctypes.c_int64)
        L.rl_attn_diag_decode_capacity.argtypes = [ctypes.c_int64] * 6 + [ctypes.c_int32] * 4 + [i64p]
        L.rl_attn_diag_extend_capacity.argtypes = [ctypes.c_int64] * 4 + [i64p]
        L.rl_attn_diag_extend_plan.argtypes = [vp, vp] + [ctypes.c_int64] * 6 + [ctypes.c_int32, i64p]
        for name in ("rl_attn_decode", "rl_attn_extend", "rl_attn_decode_ex", "rl_attn_extend_ex",
                     "rl_attn_decode_noalloc",
                     "rl_attn_decode_fp8", "rl_attn_extend_fp8", "rl_attn_append_kv", "rl_attn_append_kv_fp8",
                     "rl_attn_map_slots", "rl_attn_rope", "rl_attn_rope_append_kv", "rl_attn_rope_append_kv_fp8",
                     "rl_attn_norm_rope", "rl_attn_norm_rope_append_kv", "rl_attn_norm_rope_append_kv_fp8",
                     "rl_attn_norm_rope_backward", "rl_attn_token_logprobs", "rl_attn_token_logprobs_backward",
                     "rl_attn_fork_requests", "rl_attn_copy_pages", "rl_attn_drop_tokens",
                     "rl_attn_prefill", "rl_attn_merge", "rl_attn_check_device_errors", "rl_attn_reserve_workspace",
                     "rl_attn_profile_enable", "rl_attn_profile_read", "rl_attn_diag_read_bandwidth",
                     "rl_attn_diag_mfma_bf16", "rl_attn_diag_decode_capacity", "rl_attn_diag_extend_capacity",
                     "rl_attn_diag_extend_plan"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def header_functions() -> list:
    """Names of the functions the headers under ``include/`` declare."""
    names = set()
    for fn in sorted(os.listdir(INCLUDE)):
        if fn.endswith(".h"):
            with open(os.path.join(INCLUDE, fn)) as f:
                text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
            names.update(re.findall(r"\b(rl_attn_\w+)\s*\(", text))
    return sorted(names)


def last_error() -> str:
    return lib().rl_attn_last_error().decode()


def _check(rc: int):
    if rc != 0:
        raise RlAttnError(rc, last_error())


# (the functions behind torch.cuda.current_device() and current_stream(), without what those do besides: 3 us of a
# call whose kernel takes 5)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda device: torch.cuda.current_stream(device).cuda_stream)

_DTYPES = {torch.bfloat16: RL_BF16, torch.float32: RL_F32, torch.int32: RL_I32, torch.int64: RL_I64,
           torch.float8_e4m3fn: RL_FP8_E4M3}
_PACK_PATH = os.path.join(_PKG, "_pack.so")


def _describe(t):
    """The bytes of an rl_tensor describing a tensor (no copy of its data); None -> NULL. The library dereferences the
    pointers on the current HIP device, so a tensor elsewhere is a ValueError (a host pointer would reach a kernel)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"expected a tensor or None, got {type(t).__name__}")
    if not t.is_cuda or t.device.index != _current_device():
        raise ValueError(f"tensor on {t.device}: the library reads and writes tensors on the current device")
    if t.dim() > 4:
        raise ValueError("rl_tensor holds at most 4 dimensions")
    v = RlTensor()
    v.data, v.dtype, v.ndim = t.data_ptr() or None, _DTYPES.get(t.dtype, 0), t.dim()
    v.shape[:v.ndim], v.strides[:v.ndim] = t.shape, t.stride()
    return bytes(v)


def _first_arg(t):
    """`_describe` by the compiled module, from the first call that finds it on (0.1 us a tensor instead of 3); without
    one that loads here (not built, or for another Python or torch) calls work all the same."""
    global _arg
    if os.path.exists(_PACK_PATH):
        try:
            from ._pack import arg as _arg
        except ImportError as e:
            warnings.warn(f"{_PACK_PATH} does not load, tensors are described in Python (slower): {e}", RuntimeWarning,
                          stacklevel=3)
            _arg = _describe
        return _arg(t)
    return _describe(t)


_arg = _first_arg


def view(t: Optional[torch.Tensor]):
    """An ``rl_tensor`` describing ``t`` (no copy); None -> NULL."""
    return None if t is None else RlTensor.from_buffer_copy(_arg(t))


def _stream(stream) -> Optional[int]:
    if stream is None:
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return _current_stream(_current_device())
    return getattr(stream, "cuda_stream", stream)


def _opts(split_tokens=0, prefix_share=True, validate=False, deterministic=False):
    o = RlOpts()
    o.split_tokens = int(split_tokens)
    o.prefix_share = RL_PREFIX_AUTO if prefix_share else RL_PREFIX_OFF
    o.validate = int(bool(validate))
    o.deterministic = int(bool(deterministic))
    return o


def decode(q, k_pages, v_pages, block_table, seq_lens, scale, out=None, lse=None, *, split_tokens=0,
           prefix_share=True, validate=False, deterministic=False, stream=None):
    """``rl_attn_decode_ex``: returns ``out`` (and fills ``lse`` if given)."""
    if out is None:
        out = torch.empty_like(q)
    o = _opts(split_tokens, prefix_share, validate, deterministic)
    _check(lib().rl_attn_decode_ex(_arg(q), _arg(k_pages), _arg(v_pages), _arg(block_table), _arg(seq_lens),
                                   ctypes.c_float(scale), _arg(out), _arg(lse), ctypes.byref(o),
                                   _stream(stream)))
    return out


def decode_noalloc(q, k_pages, v_pages, block_table, seq_lens, scale, out=None, lse=None, *, split_tokens=0,
                   prefix_share=True, deterministic=False, stream=None):
    """``rl_attn_decode_noalloc``: decode with the library's static scratch array as workspace
    (``out`` must be given by a caller that cannot allocate)."""
    if out is None:
        out = torch.empty_like(q)
    o = _opts(split_tokens, prefix_share, False, deterministic)
    _check(lib().rl_attn_decode_noalloc(_arg(q), _arg(k_pages), _arg(v_pages), _arg(block_table),
                                        _arg(seq_lens), ctypes.c_float(scale), _arg(out), _arg(lse),
                                        ctypes.byref(o), _stream(stream)))
    return out


def decode_plain(q, k_pages, v_pages, block_table, seq_lens, scale, out=None, stream=None):
    """``rl_attn_decode`` (the fixed signature, no options)."""
    if out is None:
        out = torch.empty_like(q)
    _check(lib().rl_attn_decode(_arg(q), _arg(k_pages), _arg(v_pages), _arg(block_table), _arg(seq_lens),
                                ctypes.c_float(scale), _arg(out), _stream(stream)))
    return out


def extend(q, qo_indptr, k_pages, v_pages, block_table, kv_lens, scale, out=None, lse=None, *,
           validate=False, stream=None):
    """``rl_attn_extend_ex``: returns ``out`` (and fills ``lse`` if given)."""
    if out is None:
        out = torch.empty_like(q)
    o = _opts(0, True, validate)
    _check(lib().rl_attn_extend_ex(_arg(q), _arg(qo_indptr), _arg(k_pages), _arg(v_pages), _arg(block_table),
                                   _arg(kv_lens), ctypes.c_float(scale), _arg(out), _arg(lse), ctypes.byref(o),
                                   _stream(stream)))
    return out


def extend_plain(q, qo_indptr, k_pages, v_pages, block_table, kv_lens, scale, out=None, stream=None):
    """``rl_attn_extend`` (the fixed signature)."""
    if out is None:
        out = torch.empty_like(q)
    _check(lib().rl_attn_extend(_arg(q), _arg(qo_indptr), _arg(k_pages), _arg(v_pages), _arg(block_table),
                                _arg(kv_lens), ctypes.c_float(scale), _arg(out), _stream(stream)))
    return out


def decode_fp8(q, k_pages, v_pages, k_scale, v_scale, block_table, seq_lens, scale, out=None, lse=None, *,
               split_tokens=0, prefix_share=True, validate=False, deterministic=False, stream=None):
    """``rl_attn_decode_fp8``: pages are ``torch.float8_e4m3fn``, scales ``[Hkv]`` float32."""
    if out is None:
        out = torch.empty_like(q)
    o = _opts(split_tokens, prefix_share, validate, deterministic)
    _check(lib().rl_attn_decode_fp8(_arg(q), _arg(k_pages), _arg(v_pages), _arg(k_scale), _arg(v_scale),
                                    _arg(block_table), _arg(seq_lens), ctypes.c_float(scale), _arg(out),
                                    _arg(lse), ctypes.byref(o), _stream(stream)))
    return out


def extend_fp8(q, qo_indptr, k_pages, v_pages, k_scale, v_scale, block_table, kv_lens, scale, out=None, lse=None,
               *, validate=False, stream=None):
    """``rl_attn_extend_fp8``: pages are ``torch.float8_e4m3fn``, scales ``[Hkv]`` float32."""
    if out is None:
        out = torch.empty_like(q)
    o = _opts(0, True, validate)
    _check(lib().rl_attn_extend_fp8(_arg(q), _arg(qo_indptr), _arg(k_pages), _arg(v_pages), _arg(k_scale),
                                    _arg(v_scale), _arg(block_table), _arg(kv_lens), ctypes.c_float(scale),
                                    _arg(out), _arg(lse), ctypes.byref(o), _stream(stream)))
    return out


def append_kv(k_new, v_new, qo_indptr, block_table, kv_lens, k_pages, v_pages, stream=None):
    """``rl_attn_append_kv``: writes the new rows into ``k_pages``/``v_pages`` (in place)."""
    _check(lib().rl_attn_append_kv(_arg(k_new), _arg(v_new), _arg(qo_indptr), _arg(block_table), _arg(kv_lens),
                                   _arg(k_pages), _arg(v_pages), _stream(stream)))


def append_kv_fp8(k_new, v_new, qo_indptr, block_table, kv_lens, k_pages, v_pages, k_scale, v_scale, stream=None):
    """``rl_attn_append_kv_fp8``: bf16 rows quantised into ``torch.float8_e4m3fn`` pages (in place)."""
    _check(lib().rl_attn_append_kv_fp8(_arg(k_new), _arg(v_new), _arg(qo_indptr), _arg(block_table),
                                       _arg(kv_lens), _arg(k_pages), _arg(v_pages), _arg(k_scale),
                                       _arg(v_scale), _stream(stream)))


class SlotMap(NamedTuple):
    """What ``map_slots`` gives for a step (the block table is written in place)."""

    qo_indptr: torch.Tensor
    slot_map: torch.Tensor
    positions: torch.Tensor
    kv_lens: torch.Tensor
    free_used: torch.Tensor


def map_slots(kv_lens, new_lens, free_pages, free_used, block_table, page_size, num_pages, rows=None, *,
              pos_delta=None, kv_lens_out=None, free_used_out=None, qo_indptr=None, slot_map=None, positions=None,
              stream=None) -> SlotMap:
    """``rl_attn_map_slots``: ``rows`` is the length of a ``slot_map`` and ``positions`` that are not given.

    ``kv_lens_out=kv_lens, free_used_out=free_used`` advances a step in place."""
    dev = kv_lens.device
    if slot_map is None:
        if rows is None:
            raise ValueError("rows is needed where slot_map is not given")
        slot_map = torch.empty(rows, dtype=torch.int64, device=dev)
    if positions is None:
        positions = torch.empty(slot_map.shape[0], dtype=torch.int32, device=dev)
    if qo_indptr is None:
        qo_indptr = torch.empty(kv_lens.shape[0] + 1, dtype=torch.int32, device=dev)
    if kv_lens_out is None:
        kv_lens_out = torch.empty_like(kv_lens)
    if free_used_out is None:
        free_used_out = torch.empty_like(free_used)
    _check(lib().rl_attn_map_slots(_arg(kv_lens), _arg(new_lens), _arg(free_pages), _arg(free_used),
                                   _arg(pos_delta), page_size, num_pages, _arg(block_table), _arg(kv_lens_out),
                                   _arg(free_used_out), _arg(qo_indptr), _arg(slot_map), _arg(positions),
                                   _stream(stream)))
    return SlotMap(qo_indptr, slot_map, positions, kv_lens_out, free_used_out)


_ROPE_OPTS = {(i, b): RlRopeOpts(interleaved=i, inverse=b) for i in (0, 1) for b in (0, 1)}


def _rope_opts(interleaved, inverse=False):
    return ctypes.byref(_ROPE_OPTS[bool(interleaved), bool(inverse)])


def rope(q, k, positions, inv_freq, axes=None, *, interleaved=False, inverse=False, q_out=None, k_out=None,
         stream=None):
    """``rl_attn_rope``: returns ``(q_out, k_out)`` (``k`` may be None). ``q_out=q, k_out=k`` rotates in place."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k_out is None and k is not None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    _check(lib().rl_attn_rope(_arg(q), _arg(k), _arg(positions), _arg(inv_freq), _arg(axes),
                              _rope_opts(interleaved, inverse), _arg(q_out), _arg(k_out), _stream(stream)))
    return q_out, k_out


def rope_append_kv(q, k_new, v_new, positions, inv_freq, slot_map, k_pages, v_pages, axes=None, *, interleaved=False,
                   q_out=None, k_out=None, stream=None):
    """``rl_attn_rope_append_kv``: returns ``q_out``; ``k_out`` (rows of rotated keys) is written only if given."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _check(lib().rl_attn_rope_append_kv(_arg(q), _arg(k_new), _arg(v_new), _arg(positions), _arg(inv_freq),
                                        _arg(axes), _rope_opts(interleaved), _arg(slot_map), _arg(q_out),
                                        _arg(k_out), _arg(k_pages), _arg(v_pages), _stream(stream)))
    return q_out


def rope_append_kv_fp8(q, k_new, v_new, positions, inv_freq, slot_map, k_pages, v_pages, k_scale, v_scale, axes=None,
                       *, interleaved=False, q_out=None, k_out=None, stream=None):
    """``rl_attn_rope_append_kv_fp8``: as ``rope_append_kv`` into ``torch.float8_e4m3fn`` pages."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _check(lib().rl_attn_rope_append_kv_fp8(_arg(q), _arg(k_new), _arg(v_new), _arg(positions), _arg(inv_freq),
                                            _arg(axes), _rope_opts(interleaved), _arg(slot_map), _arg(q_out),
                                            _arg(k_out), _arg(k_pages), _arg(v_pages), _arg(k_scale),
                                            _arg(v_scale), _stream(stream)))
    return q_out


def norm_rope(q, k, q_weight, k_weight, eps, positions, inv_freq, axes=None, *, interleaved=False, q_out=None,
              k_out=None, stream=None):
    """``rl_attn_norm_rope``: returns ``(q_out, k_out)`` (``k`` and ``k_weight`` may be None)."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k_out is None and k is not None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    _check(lib().rl_attn_norm_rope(_arg(q), _arg(k), _arg(q_weight), _arg(k_weight), eps, _arg(positions),
                                   _arg(inv_freq), _arg(axes), _rope_opts(interleaved), _arg(q_out), _arg(k_out),
                                   _stream(stream)))
    return q_out, k_out


def norm_rope_append_kv(q, k_new, v_new, q_weight, k_weight, eps, positions, inv_freq, slot_map, k_pages, v_pages,
                        axes=None, *, interleaved=False, q_out=None, k_out=None, stream=None):
    """``rl_attn_norm_rope_append_kv``: returns ``q_out``; ``k_out`` (rows of keys) is written only if given."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _check(lib().rl_attn_norm_rope_append_kv(_arg(q), _arg(k_new), _arg(v_new), _arg(q_weight), _arg(k_weight), eps,
                                             _arg(positions), _arg(inv_freq), _arg(axes), _rope_opts(interleaved),
                                             _arg(slot_map), _arg(q_out), _arg(k_out), _arg(k_pages), _arg(v_pages),
                                             _stream(stream)))
    return q_out


def norm_rope_append_kv_fp8(q, k_new, v_new, q_weight, k_weight, eps, positions, inv_freq, slot_map, k_pages, v_pages,
                            k_scale, v_scale, axes=None, *, interleaved=False, q_out=None, k_out=None, stream=None):
    """``rl_attn_norm_rope_append_kv_fp8``: as ``norm_rope_append_kv`` into ``torch.float8_e4m3fn`` pages."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _check(lib().rl_attn_norm_rope_append_kv_fp8(
        _arg(q), _arg(k_new), _arg(v_new), _arg(q_weight), _arg(k_weight), eps, _arg(positions), _arg(inv_freq),
        _arg(axes), _rope_opts(interleaved), _arg(slot_map), _arg(q_out), _arg(k_out), _arg(k_pages), _arg(v_pages),
        _arg(k_scale), _arg(v_scale), _stream(stream)))
    return q_out


class NormRopeGrads(NamedTuple):
    """What ``norm_rope_backward`` gives (None for k where there is none)."""

    dq: torch.Tensor
    dk: Optional[torch.Tensor]
    dq_weight: torch.Tensor
    dk_weight: Optional[torch.Tensor]


def norm_rope_backward(dq_out, dk_out, q, k, q_weight, k_weight, eps, positions, inv_freq, axes=None, *,
                       interleaved=False, dq=None, dk=None, dq_weight=None, dk_weight=None,
                       stream=None) -> NormRopeGrads:
    """``rl_attn_norm_rope_backward``: gradients of ``norm_rope``. ``dq=dq_out, dk=dk_out`` works in place."""
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dq_weight is None:
        dq_weight = torch.empty(q_weight.shape, dtype=torch.float32, device=q.device)
    if k is not None:
        if dk is None:
            dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        if dk_weight is None:
            dk_weight = torch.empty(k_weight.shape, dtype=torch.float32, device=k.device)
    _check(lib().rl_attn_norm_rope_backward(_arg(dq_out), _arg(dk_out), _arg(q), _arg(k), _arg(q_weight),
                                            _arg(k_weight), eps, _arg(positions), _arg(inv_freq), _arg(axes),
                                            _rope_opts(interleaved), _arg(dq), _arg(dk), _arg(dq_weight),
                                            _arg(dk_weight), _stream(stream)))
    return NormRopeGrads(dq, dk, dq_weight, dk_weight)


def norm_rope_backward_workspace_size() -> int:
    return int(lib().rl_attn_norm_rope_backward_workspace_size())


class TokenLogprobs(NamedTuple):
    """What ``token_logprobs`` gives (None for alternatives that were not asked for)."""

    logprobs: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_ids: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


def token_logprobs(logits, tokens, row_scale=None, *, top=0, logprobs=None, entropy=None, lse=None, top_ids=None,
                   top_logprobs=None, stream=None) -> TokenLogprobs:
    """``rl_attn_token_logprobs``: ``top`` is the number of alternatives where ``top_ids`` is not given."""
    rows, dev = logits.shape[0], logits.device
    if logprobs is None:
        logprobs = torch.empty(rows, dtype=torch.float32, device=dev)
    if entropy is None:
        entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    if lse is None:
        lse = torch.empty(rows, dtype=torch.float32, device=dev)
    if top_ids is not None:
        top = top_ids.shape[-1]
    elif top_logprobs is not None:
        top = top_logprobs.shape[-1]
    if top_ids is None and top:
        top_ids = torch.empty((rows, top), dtype=torch.int32, device=dev)
    if top_logprobs is None and top_ids is not None:
        top_logprobs = torch.empty((rows, top), dtype=torch.float32, device=dev)
    _check(lib().rl_attn_token_logprobs(_arg(logits), _arg(tokens), _arg(row_scale), _arg(logprobs), _arg(entropy),
                                        _arg(lse), _arg(top_ids), _arg(top_logprobs), _stream(stream)))
    return TokenLogprobs(logprobs, entropy, lse, top_ids, top_logprobs)


def token_logprobs_backward(logits, tokens, lse, d_logprobs, row_scale=None, *, entropy=None, d_entropy=None,
                            d_logits=None, stream=None):
    """``rl_attn_token_logprobs_backward``: returns ``d_logits`` (``d_logits=logits`` works in place)."""
    if d_logits is None:
        d_logits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _check(lib().rl_attn_token_logprobs_backward(_arg(logits), _arg(tokens), _arg(row_scale), _arg(lse), _arg(entropy),
                                                 _arg(d_logprobs), _arg(d_entropy), _arg(d_logits),
                                                 _stream(stream)))
    return d_logits


def token_logprobs_workspace_size(rows: int, vocab: int, top: int = 0) -> int:
    return int(lib().rl_attn_token_logprobs_workspace_size(rows, vocab, top))


class Forked(NamedTuple):
    """What ``fork_requests`` gives (the block table is written in place)."""

    kv_lens: torch.Tensor
    free_used: torch.Tensor
    copies: torch.Tensor


def fork_requests(parents, fork_lens, kv_lens, free_pages, free_used, block_table, page_size, num_pages, *,
                  kv_lens_out=None, free_used_out=None, copies=None, stream=None) -> Forked:
    """``rl_attn_fork_requests``. ``kv_lens_out=kv_lens, free_used_out=free_used`` works in place."""
    if kv_lens_out is None:
        kv_lens_out = torch.empty_like(kv_lens)
    if free_used_out is None:
        free_used_out = torch.empty_like(free_used)
    if copies is None:
        copies = torch.empty((kv_lens.shape[0], 3), dtype=torch.int32, device=kv_lens.device)
    _check(lib().rl_attn_fork_requests(_arg(parents), _arg(fork_lens), _arg(kv_lens), _arg(free_pages),
                                       _arg(free_used), page_size, num_pages, _arg(block_table), _arg(kv_lens_out),
                                       _arg(free_used_out), _arg(copies), _stream(stream)))
    return Forked(kv_lens_out, free_used_out, copies)


def copy_pages(copies, k_pages, v_pages, *, stream=None):
    """``rl_attn_copy_pages``: the rows that a fork copies, in one layer's pages (in place)."""
    _check(lib().rl_attn_copy_pages(_arg(copies), _arg(k_pages), _arg(v_pages), _stream(stream)))


def drop_tokens(kv_lens, keep_lens, block_table, free_pages, free_used, page_size, num_pages, *, kv_lens_out=None,
                free_used_out=None, stream=None):
    """``rl_attn_drop_tokens``: writes ``free_pages``, returns ``(kv_lens_out, free_used_out)``.

    ``kv_lens_out=kv_lens, free_used_out=free_used`` works in place."""
    if kv_lens_out is None:
        kv_lens_out = torch.empty_like(kv_lens)
    if free_used_out is None:
        free_used_out = torch.empty_like(free_used)
    _check(lib().rl_attn_drop_tokens(_arg(kv_lens), _arg(keep_lens), _arg(block_table), page_size, num_pages,
                                     _arg(free_pages), _arg(free_used), _arg(kv_lens_out), _arg(free_used_out),
                                     _stream(stream)))
    return kv_lens_out, free_used_out


def prefill(q, k, v, seq_indptr, scale, out=None, lse=None, *, stream=None):
    """``rl_attn_prefill``: causal attention over packed prompts; returns ``out`` (and fills ``lse`` if given)."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _check(lib().rl_attn_prefill(_arg(q), _arg(k), _arg(v), _arg(seq_indptr), ctypes.c_float(scale), _arg(out),
                                 _arg(lse), _stream(stream)))
    return out


def merge(o_parts, lse_parts, num_parts, out=None, lse=None, stream=None):
    """``rl_attn_merge``: log-sum-exp merge of partial results."""
    n, _, h, d = o_parts.shape
    if out is None:
        out = torch.empty((n, h, d), dtype=torch.float32, device=o_parts.device)
    _check(lib().rl_attn_merge(_arg(o_parts), _arg(lse_parts), _arg(num_parts), _arg(out), _arg(lse),
                               _stream(stream)))
    return out


def check_device_errors(stream=None):
    _check(lib().rl_attn_check_device_errors(_stream(stream)))


def reserve_workspace(nbytes: int, stream=None):
    _check(lib().rl_attn_reserve_workspace(ctypes.c_size_t(nbytes), _stream(stream)))


def decode_workspace_size(batch: int, num_q_heads: int, num_kv_heads: int, max_pages: int, page_size: int,
                          query_tokens: int = 1, split_tokens: int = 0) -> int:
    """Workspace bytes a decode call may need (``query_tokens`` per sequence, the call's ``split_tokens``)."""
    return int(lib().rl_attn_decode_workspace_size(batch, num_q_heads, num_kv_heads, max_pages, page_size,
                                                   query_tokens, split_tokens))


def extend_workspace_size(batch: int, total_q: int, num_q_heads: int, num_kv_heads: int, max_pages: int,
                          page_size: int) -> int:
    return int(lib().rl_attn_extend_workspace_size(batch, total_q, num_q_heads, num_kv_heads, max_pages, page_size))


def profile_enable(on: bool = True):
    _check(lib().rl_attn_profile_enable(int(bool(on))))


def profile_read(kind: str):
    """(launches, mean ms) of the main kernel timed since the last read; kind 'decode', 'extend', 'append',
    'prefill' or 'rope'."""
    n = ctypes.c_int()
    ms = ctypes.c_double()
    _check(lib().rl_attn_profile_read({"decode": 0, "extend": 1, "append": 2, "prefill": 3, "rope": 4}[kind],
                                      ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


def release():
    lib().rl_attn_release()


def diag_read_bandwidth(buf: torch.Tensor, reps: int = 10, stream=None) -> float:
    """HBM read rate (GB/s) of streaming ``buf`` (a device tensor) ``reps`` times."""
    r = ctypes.c_double(0.0)
    _check(lib().rl_attn_diag_read_bandwidth(ctypes.c_void_p(buf.data_ptr()), buf.numel() * buf.element_size(),
                                             reps, ctypes.byref(r), _stream(stream)))
    return r.value


def diag_mfma_bf16(iters: int = 20000, stream=None) -> float:
    """TFLOP/s of a register-only bf16 MFMA loop on every CU."""
    t = ctypes.c_double(0.0)
    _check(lib().rl_attn_diag_mfma_bf16(iters, ctypes.byref(t), _stream(stream)))
    return t.value


def diag_decode_capacity(batch, num_q_heads, num_kv_heads, max_pages, page_size, query_tokens=1, split_tokens=0,
                         prefix_share=True, cus=256, workers_per_cu=1) -> dict:
    """Workspace capacities a decode call would be given (host arithmetic only)."""
    out = (ctypes.c_int64 * 7)()
    _check(lib().rl_attn_diag_decode_capacity(batch, num_q_heads, num_kv_heads, max_pages, page_size,
                                              query_tokens, split_tokens, int(bool(prefix_share)), cus,
                                              workers_per_cu, out))
    keys = ("max_items", "max_slots", "max_workers", "group_cap", "target_items", "prefix_grid", "bytes")
    return dict(zip(keys, (int(x) for x in out)))


def diag_extend_capacity(batch, total_q, num_q_heads, num_kv_heads) -> dict:
    """Work-unit capacity of an extend call (host arithmetic only)."""
    out = (ctypes.c_int64 * 4)()
    _check(lib().rl_attn_diag_extend_capacity(batch, total_q, num_q_heads, num_kv_heads, out))
    return dict(zip(("max_items", "rows_head", "tile_tokens", "head_blocks"), (int(x) for x in out)))


def diag_extend_plan(kv_lens, num_q_heads, num_kv_heads, max_tokens, qo_indptr=None, total_q=None, query_tokens=0,
                     cus=256) -> dict:
    """The work list of an extend call (``qo_indptr`` given) or of a deterministic decode of ``query_tokens`` tokens
    per sequence, planned on the host from host lengths."""
    b = len(kv_lens)
    lens = (ctypes.c_int32 * b)(*[int(x) for x in kv_lens])
    ind = None if qo_indptr is None else (ctypes.c_int32 * (b + 1))(*[int(x) for x in qo_indptr])
    if total_q is None:
        total_q = b * query_tokens if qo_indptr is None else int(qo_indptr[-1])
    out = (ctypes.c_int64 * 8)()
    _check(lib().rl_attn_diag_extend_plan(ind, lens, b, total_q, query_tokens, num_q_heads, num_kv_heads,
                                          max_tokens, cus, out))
    keys = ("items", "parts", "split_seqs", "split_units", "broken_units", "errors", "max_units", "mode")
    return dict(zip(keys, (int(x) for x in out)))
