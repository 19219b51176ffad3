"""Python binding of libsonic.so: argument marshalling only.

Every function here forwards torch tensors' device pointers, sizes and the
current HIP stream to the C entry point of the same name (see include/sonic.h)
and returns its status code.  No arithmetic of the path happens in Python, and
there is no fallback: if the library is missing or no GPU is present, calls
raise.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch  # loads the HIP runtime the library shares with torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsonic.so")

OK = 0
ERR_INVALID_ARG = 1
ERR_BAD_LAYOUT = 2
ERR_CAPACITY = 3
ERR_WORKSPACE = 4
ERR_UNSUPPORTED = 5
ERR_HIP = 6

ROLE_SYSTEM, ROLE_HISTORY_TEXT, ROLE_NEXUS, ROLE_CURRENT = 0, 1, 2, 3
NEXUS_ALL, NEXUS_UP_TO_OWN = 0, 1   # Nexus <-> Nexus visibility scope of the prefill mask

EXPORTS = (
    "sonic_abi_version", "sonic_status_string", "sonic_validate_layout_host", "sonic_layout_stats_host",
    "sonic_prefill_workspace_bytes", "sonic_segment_attn_prefill", "sonic_kv_compact",
    "sonic_decode_workspace_bytes", "sonic_compressed_decode", "sonic_compressed_decode_noalloc",
    "sonic_nexus_extend_workspace_bytes",
    "sonic_nexus_extend", "sonic_role_projection_workspace_bytes", "sonic_role_projection",
    "sonic_nexus_recon_workspace_bytes", "sonic_nexus_recon_targets",
    "sonic_kv_compact_q4", "sonic_cache_expand_q4", "sonic_decode_q4_workspace_bytes", "sonic_compressed_decode_q4",
    "sonic_decode_weighted_workspace_bytes", "sonic_compressed_decode_weighted", "sonic_kv_compact_weights",
    "sonic_cache_evict_workspace_bytes", "sonic_cache_evict",
    "sonic_tree_plan_bytes", "sonic_tree_plan", "sonic_tree_decode_workspace_bytes", "sonic_tree_decode",
    "sonic_logits_process_workspace_bytes", "sonic_logits_process", "sonic_tree_accept", "sonic_cache_append",
)

_lib = None

_i32, _i64, _f32, _sz, _p = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p


class SonicError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


def lib() -> ctypes.CDLL:
    """Load libsonic.so once; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_21927_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    L.sonic_abi_version.restype = _i32
    L.sonic_abi_version.argtypes = []
    L.sonic_status_string.restype = ctypes.c_char_p
    L.sonic_status_string.argtypes = [_i32]
    L.sonic_validate_layout_host.restype = _i32
    L.sonic_validate_layout_host.argtypes = [_i32, _p, _p, _p, _p]
    L.sonic_layout_stats_host.restype = _i32
    L.sonic_layout_stats_host.argtypes = [_i32, _p, _p, _p, _i32, _p, _p]
    L.sonic_prefill_workspace_bytes.restype = _sz
    L.sonic_prefill_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.sonic_segment_attn_prefill.restype = _i32
    L.sonic_segment_attn_prefill.argtypes = [_i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _f32, _i32, _p,
                                             _p, _p, _p, _sz, _p, _p]
    L.sonic_kv_compact.restype = _i32
    L.sonic_kv_compact.argtypes = [_i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p]
    L.sonic_decode_workspace_bytes.restype = _sz
    L.sonic_decode_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32]
    L.sonic_compressed_decode.restype = _i32
    L.sonic_compressed_decode.argtypes = [_i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p, _f32,
                                          _p, _p, _sz, _p, _p]
    L.sonic_compressed_decode_noalloc.restype = _i32
    L.sonic_compressed_decode_noalloc.argtypes = [_i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                                  _f32, _p, _p, _p]
    L.sonic_nexus_extend_workspace_bytes.restype = _sz
    L.sonic_nexus_extend_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.sonic_nexus_extend.restype = _i32
    L.sonic_nexus_extend.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                     _f32, _p, _p, _sz, _p, _p]
    L.sonic_role_projection_workspace_bytes.restype = _sz
    L.sonic_role_projection_workspace_bytes.argtypes = [_i32]
    L.sonic_role_projection.restype = _i32
    L.sonic_role_projection.argtypes = [_i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _sz, _p, _p]
    L.sonic_nexus_recon_workspace_bytes.restype = _sz
    L.sonic_nexus_recon_workspace_bytes.argtypes = [_i32, _i32]
    L.sonic_nexus_recon_targets.restype = _i32
    L.sonic_nexus_recon_targets.argtypes = [_i32, _i32, _i32, _p, _p, _p, _p, _i32, _p, _p, _p, _p, _sz, _p, _p]
    L.sonic_kv_compact_q4.restype = _i32
    L.sonic_kv_compact_q4.argtypes = [_i32] * 5 + [_p] * 14
    L.sonic_cache_expand_q4.restype = _i32
    L.sonic_cache_expand_q4.argtypes = [_i32] * 4 + [_p] * 14
    L.sonic_decode_q4_workspace_bytes.restype = _sz
    L.sonic_decode_q4_workspace_bytes.argtypes = [_i32] * 5
    L.sonic_compressed_decode_q4.restype = _i32
    L.sonic_compressed_decode_q4.argtypes = [_i32] * 5 + [_p] * 10 + [_f32, _p, _p, _p, _sz, _p, _p]
    L.sonic_decode_weighted_workspace_bytes.restype = _sz
    L.sonic_decode_weighted_workspace_bytes.argtypes = [_i32] * 4
    L.sonic_compressed_decode_weighted.restype = _i32
    L.sonic_compressed_decode_weighted.argtypes = [_i32] * 5 + [_p] * 8 + [_f32, _p, _p, _p, _sz, _p, _p]
    L.sonic_kv_compact_weights.restype = _i32
    L.sonic_kv_compact_weights.argtypes = [_i32] * 3 + [_p] * 8
    L.sonic_cache_evict_workspace_bytes.restype = _sz
    L.sonic_cache_evict_workspace_bytes.argtypes = [_i32] * 2
    L.sonic_cache_evict.restype = _i32
    L.sonic_cache_evict.argtypes = [_i32] * 4 + [_p] * 20 + [_sz, _p, _p]
    L.sonic_tree_plan_bytes.restype = _sz
    L.sonic_tree_plan_bytes.argtypes = [_i32] * 3
    L.sonic_tree_plan.restype = _i32
    L.sonic_tree_plan.argtypes = [_i32] * 3 + [_p] * 3 + [_sz, _p, _p]
    L.sonic_tree_decode_workspace_bytes.restype = _sz
    L.sonic_tree_decode_workspace_bytes.argtypes = [_i32] * 5
    L.sonic_tree_decode.restype = _i32
    L.sonic_tree_decode.argtypes = [_i32] * 7 + [_p, _sz] + [_p] * 9 + [_f32, _p, _i32, _p, _sz, _p, _p]
    L.sonic_logits_process_workspace_bytes.restype = _sz
    L.sonic_logits_process_workspace_bytes.argtypes = [_i32] * 2
    L.sonic_logits_process.restype = _i32
    L.sonic_logits_process.argtypes = [_i32] * 4 + [_p, _i32, _p, _sz] + [_p] * 16 + [_sz, _p, _p]
    L.sonic_tree_accept.restype = _i32
    L.sonic_tree_accept.argtypes = [_i32] * 3 + [_p, _sz] + [_p] * 12
    L.sonic_cache_append.restype = _i32
    L.sonic_cache_append.argtypes = [_i32] * 5 + [_p] * 14
    _lib = L
    return L


def status_string(code: int) -> str:
    return lib().sonic_status_string(int(code)).decode()


def abi_version() -> int:
    return int(lib().sonic_abi_version())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libsonic must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _np_ptr(a):
    return ctypes.c_void_p(a.ctypes.data) if a is not None else None


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dev(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("libsonic GPU entry points take device tensors")


_I32, _I64, _U8, _BF16, _F32 = torch.int32, torch.int64, torch.uint8, torch.bfloat16, torch.float32


def _types(**named):
    """named=(tensor, dtype): the C ABI reads raw memory, so a wrong element type is refused here."""
    for name, (t, dt) in named.items():
        if t is not None and t.dtype != dt:
            raise TypeError(f"{name} must be {dt}, got {t.dtype}")


# ----------------------------------------------------------------- host helpers
def validate_layout_host(cu_seqlens, role, turn_id):
    """(status, first bad request) for numpy int32 cu, uint8 role, int32 turn_id."""
    import numpy as np
    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    r = np.ascontiguousarray(role, dtype=np.uint8)
    t = np.ascontiguousarray(turn_id, dtype=np.int32)
    bad = ctypes.c_int32(-1)
    st = lib().sonic_validate_layout_host(len(cu) - 1, _np_ptr(cu), _np_ptr(r), _np_ptr(t), ctypes.byref(bad))
    return int(st), int(bad.value)


def layout_stats_host(cu_seqlens, role, turn_id, nexus_scope: int = NEXUS_ALL):
    """(visible pairs per request int64[B], kept rows per request int32[B])."""
    import numpy as np
    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    r = np.ascontiguousarray(role, dtype=np.uint8)
    t = np.ascontiguousarray(turn_id, dtype=np.int32)
    B = len(cu) - 1
    vis = np.zeros(max(B, 1), np.int64)
    kept = np.zeros(max(B, 1), np.int32)
    st = lib().sonic_layout_stats_host(B, _np_ptr(cu), _np_ptr(r), _np_ptr(t), int(nexus_scope), _np_ptr(vis),
                                       _np_ptr(kept))
    if st != OK:
        raise SonicError(st, "sonic_layout_stats_host")
    return vis[:B], kept[:B]


# ----------------------------------------------------------------- step 1: prefill
def prefill_workspace_bytes(batch: int, total_tokens: int, num_q_heads: int, num_kv_heads: int, head_dim: int) -> int:
    return int(lib().sonic_prefill_workspace_bytes(batch, total_tokens, num_q_heads, num_kv_heads, head_dim))


def segment_attn_prefill(cu_seqlens, role, turn_id, q, k, v, out, workspace, dev_status, softmax_scale=None,
                         nexus_scope: int = NEXUS_ALL, nexus_mass=None, key_weight=None, stream=None) -> int:
    """q [T,Hq,d] bf16, k/v [T,Hkv,d] bf16, out [T,Hq,d] fp32; cu int32 [B+1]; role uint8 [T];
    turn_id int32 [T]; workspace uint8 [>= prefill_workspace_bytes]; dev_status int32 [1];
    optional statistics nexus_mass fp32 [T,Hq] and key_weight fp32 [T]."""
    _dev(cu_seqlens, role, turn_id, q, k, v, out, workspace, dev_status, nexus_mass, key_weight)
    _types(cu_seqlens=(cu_seqlens, _I32), role=(role, _U8), turn_id=(turn_id, _I32), q=(q, _BF16), k=(k, _BF16),
           v=(v, _BF16), out=(out, _F32), dev_status=(dev_status, _I32), nexus_mass=(nexus_mass, _F32),
           key_weight=(key_weight, _F32))
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return int(lib().sonic_segment_attn_prefill(
        cu_seqlens.numel() - 1, T, Hq, Hkv, d, _ptr(cu_seqlens), _ptr(role), _ptr(turn_id), _ptr(q), _ptr(k),
        _ptr(v), scale, int(nexus_scope), _ptr(out), _ptr(nexus_mass), _ptr(key_weight), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)))


# ----------------------------------------------------------------- step 2: compaction
def kv_compact(cu_seqlens, role, k, v, k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, keep_idx,
               dev_status, max_seqlen: int, stream=None) -> int:
    """k/v [T,Hkv,d] bf16 -> k_cache/v_cache [rows,Hkv,d]; cache_row_off int64 [B]; cache_row_cap int32 [B];
    cache_len int32 [B]; keep_idx int32 [rows]."""
    _dev(cu_seqlens, role, k, v, k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, keep_idx, dev_status)
    _types(cu_seqlens=(cu_seqlens, _I32), role=(role, _U8), k=(k, _BF16), v=(v, _BF16), k_cache=(k_cache, _BF16),
           v_cache=(v_cache, _BF16), cache_row_off=(cache_row_off, _I64), cache_row_cap=(cache_row_cap, _I32),
           cache_len=(cache_len, _I32), keep_idx=(keep_idx, _I32), dev_status=(dev_status, _I32))
    T, Hkv, d = k.shape
    return int(lib().sonic_kv_compact(
        cu_seqlens.numel() - 1, T, int(max_seqlen), Hkv, d, _ptr(cu_seqlens), _ptr(role), _ptr(k), _ptr(v),
        _ptr(k_cache), _ptr(v_cache), _ptr(cache_row_off), _ptr(cache_row_cap), _ptr(cache_len), _ptr(keep_idx),
        _ptr(dev_status), _stream(stream)))


# ----------------------------------------------------------------- step 3: decode
def decode_workspace_bytes(batch: int, num_q_heads: int, head_dim: int, max_ctx: int) -> int:
    return int(lib().sonic_decode_workspace_bytes(batch, num_q_heads, head_dim, max_ctx))


def compressed_decode(k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out, workspace,
                      dev_status, max_ctx: int, row_role=None, softmax_scale=None, stream=None) -> int:
    """q [B,Hq,d] bf16; k_new/v_new [B,Hkv,d] bf16; out [B,Hq,d] fp32; row_role uint8 [rows] or None."""
    _dev(k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out, workspace, dev_status,
         row_role)
    _types(k_cache=(k_cache, _BF16), v_cache=(v_cache, _BF16), cache_row_off=(cache_row_off, _I64),
           cache_row_cap=(cache_row_cap, _I32), cache_len=(cache_len, _I32), q=(q, _BF16), k_new=(k_new, _BF16),
           v_new=(v_new, _BF16), out=(out, _F32), dev_status=(dev_status, _I32), row_role=(row_role, _U8))
    B, Hq, d = q.shape
    Hkv = k_new.shape[1]
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return int(lib().sonic_compressed_decode(
        B, Hq, Hkv, d, int(max_ctx), _ptr(k_cache), _ptr(v_cache), _ptr(cache_row_off), _ptr(cache_row_cap),
        _ptr(cache_len), _ptr(row_role), _ptr(q), _ptr(k_new), _ptr(v_new), scale, _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)))


def compressed_decode_noalloc(k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out,
                              dev_status, max_ctx: int, row_role=None, softmax_scale=None, stream=None) -> int:
    """compressed_decode without a workspace: the library's fixed per-GPU scratch is used."""
    _dev(k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out, dev_status, row_role)
    _types(k_cache=(k_cache, _BF16), v_cache=(v_cache, _BF16), cache_row_off=(cache_row_off, _I64),
           cache_row_cap=(cache_row_cap, _I32), cache_len=(cache_len, _I32), q=(q, _BF16), k_new=(k_new, _BF16),
           v_new=(v_new, _BF16), out=(out, _F32), dev_status=(dev_status, _I32), row_role=(row_role, _U8))
    B, Hq, d = q.shape
    Hkv = k_new.shape[1]
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return int(lib().sonic_compressed_decode_noalloc(
        B, Hq, Hkv, d, int(max_ctx), _ptr(k_cache), _ptr(v_cache), _ptr(cache_row_off), _ptr(cache_row_cap),
        _ptr(cache_len), _ptr(row_role), _ptr(q), _ptr(k_new), _ptr(v_new), scale, _ptr(out), _ptr(dev_status),
        _stream(stream)))


# ----------------------------------------------------------------- next turn: Nexus step
def nexus_extend_workspace_bytes(batch: int, total_new: int, max_rows: int, num_kv_heads: int,
                                 head_dim: int) -> int:
    return int(lib().sonic_nexus_extend_workspace_bytes(batch, total_new, max_rows, num_kv_heads, head_dim))


def nexus_extend(nexus_cu, keep_len, k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k, v, out,
                 workspace, dev_status, max_rows: int, body_len=None, softmax_scale=None, stream=None) -> int:
    """nexus_cu int32 [B+1]; keep_len int32 [B]; body_len int32 [B] or None (the whole tail);
    q [N,Hq,d] bf16; k/v [N,Hkv,d] bf16; out [N,Hq,d] fp32."""
    _dev(nexus_cu, keep_len, body_len, k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k, v, out,
         workspace, dev_status)
    _types(nexus_cu=(nexus_cu, _I32), keep_len=(keep_len, _I32), body_len=(body_len, _I32),
           k_cache=(k_cache, _BF16), v_cache=(v_cache, _BF16), cache_row_off=(cache_row_off, _I64),
           cache_row_cap=(cache_row_cap, _I32), cache_len=(cache_len, _I32), q=(q, _BF16), k=(k, _BF16),
           v=(v, _BF16), out=(out, _F32), dev_status=(dev_status, _I32))
    N, Hq, d = q.shape
    Hkv = k.shape[1]
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return int(lib().sonic_nexus_extend(
        nexus_cu.numel() - 1, N, Hq, Hkv, d, int(max_rows), _ptr(nexus_cu), _ptr(keep_len), _ptr(body_len),
        _ptr(k_cache), _ptr(v_cache), _ptr(cache_row_off), _ptr(cache_row_cap), _ptr(cache_len), _ptr(q), _ptr(k),
        _ptr(v), scale, _ptr(out), _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(dev_status),
        _stream(stream)))


# ----------------------------------------------------------------- role-routed projection
def role_projection_workspace_bytes(total_tokens: int) -> int:
    return int(lib().sonic_role_projection_workspace_bytes(total_tokens))


def role_projection(role, x, w_text, w_nexus, y, workspace, dev_status, stream=None) -> int:
    """role uint8 [T]; x [T,K] bf16; w_text / w_nexus [N,K] bf16; y [T,N] fp32 (Nexus rows use w_nexus)."""
    _dev(role, x, w_text, w_nexus, y, workspace, dev_status)
    _types(role=(role, _U8), x=(x, _BF16), w_text=(w_text, _BF16), w_nexus=(w_nexus, _BF16), y=(y, _F32),
           dev_status=(dev_status, _I32))
    T, K = x.shape
    N = w_text.shape[0]
    if tuple(w_nexus.shape) != (N, K) or tuple(w_text.shape) != (N, K) or tuple(y.shape) != (T, N) or \
            role.numel() != T:
        raise ValueError("role_projection: inconsistent shapes")
    return int(lib().sonic_role_projection(
        T, K, N, _ptr(role), _ptr(x), _ptr(w_text), _ptr(w_nexus), _ptr(y), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)))


# ----------------------------------------------------------------- reconstruction targets
def nexus_recon_workspace_bytes(batch: int, total_tokens: int) -> int:
    return int(lib().sonic_nexus_recon_workspace_bytes(batch, total_tokens))


def nexus_recon_targets(cu_seqlens, role, turn_id, h, target, cos_target, entropy_ratio, workspace, dev_status,
                        stream=None) -> int:
    """h [T,Dm] bf16; target [n,Dm] fp32, cos_target [n] fp32, entropy_ratio [n] fp32 with n >= the
    batch's Nexus count (rows in packed position order)."""
    _dev(cu_seqlens, role, turn_id, h, target, cos_target, entropy_ratio, workspace, dev_status)
    _types(cu_seqlens=(cu_seqlens, _I32), role=(role, _U8), turn_id=(turn_id, _I32), h=(h, _BF16),
           target=(target, _F32), cos_target=(cos_target, _F32), entropy_ratio=(entropy_ratio, _F32),
           dev_status=(dev_status, _I32))
    T, Dm = h.shape
    n = target.shape[0]
    if target.shape[1] != Dm or cos_target.numel() < n or entropy_ratio.numel() < n:
        raise ValueError("nexus_recon_targets: inconsistent output shapes")
    return int(lib().sonic_nexus_recon_targets(
        cu_seqlens.numel() - 1, T, Dm, _ptr(cu_seqlens), _ptr(role), _ptr(turn_id), _ptr(h), n, _ptr(target),
        _ptr(cos_target), _ptr(entropy_ratio), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _ptr(dev_status), _stream(stream)))


# ----------------------------------------------------------------- 4-bit rows
def _pass(where, fn, stream, head, tensors, tail=()):
    """Call fn(*head, pointers, *tail, stream) for tensors = [(name, tensor, dtype, shape or None)], or a number in a
    tensor's place, once every tensor is contiguous, of its type and shape, and on one GPU.  The call is made on that
    GPU, on its current stream unless one is given."""
    dev, args = None, list(head)
    for name, t, dtype, shape in tensors:
        if t is None or dtype is None:
            args.append(t)
            continue
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if shape is not None and t.shape != shape:
            raise ValueError(f"{where}: {name} must be {shape}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError("tensors passed to libsonic must be contiguous")
        d = t.get_device()
        if d != dev:
            if d < 0:
                raise ValueError("libsonic GPU entry points take device tensors")
            if dev is not None:
                raise ValueError("tensors of one call must be on one GPU")
            dev = d
        args.append(t.data_ptr())
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    elif stream.device_index != dev:
        raise ValueError("the stream must be one of the tensors' GPU")
    args += tail
    args.append(stream.cuda_stream)
    if dev == torch.cuda.current_device():
        return fn(*args)
    with torch.cuda.device(dev):
        return fn(*args)


def _number(x):
    """A plain argument between the tensors of _pass."""
    return ("", x, None, None)


def _q4_planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale):
    return [("k_cache", k_cache, _U8, (rows, Hkv, d // 2)), ("k_scale", k_scale, _U8, (rows, Hkv, d // 32)),
            ("v_cache", v_cache, _U8, (rows, Hkv, d // 2)), ("v_scale", v_scale, _U8, (rows, Hkv, d // 32))]


def kv_compact_q4(cu_seqlens, role, k, v, k_cache, k_scale, v_cache, v_scale, cache_row_off, cache_row_cap, cache_len, keep_idx,
                  dev_status, max_seqlen: int, stream=None) -> int:
    """kv_compact into 4-bit rows: k_cache/v_cache uint8 [rows,Hkv,d/2] codes, k_scale/v_scale uint8 [rows,Hkv,d/32]."""
    T, Hkv, d = k.shape
    B, rows = cu_seqlens.numel() - 1, k_cache.shape[0]
    return _pass("kv_compact_q4", lib().sonic_kv_compact_q4, stream, (B, T, int(max_seqlen), Hkv, d), [
        ("cu_seqlens", cu_seqlens, _I32, None), ("role", role, _U8, (T,)), ("k", k, _BF16, None), ("v", v, _BF16, (T, Hkv, d)),
        *_q4_planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale), ("cache_row_off", cache_row_off, _I64, (B,)),
        ("cache_row_cap", cache_row_cap, _I32, (B,)), ("cache_len", cache_len, _I32, (B,)), ("keep_idx", keep_idx, _I32, (rows,)),
        ("dev_status", dev_status, _I32, None)])


def cache_expand_q4(k_cache, k_scale, v_cache, v_scale, cache_row_off, cache_row_cap, row_begin, row_end, k, v, out_row_off,
                    out_row_cap, dev_status, max_rows: int, stream=None) -> int:
    """4-bit rows row_begin[b] .. row_end[b] of every request to rows out_row_off[b] .. of k/v [n,Hkv,d] bf16."""
    n, Hkv, d = k.shape
    B = cache_row_off.numel()
    return _pass("cache_expand_q4", lib().sonic_cache_expand_q4, stream, (B, int(max_rows), Hkv, d), [
        *_q4_planes(k_cache.shape[0], Hkv, d, k_cache, k_scale, v_cache, v_scale), ("cache_row_off", cache_row_off, _I64, None),
        ("cache_row_cap", cache_row_cap, _I32, (B,)), ("row_begin", row_begin, _I32, (B,)), ("row_end", row_end, _I32, (B,)),
        ("k", k, _BF16, None), ("v", v, _BF16, (n, Hkv, d)), ("out_row_off", out_row_off, _I64, (B,)),
        ("out_row_cap", out_row_cap, _I32, (B,)), ("dev_status", dev_status, _I32, None)])


def _decode_tensors(planes, B, Hq, Hkv, d, rows, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, softmax_scale, out,
                    row_weight, workspace):
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return [*planes, ("cache_row_off", cache_row_off, _I64, (B,)), ("cache_row_cap", cache_row_cap, _I32, (B,)),
            ("cache_len", cache_len, _I32, (B,)), ("q", q, _BF16, None), ("k_new", k_new, _BF16, (B, Hkv, d)),
            ("v_new", v_new, _BF16, (B, Hkv, d)), _number(scale), ("out", out, _F32, (B, Hq, d)),
            ("row_weight", row_weight, _F32, (rows,)), ("workspace", workspace, workspace.dtype, None),
            _number(workspace.numel() * workspace.element_size())]


def decode_q4_workspace_bytes(batch: int, num_q_heads: int, head_dim: int, max_ctx: int, weighted: bool) -> int:
    return int(lib().sonic_decode_q4_workspace_bytes(batch, num_q_heads, head_dim, max_ctx, int(bool(weighted))))


def compressed_decode_q4(k_cache, k_scale, v_cache, v_scale, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out, workspace,
                         dev_status, max_ctx: int, row_weight=None, softmax_scale=None, stream=None) -> int:
    """compressed_decode over 4-bit rows; row_weight fp32 [rows] or None: each row's attention is added to it."""
    B, Hq, d = q.shape
    Hkv, rows = k_new.shape[1], k_cache.shape[0]
    return _pass("compressed_decode_q4", lib().sonic_compressed_decode_q4, stream, (B, Hq, Hkv, d, int(max_ctx)), [
        *_decode_tensors(_q4_planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale), B, Hq, Hkv, d, rows, cache_row_off,
                         cache_row_cap, cache_len, q, k_new, v_new, softmax_scale, out, row_weight, workspace),
        ("dev_status", dev_status, _I32, None)])


# ----------------------------------------------------------------- row weights, eviction
def decode_weighted_workspace_bytes(batch: int, num_q_heads: int, head_dim: int, max_ctx: int) -> int:
    return int(lib().sonic_decode_weighted_workspace_bytes(batch, num_q_heads, head_dim, max_ctx))


def compressed_decode_weighted(k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, out, row_weight, workspace,
                               dev_status, max_ctx: int, softmax_scale=None, stream=None) -> int:
    """compressed_decode that also adds each row's attention, averaged over the q-heads, to row_weight fp32 [rows]."""
    B, Hq, d = q.shape
    Hkv, rows = k_new.shape[1], k_cache.shape[0]
    planes = [("k_cache", k_cache, _BF16, (rows, Hkv, d)), ("v_cache", v_cache, _BF16, (rows, Hkv, d))]
    return _pass("compressed_decode_weighted", lib().sonic_compressed_decode_weighted, stream, (B, Hq, Hkv, d, int(max_ctx)), [
        *_decode_tensors(planes, B, Hq, Hkv, d, rows, cache_row_off, cache_row_cap, cache_len, q, k_new, v_new, softmax_scale, out,
                         row_weight, workspace), ("dev_status", dev_status, _I32, None)])


def kv_compact_weights(cu_seqlens, key_weight, cache_row_off, cache_len, keep_idx, row_weight, dev_status, max_rows: int,
                       stream=None) -> int:
    """The prefill's key_weight fp32 [T] to the rows a compaction kept: row_weight fp32 [rows], keep_idx int32 [rows]."""
    B = cu_seqlens.numel() - 1
    return _pass("kv_compact_weights", lib().sonic_kv_compact_weights, stream, (B, key_weight.numel(), int(max_rows)), [
        ("cu_seqlens", cu_seqlens, _I32, None), ("key_weight", key_weight, _F32, None), ("cache_row_off", cache_row_off, _I64, (B,)),
        ("cache_len", cache_len, _I32, (B,)), ("keep_idx", keep_idx, _I32, row_weight.shape), ("row_weight", row_weight, _F32, None),
        ("dev_status", dev_status, _I32, None)])


def cache_evict_workspace_bytes(batch: int, max_rows: int) -> int:
    return int(lib().sonic_cache_evict_workspace_bytes(batch, max_rows))


def cache_evict(k_cache, v_cache, cache_row_off, cache_len, row_weight, keep_head, keep_tail, budget, workspace, dev_status,
                max_rows: int, k_scale=None, v_scale=None, k_out=None, v_out=None, k_scale_out=None, v_scale_out=None,
                out_row_off=None, out_row_cap=None, out_len=None, out_weight=None, keep_idx=None, stream=None) -> int:
    """Keep the first keep_head[b], the last keep_tail[b] and the heaviest other rows, budget[b] in all.  bf16 rows
    [rows,Hkv,d], or codes [rows,Hkv,d/2] with k_scale/v_scale [rows,Hkv,d/32].  Without k_out the rows move down in
    place; with it (and v_out, the scales, out_row_off, out_row_cap, out_len, out_weight) they go to another cache.
    keep_idx int32 [rows of the cache written] or None: the kept rows' places before the call."""
    rows, Hkv, width = k_cache.shape
    B = cache_row_off.numel()
    kind, d = (_BF16, width) if k_scale is None else (_U8, 2 * width)
    n = rows if k_out is None else k_out.shape[0]
    row, scales, new_row, new_scales = (rows, Hkv, width), (rows, Hkv, d // 32), (n, Hkv, width), (n, Hkv, d // 32)
    return _pass("cache_evict", lib().sonic_cache_evict, stream, (B, int(max_rows), Hkv, d), [
        ("k_cache", k_cache, kind, None), ("k_scale", k_scale, _U8, scales), ("v_cache", v_cache, kind, row),
        ("v_scale", v_scale, _U8, scales), ("cache_row_off", cache_row_off, _I64, None), ("cache_len", cache_len, _I32, (B,)),
        ("row_weight", row_weight, _F32, (rows,)), ("keep_head", keep_head, _I32, (B,)), ("keep_tail", keep_tail, _I32, (B,)),
        ("budget", budget, _I32, (B,)), ("k_out", k_out, kind, new_row), ("k_scale_out", k_scale_out, _U8, new_scales),
        ("v_out", v_out, kind, new_row), ("v_scale_out", v_scale_out, _U8, new_scales), ("out_row_off", out_row_off, _I64, (B,)),
        ("out_row_cap", out_row_cap, _I32, (B,)), ("out_len", out_len, _I32, (B,)), ("out_weight", out_weight, _F32, (n,)),
        ("keep_idx", keep_idx, _I32, (n,)), ("workspace", workspace, workspace.dtype, None),
        _number(workspace.numel() * workspace.element_size()), ("dev_status", dev_status, _I32, None)])


# ----------------------------------------------------------------- a step over drafted tokens
def _sized(name, t):
    """A workspace between the tensors of _pass, and its bytes."""
    return [(name, t, None if t is None else t.dtype, None), _number(0 if t is None else t.numel() * t.element_size())]


def tree_plan_bytes(batch: int, total_nodes: int, max_nodes: int) -> int:
    return int(lib().sonic_tree_plan_bytes(batch, total_nodes, max_nodes))


def tree_plan(cu_nodes, parent, total_nodes: int, max_nodes: int, plan, dev_status, stream=None) -> int:
    """Which nodes every node sees: cu_nodes int32 [B+1]; parent int32 [total_nodes], or None for chains; plan uint8
    [>= tree_plan_bytes]."""
    return _pass("tree_plan", lib().sonic_tree_plan, stream, (cu_nodes.numel() - 1, int(total_nodes), int(max_nodes)), [
        ("cu_nodes", cu_nodes, _I32, None), ("parent", parent, _I32, (total_nodes,)), *_sized("plan", plan),
        ("dev_status", dev_status, _I32, None)])


def tree_decode_workspace_bytes(batch: int, max_nodes: int, num_q_heads: int, head_dim: int, max_ctx: int) -> int:
    return int(lib().sonic_tree_decode_workspace_bytes(batch, max_nodes, num_q_heads, head_dim, max_ctx))


def tree_decode(plan, k_cache, v_cache, cache_row_off, cache_len, q, k_new, v_new, out, workspace, dev_status, max_nodes: int,
                max_ctx: int, k_scale=None, v_scale=None, softmax_scale=None, stream=None) -> int:
    """The nodes' attention: q [N,Hq,d] bf16; k_new/v_new [N,Hkv,d] bf16; out [N,Hq,d] fp32 or bf16; a cache of bf16 rows
    [rows,Hkv,d], or of codes [rows,Hkv,d/2] with k_scale/v_scale [rows,Hkv,d/32]."""
    N, Hq, d = q.shape
    Hkv, rows, B = k_new.shape[1], k_cache.shape[0], cache_len.numel()
    if out.dtype not in (_F32, _BF16):
        raise TypeError(f"out must be {_F32} or {_BF16}, got {out.dtype}")
    planes = _planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale)
    scale = 0.0 if softmax_scale is None else float(softmax_scale)   # 0: the library's 1/sqrt(d)
    return _pass("tree_decode", lib().sonic_tree_decode, stream, (B, N, int(max_nodes), Hq, Hkv, d, int(max_ctx)), [
        *_sized("plan", plan), *planes, ("cache_row_off", cache_row_off, _I64, (B,)), ("cache_len", cache_len, _I32, None),
        ("q", q, _BF16, None), ("k_new", k_new, _BF16, (N, Hkv, d)), ("v_new", v_new, _BF16, (N, Hkv, d)), _number(scale),
        ("out", out, out.dtype, (N, Hq, d)), _number(int(out.dtype is _BF16)), *_sized("workspace", workspace),
        ("dev_status", dev_status, _I32, None)])


def _planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale):
    """A cache's arrays in the order of the C ABI: codes with scales, or bf16 rows with none."""
    if (k_scale is None) != (v_scale is None):
        raise ValueError("k_scale and v_scale are given together")
    if k_scale is not None:
        return _q4_planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale)
    return [("k_cache", k_cache, _BF16, (rows, Hkv, d)), _number(None), ("v_cache", v_cache, _BF16, (rows, Hkv, d)), _number(None)]


def logits_process_workspace_bytes(total_rows: int, vocab: int) -> int:
    return int(lib().sonic_logits_process_workspace_bytes(total_rows, vocab))


def logits_process(logits, best, workspace, dev_status, plan=None, batch=None, max_nodes: int = 1, node_token=None, tokens=None,
                   token_off=None, token_len=None, prompt_len=None, repetition=None, presence=None, frequency=None, bias_cu=None,
                   bias_token=None, bias_value=None, allowed=None, best_value=None, out=None, stream=None) -> int:
    """Penalties, biases and masks on logits [n,V] (fp32 or bf16), and the rows' best tokens: best int32 [n] or None, best_value
    fp32 [n] or None, out fp32 [n,V] or None.  Rows are the nodes of a plan (of `batch` requests), or one a request.
    node_token int32 [n]; tokens int32 with token_off int64 [B], token_len and prompt_len int32 [B]; repetition, presence,
    frequency fp32 [B]; bias_cu int32 [B+1], bias_token int32 and bias_value fp32; allowed int32 [n,(V+31)//32]."""
    n, V = logits.shape
    if plan is not None and batch is None:
        raise ValueError("a plan comes with the batch that it was made for")
    B = int(batch) if batch is not None else n
    if logits.dtype not in (_F32, _BF16):
        raise TypeError(f"logits must be {_F32} or {_BF16}, got {logits.dtype}")
    if tokens is not None and tokens.numel() == 0:           # (an empty tensor has no address: no history, ..
        tokens = token_off = token_len = prompt_len = None
    if bias_token is not None and bias_token.numel() == 0:   # .. and no biases)
        bias_cu = bias_token = bias_value = None
    m = 0 if bias_token is None else bias_token.numel()
    return _pass("logits_process", lib().sonic_logits_process, stream, (B, n, int(max_nodes), V), [
        ("logits", logits, logits.dtype, None), _number(int(logits.dtype is _BF16)), *_sized("plan", plan),
        ("node_token", node_token, _I32, (n,)), ("tokens", tokens, _I32, None), ("token_off", token_off, _I64, (B,)),
        ("token_len", token_len, _I32, (B,)), ("prompt_len", prompt_len, _I32, (B,)), ("repetition", repetition, _F32, (B,)),
        ("presence", presence, _F32, (B,)), ("frequency", frequency, _F32, (B,)), ("bias_cu", bias_cu, _I32, (B + 1,)),
        ("bias_token", bias_token, _I32, None), ("bias_value", bias_value, _F32, (m,)), ("allowed", allowed, _I32, (n, (V + 31) // 32)),
        ("out", out, _F32, (n, V)), ("best", best, _I32, (n,)), ("best_value", best_value, _F32, (n,)), *_sized("workspace", workspace),
        ("dev_status", dev_status, _I32, None)])


def tree_accept(plan, parent, node_token, chosen, path, path_len, next_token, dev_status, max_nodes: int, tokens=None, token_off=None,
                token_cap=None, token_len=None, stream=None) -> int:
    """The nodes that the chosen tokens confirm: parent int32 [N] or None; node_token, chosen, path int32 [N]; path_len,
    next_token int32 [B]; tokens int32 with token_off int64 [B], token_cap and token_len int32 [B], or none of them."""
    N, B = node_token.numel(), path_len.numel()
    return _pass("tree_accept", lib().sonic_tree_accept, stream, (B, N, int(max_nodes)), [
        *_sized("plan", plan), ("parent", parent, _I32, (N,)), ("node_token", node_token, _I32, None), ("chosen", chosen, _I32, (N,)),
        ("path", path, _I32, (N,)), ("path_len", path_len, _I32, None), ("next_token", next_token, _I32, (B,)),
        ("tokens", tokens, _I32, None), ("token_off", token_off, _I64, (B,)), ("token_cap", token_cap, _I32, (B,)),
        ("token_len", token_len, _I32, (B,)), ("dev_status", dev_status, _I32, None)])


def cache_append(new_cu, k_new, v_new, k_cache, v_cache, cache_row_off, cache_row_cap, cache_len, dev_status, max_rows: int, select=None,
                 select_len=None, k_scale=None, v_scale=None, stream=None) -> int:
    """New rows k_new/v_new [N,Hkv,d] bf16 to the end of the caches: all of a request's, or those at select int32 [N],
    select_len int32 [B]; bf16 rows, or codes with scales."""
    N, Hkv, d = k_new.shape
    B, rows = new_cu.numel() - 1, k_cache.shape[0]
    if N == 0:   # (an empty tensor has no address; there is nothing to select)
        select = select_len = None
    k, ks, v, vs = _planes(rows, Hkv, d, k_cache, k_scale, v_cache, v_scale)
    return _pass("cache_append", lib().sonic_cache_append, stream, (B, N, int(max_rows), Hkv, d), [
        ("new_cu", new_cu, _I32, None), ("select", select, _I32, (N,)), ("select_len", select_len, _I32, (B,)),
        ("k_new", k_new, _BF16, None), ("v_new", v_new, _BF16, (N, Hkv, d)), k, ks, v, vs,
        ("cache_row_off", cache_row_off, _I64, (B,)), ("cache_row_cap", cache_row_cap, _I32, (B,)),
        ("cache_len", cache_len, _I32, (B,)), ("dev_status", dev_status, _I32, None)])
