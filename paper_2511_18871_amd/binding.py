"""ctypes binding of libsp_attn.so.  Argument marshalling only: every step of the
attention runs in the HIP kernels behind the C ABI declared in include/sp_attn.h.
torch is used for device memory and streams, nothing else.  There is no CPU fallback:
if the library is missing, loading raises."""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsp_attn.so")

SP_OK = 0
SP_ERR_INVALID_ARG, SP_ERR_UNSUPPORTED, SP_ERR_WORKSPACE, SP_ERR_DEVICE = 1, 2, 3, 4
SP_BF16, SP_F32 = 0, 1
SP_SCHED_SHARED, SP_SCHED_NAIVE_CAUSAL = 0, 1

SP_BWD_STAGE_ROWSUM, SP_BWD_STAGE_DKDV, SP_BWD_STAGE_DQ, SP_BWD_STAGE_ALL = 1, 2, 4, 7
SP_MAX_DRAFT = 1024
SP_FLAG_RESPONSE_ROWS, SP_FLAG_ACCUMULATE_DKDV, SP_FLAG_ZERO_PROMPT_ROWS, SP_FLAG_OWN_TOKEN, SP_FLAG_MARK_ORPHANS = 1, 2, 4, 8, 16

EXPORTS = ("sp_attn_workspace_bytes", "sp_attn_reserve_bytes", "sp_attn_row_parts_bytes", "sp_attn_full_workspace_bytes", "sp_attn_kept_workspace_bytes", "sp_attn_sums_bytes", "sp_attn_fwd", "sp_attn_bwd", "sp_attn_fwd_batched",
           "sp_attn_bwd_batched", "sp_attn_bwd_batched_static", "sp_attn_bwd_batched_stages", "sp_attn_fwd_multi", "sp_attn_rope", "sp_attn_rope_qk", "sp_attn_fwd_batched_ex", "sp_attn_bwd_batched_ex", "sp_attn_fwd_batched_sums", "sp_attn_bwd_batched_sums",
           "sp_attn_loss_workspace_bytes", "sp_attn_logprob_fwd", "sp_attn_logprob_bwd", "sp_attn_logprob_bwd_ex", "sp_attn_grpo_loss",
           "sp_attn_cache_append", "sp_attn_decode_workspace_bytes", "sp_attn_decode", "sp_attn_adjust_logits",
           "sp_attn_tree_decode_workspace_bytes", "sp_attn_tree_decode", "sp_attn_cache_keep", "sp_attn_pages_workspace_bytes", "sp_attn_pages_fit",
           "sp_attn_cache_fork",
           "sp_attn_adjusted_logprob_workspace_bytes", "sp_attn_adjusted_logprob_fwd", "sp_attn_adjusted_logprob_bwd",
           "sp_attn_segment_table", "sp_attn_row_tile", "sp_attn_dkdv_waves", "sp_attn_pieces", "sp_attn_f32_rows", "sp_attn_mfma_ceiling", "sp_attn_probe_atomic_add", "sp_attn_set_small_shape_steps", "sp_attn_last_error", "sp_attn_version")

_lib = None


class _KvCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int)]


class _LogitRulesStruct(ctypes.Structure):
    _fields_ = [("repetition", ctypes.c_float), ("presence", ctypes.c_float), ("frequency", ctypes.c_float),
                ("temperature", ctypes.c_float), ("bias", ctypes.c_void_p)]


class SpAttnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"sp_attn status {status}: {message}")
        self.status = status


def load_library() -> ctypes.CDLL:
    """Load the in-tree library, building it first only if it has never been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from .build import build_library
        build_library(verbose=False)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    ip = ctypes.POINTER(ctypes.c_int32)
    lib.sp_attn_workspace_bytes.restype = sz
    lib.sp_attn_workspace_bytes.argtypes = [ctypes.c_int, i64, i32, i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_reserve_bytes.restype = sz
    lib.sp_attn_reserve_bytes.argtypes = [i64, i32, i32, ctypes.c_int]
    lib.sp_attn_row_parts_bytes.restype = sz
    lib.sp_attn_row_parts_bytes.argtypes = [i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_full_workspace_bytes.restype = sz
    lib.sp_attn_full_workspace_bytes.argtypes = [i64, i32, i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_kept_workspace_bytes.restype = sz
    lib.sp_attn_kept_workspace_bytes.argtypes = [i64, i32, i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_sums_bytes.restype = sz
    lib.sp_attn_sums_bytes.argtypes = [i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_fwd.restype = ctypes.c_int
    lib.sp_attn_fwd.argtypes = [vp, vp, vp, vp, vp, i32, ip, i32, i32, i32, i32, f32, ctypes.c_int, vp, sz, vp]
    lib.sp_attn_bwd.restype = ctypes.c_int
    lib.sp_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, i32, i32, i32, i32, f32,
                                ctypes.c_int, vp, sz, vp]
    lib.sp_attn_fwd_batched.restype = ctypes.c_int
    lib.sp_attn_fwd_batched.argtypes = [vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32, ctypes.c_int,
                                        ctypes.c_int, vp, sz, vp]
    lib.sp_attn_bwd_batched.restype = ctypes.c_int
    lib.sp_attn_bwd_batched.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32,
                                        ctypes.c_int, vp, sz, vp]
    lib.sp_attn_bwd_batched_static.restype = ctypes.c_int
    lib.sp_attn_bwd_batched_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32,
                                               ctypes.c_int, vp]
    lib.sp_attn_bwd_batched_stages.restype = ctypes.c_int
    lib.sp_attn_bwd_batched_stages.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32,
                                               f32, ctypes.c_int, ctypes.c_uint32, vp, sz, vp]
    pp = ctypes.POINTER(ctypes.c_void_p)
    lib.sp_attn_fwd_multi.restype = ctypes.c_int
    lib.sp_attn_fwd_multi.argtypes = [i32, pp, pp, pp, pp, pp, i32, ip, ip, ip, i32, i32, i32, f32, ctypes.c_int, vp, sz, vp]
    lib.sp_attn_fwd_batched_ex.restype = ctypes.c_int
    lib.sp_attn_fwd_batched_ex.argtypes = [vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32, ctypes.c_int,
                                           ctypes.c_int, ctypes.c_uint32, vp, vp, sz, vp]
    lib.sp_attn_bwd_batched_ex.restype = ctypes.c_int
    lib.sp_attn_bwd_batched_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32,
                                           ctypes.c_int, ctypes.c_uint32, ctypes.c_uint32, vp, vp, sz, vp]
    lib.sp_attn_fwd_batched_sums.restype = ctypes.c_int
    lib.sp_attn_fwd_batched_sums.argtypes = [vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32, ctypes.c_int,
                                             ctypes.c_int, ctypes.c_uint32, vp, vp, sz, vp, sz, vp]
    lib.sp_attn_bwd_batched_sums.restype = ctypes.c_int
    lib.sp_attn_bwd_batched_sums.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ip, ip, ip, i32, i32, i32, f32,
                                             ctypes.c_int, ctypes.c_uint32, ctypes.c_uint32, vp, vp, sz, vp, sz, vp]
    lib.sp_attn_loss_workspace_bytes.restype = sz
    lib.sp_attn_loss_workspace_bytes.argtypes = [i64, i32, i64]
    lib.sp_attn_logprob_fwd.restype = ctypes.c_int
    lib.sp_attn_logprob_fwd.argtypes = [vp, vp, vp, vp, i64, i32, ip, ip, ip, ctypes.c_int, vp, sz, vp]
    lib.sp_attn_logprob_bwd.restype = ctypes.c_int
    lib.sp_attn_logprob_bwd.argtypes = [vp, vp, vp, vp, vp, i64, i32, ip, ip, ip, ctypes.c_int, vp, sz, vp]
    lib.sp_attn_logprob_bwd_ex.restype = ctypes.c_int
    lib.sp_attn_logprob_bwd_ex.argtypes = [vp, vp, vp, vp, vp, i64, i32, ip, ip, ip, ctypes.c_int, ctypes.c_uint32, vp, sz, vp]
    lib.sp_attn_grpo_loss.restype = ctypes.c_int
    lib.sp_attn_grpo_loss.argtypes = [vp, vp, vp, vp, f32, f32, f32, vp, vp, i32, ip, ip, ip, vp, sz, vp]
    lib.sp_attn_rope.restype = ctypes.c_int
    lib.sp_attn_rope.argtypes = [vp, vp, i32, i32, i32, ip, ip, ip, i32, ctypes.c_double, ctypes.c_int, vp, sz, vp]
    lib.sp_attn_rope_qk.restype = ctypes.c_int
    lib.sp_attn_rope_qk.argtypes = [vp, vp, i32, vp, vp, i32, i32, i32, ip, ip, ip, i32, ctypes.c_double, ctypes.c_int, vp, sz, vp]
    cache_p, rules_p = ctypes.POINTER(_KvCacheStruct), ctypes.POINTER(_LogitRulesStruct)
    lib.sp_attn_cache_append.restype = ctypes.c_int
    lib.sp_attn_cache_append.argtypes = [cache_p, vp, i64, vp, i32, vp, i64, vp, vp, i64, i32, ip, vp, i32, vp, vp, vp, ctypes.c_double, vp]
    lib.sp_attn_decode_workspace_bytes.restype = sz
    lib.sp_attn_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_decode.restype = ctypes.c_int
    lib.sp_attn_decode.argtypes = [cache_p, vp, vp, vp, i32, i32, i32, ip, vp, i32, vp, vp, i32, vp, f32, vp, sz, vp]
    lib.sp_attn_tree_decode_workspace_bytes.restype = sz
    lib.sp_attn_tree_decode_workspace_bytes.argtypes = [i32, i32, i64, i32, i32, i32, ctypes.c_int]
    lib.sp_attn_tree_decode.restype = ctypes.c_int
    lib.sp_attn_tree_decode.argtypes = [cache_p, vp, vp, vp, i32, i32, i32, ip, ip, vp, i64, vp, i32, vp, vp, i32, vp, f32, vp, sz, vp]
    lib.sp_attn_cache_keep.restype = ctypes.c_int
    lib.sp_attn_cache_keep.argtypes = [cache_p, i32, i64, i32, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.sp_attn_pages_workspace_bytes.restype = sz
    lib.sp_attn_pages_workspace_bytes.argtypes = [i64, i32]
    lib.sp_attn_pages_fit.restype = ctypes.c_int
    lib.sp_attn_pages_fit.argtypes = [vp, i64, i32, i32, vp, i32, vp, vp, vp, sz, vp]
    lib.sp_attn_cache_fork.restype = ctypes.c_int
    lib.sp_attn_cache_fork.argtypes = [cache_p, i32, i64, vp, i32, vp, i32, vp, i32, vp, vp, i32, vp, ctypes.c_uint32, vp, sz, vp]
    lib.sp_attn_adjust_logits.restype = ctypes.c_int
    lib.sp_attn_adjust_logits.argtypes = [vp, i64, vp, i64, i64, rules_p, vp, i64, i32, i32, ip, vp, i32, vp, vp, i32, vp, ctypes.c_int, vp]
    lib.sp_attn_adjusted_logprob_workspace_bytes.restype = sz
    lib.sp_attn_adjusted_logprob_workspace_bytes.argtypes = [i64, i32, i64, i64]
    lib.sp_attn_adjusted_logprob_fwd.restype = ctypes.c_int
    lib.sp_attn_adjusted_logprob_fwd.argtypes = [vp, vp, vp, vp, vp, i64, rules_p, vp, i64, i32, ip, ip, ip, ctypes.c_int, ctypes.c_uint32, vp, sz, vp]
    lib.sp_attn_adjusted_logprob_bwd.restype = ctypes.c_int
    lib.sp_attn_adjusted_logprob_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, rules_p, vp, i64, i32, ip, ip, ip, ctypes.c_int, ctypes.c_uint32, vp, sz, vp]
    lib.sp_attn_segment_table.restype = ctypes.c_int
    lib.sp_attn_segment_table.argtypes = [i32, ip, ip, ip, ip, sz, ctypes.POINTER(sz)]
    lib.sp_attn_dkdv_waves.restype = ctypes.c_int
    lib.sp_attn_dkdv_waves.argtypes = [i32, ip, ip, ip, i32, i32, ctypes.c_uint32, ctypes.POINTER(ctypes.c_int32)]
    lib.sp_attn_pieces.restype = ctypes.c_int
    lib.sp_attn_pieces.argtypes = [i32, ip, ip, ip, i32, i32, ctypes.c_uint32, i32, ctypes.POINTER(ctypes.c_uint32), sz, ip]
    lib.sp_attn_f32_rows.restype = ctypes.c_int
    lib.sp_attn_f32_rows.argtypes = [i32, ip, ip, ip, i32, i32, i32, ctypes.c_uint32, ctypes.POINTER(ctypes.c_int32)]
    lib.sp_attn_row_tile.restype = ctypes.c_int
    lib.sp_attn_row_tile.argtypes = [i32, ip, ip, ip, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64),
                                     ctypes.POINTER(ctypes.c_int64)]
    lib.sp_attn_mfma_ceiling.restype = ctypes.c_int
    lib.sp_attn_mfma_ceiling.argtypes = [i32, vp, vp, i32, i32, vp, vp]
    lib.sp_attn_probe_atomic_add.restype = ctypes.c_int
    lib.sp_attn_probe_atomic_add.argtypes = [vp, i64, i32, i32, i32, i32, vp]
    lib.sp_attn_set_small_shape_steps.restype = None
    lib.sp_attn_set_small_shape_steps.argtypes = [i32]
    lib.sp_attn_last_error.restype = ctypes.c_char_p
    lib.sp_attn_last_error.argtypes = []
    lib.sp_attn_version.restype = ctypes.c_char_p
    lib.sp_attn_version.argtypes = []
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != SP_OK:
        raise SpAttnError(status, load_library().sp_attn_last_error().decode())


def sp_attn_segment_table(prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int]) -> list:
    """The segment table (list of ints) that a call with these host arrays hands to its kernels."""
    lib = load_library()
    n = ctypes.c_size_t(0)
    args = (len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat))
    st = lib.sp_attn_segment_table(*args, None, 0, ctypes.byref(n))
    if st != SP_ERR_WORKSPACE:
        _check(st)
    buf = (ctypes.c_int32 * n.value)()
    _check(lib.sp_attn_segment_table(*args, buf, n.value, ctypes.byref(n)))
    return list(buf)


def sp_attn_row_tile(prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int]):
    """(rows, steps_256, steps_128): the workgroup shape (256 or 128 query rows, eight or four waves) that a bf16 call on this packing
    takes, and the 64-key steps of one q head's row tiles of either size.  Host arithmetic only."""
    lib = load_library()
    rows = ctypes.c_int32(0)
    s256, s128 = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib.sp_attn_row_tile(len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat),
                                ctypes.byref(rows), ctypes.byref(s256), ctypes.byref(s128)))
    return rows.value, s256.value, s128.value


def sp_attn_dkdv_waves(prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int], n_q_heads: int,
                       n_kv_heads: int, flags: int = 0) -> int:
    """Waves per workgroup (8 or 4) of the dkdv pass of a bf16 backward on this packing.  Host arithmetic only."""
    waves = ctypes.c_int32(0)
    _check(load_library().sp_attn_dkdv_waves(len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), n_q_heads,
                                             n_kv_heads, flags, ctypes.byref(waves)))
    return waves.value


def sp_attn_pieces(prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int], n_q_heads: int, n_kv_heads: int,
                   flags: int = 0, of_rows: bool = False):
    """(list, sums, first_slot, n_slots): how a bf16 call with room for partial sums cuts the key tiles of its dkdv pass, or (of_rows) the key
    loops of its dq pass and of a forward of response rows.  Host arithmetic only."""
    words, info = (ctypes.c_uint32 * 1536)(), (ctypes.c_int32 * 4)()
    _check(load_library().sp_attn_pieces(len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), n_q_heads, n_kv_heads,
                                         flags, int(of_rows), words, len(words), info))
    return list(words[:info[0]]), list(words[info[0]:info[0] + info[1]]), info[2], info[3]


def sp_attn_f32_rows(prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int], n_q_heads: int, n_kv_heads: int,
                     head_dim: int, flags: int = 0):
    """Rows (keys) per workgroup, 16, 4 or 1, of the forward, the dq pass and the dkdv pass of a float32 call on this packing.  Host
    arithmetic only."""
    rows = (ctypes.c_int32 * 3)()
    _check(load_library().sp_attn_f32_rows(len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), n_q_heads, n_kv_heads,
                                           head_dim, flags, rows))
    return tuple(rows)


def _i32(xs: Sequence[int]):
    arr = (ctypes.c_int32 * max(1, len(xs)))(*xs)
    return arr


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return SP_BF16
    if t.dtype == torch.float32:
        return SP_F32
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def workspace_bytes(is_bwd: bool, total_tokens: int, n_groups: int, total_responses: int, n_q_heads: int,
                    n_kv_heads: int, head_dim: int, dtype_code: int) -> int:
    return load_library().sp_attn_workspace_bytes(int(is_bwd), total_tokens, n_groups, total_responses, n_q_heads,
                                                  n_kv_heads, head_dim, dtype_code)


def reserve_bytes(total_tokens: int, n_q_heads: int, head_dim: int, dtype_code: int) -> int:
    return load_library().sp_attn_reserve_bytes(total_tokens, n_q_heads, head_dim, dtype_code)


def row_parts_bytes(total_tokens: int, n_groups: int, n_q_heads: int, n_kv_heads: int, dtype_code: int) -> int:
    return load_library().sp_attn_row_parts_bytes(total_tokens, n_groups, n_q_heads, n_kv_heads, dtype_code)


def full_workspace_bytes(total_tokens: int, n_groups: int, total_responses: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                         dtype_code: int) -> int:
    return load_library().sp_attn_full_workspace_bytes(total_tokens, n_groups, total_responses, n_q_heads, n_kv_heads, head_dim,
                                                       dtype_code)


def kept_workspace_bytes(total_tokens: int, n_groups: int, total_responses: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                         dtype_code: int) -> int:
    return load_library().sp_attn_kept_workspace_bytes(total_tokens, n_groups, total_responses, n_q_heads, n_kv_heads, head_dim,
                                                       dtype_code)


def sums_bytes(total_tokens: int, n_groups: int, n_q_heads: int, n_kv_heads: int, dtype_code: int) -> int:
    return load_library().sp_attn_sums_bytes(total_tokens, n_groups, n_q_heads, n_kv_heads, dtype_code)


def _workspace(is_bwd, q, n_groups, n_resp, n_kv_heads, workspace, o=None, reserve=False):
    """The workspace tensor of a call.  When the caller passes none: a forward allocates one that also has
    room for the forward-to-backward reserve and for row parts and hangs it on the output tensor it returns (attribute
    ``_sp_workspace``); the backward that is given that output finds it there and passes it on, which is
    all the library needs to use the reserve.  A backward with a residual of its own allocates the same.  The attribute ``_sp_sums`` of such
    a workspace says that calls on it get room for partial sums (_sums), which is not kept.  Plumbing only:
    what the reserve is and whether it is valid is decided by the library."""
    if workspace is not None:
        return workspace
    if is_bwd:
        workspace = getattr(o, "_sp_workspace", None)
        if workspace is not None:
            return workspace
    T, Hq, d = q.shape
    code = _dtype_code(q)
    need = (load_library().sp_attn_kept_workspace_bytes(T, n_groups, n_resp, Hq, n_kv_heads, d, code) if reserve else
            workspace_bytes(is_bwd, T, n_groups, n_resp, Hq, n_kv_heads, d, code))
    workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    if reserve and code == SP_BF16:
        workspace._sp_sums = True
    if reserve and not is_bwd and o is not None:
        o._sp_workspace = workspace        # sized for the backward too
    return workspace


def _sums(workspace, q, n_groups, n_kv_heads, stream):
    """Room for the partial sums of one call on a workspace of _workspace()'s, or None."""
    if not getattr(workspace, "_sp_sums", False):
        return None
    need = sums_bytes(q.shape[0], n_groups, q.shape[1], n_kv_heads, _dtype_code(q))
    if need == 0:
        return None
    sums = torch.empty(need, dtype=torch.uint8, device=q.device)
    if stream is not None:
        sums.record_stream(stream)         # let go when the call returns, while its kernels may still run
    return sums


def sp_attn_fwd(q, k, v, prompt_len: int, resp_lens: Sequence[int], softmax_scale: float,
                o=None, lse=None, workspace=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Forward for one group.  q [T,Hq,d]; k, v [T,Hkv,d] on the GPU.  Returns (o, lse)."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    o = torch.empty_like(q) if o is None else o
    lse = torch.empty(Hq, T, dtype=torch.float32, device=q.device) if lse is None else lse
    workspace = _workspace(False, q, 1, len(resp_lens), Hkv, workspace, o=o, reserve=True)
    _check(lib.sp_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), prompt_len,
                           _i32(resp_lens), len(resp_lens), Hq, Hkv, d, softmax_scale, _dtype_code(q),
                           workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return o, lse


def sp_attn_bwd(q, k, v, o, lse, d_o, prompt_len: int, resp_lens: Sequence[int], softmax_scale: float,
                dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Backward for one group.  Returns (dq, dk, dv)."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    workspace = _workspace(True, q, 1, len(resp_lens), Hkv, workspace, o=o)
    sums = _sums(workspace, q, 1, Hkv, stream)
    tensors = (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr())
    shape = (Hq, Hkv, d, softmax_scale, _dtype_code(q))
    room = (workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if sums is None:
        _check(lib.sp_attn_bwd(*tensors, prompt_len, _i32(resp_lens), len(resp_lens), *shape, *room))
    else:
        _check(lib.sp_attn_bwd_batched_sums(*tensors, 1, _i32([prompt_len]), _i32([len(resp_lens)]), _i32(resp_lens), *shape,
                                            SP_BWD_STAGE_ALL, 0, None, sums.data_ptr(), sums.numel(), *room))
    return dq, dk, dv


def sp_attn_fwd_batched(q, k, v, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int],
                        softmax_scale: float, schedule: int = SP_SCHED_SHARED, o=None, lse=None, workspace=None,
                        stream=None):
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    o = torch.empty_like(q) if o is None else o
    lse = torch.empty(Hq, T, dtype=torch.float32, device=q.device) if lse is None else lse
    workspace = _workspace(False, q, len(prompt_lens), len(resp_lens_flat), Hkv, workspace, o=o, reserve=True)
    _check(lib.sp_attn_fwd_batched(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                   len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq, Hkv, d,
                                   softmax_scale, _dtype_code(q), schedule, workspace.data_ptr(),
                                   workspace.numel(), _stream_ptr(stream)))
    return o, lse


def sp_attn_fwd_multi(qs, ks, vs, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int],
                      softmax_scale: float, os=None, lses=None, workspace=None, stream=None):
    """Forward of several (q, k, v) sets that share one packing, in one launch.  Returns (os, lses)."""
    lib = load_library()
    n = len(qs)
    T, Hq, d = qs[0].shape
    Hkv = ks[0].shape[1]
    os = [torch.empty_like(q) for q in qs] if os is None else os
    lses = [torch.empty(Hq, T, dtype=torch.float32, device=qs[0].device) for _ in qs] if lses is None else lses
    workspace = _workspace(False, qs[0], len(prompt_lens), len(resp_lens_flat), Hkv, workspace)
    arr = lambda ts: (ctypes.c_void_p * max(1, len(ts)))(*[t.data_ptr() for t in ts])
    _check(lib.sp_attn_fwd_multi(n, arr(qs), arr(ks), arr(vs), arr(os), arr(lses), len(prompt_lens),
                                 _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq, Hkv, d, softmax_scale,
                                 _dtype_code(qs[0]), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return os, lses


def sp_attn_fwd_batched_ex(q, k, v, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int],
                           softmax_scale: float, flags: int, o=None, lse=None, workspace=None, stream=None,
                           schedule: int = SP_SCHED_SHARED, o_lo=None):
    """sp_attn_fwd_batched with a flags word (SP_FLAG_RESPONSE_ROWS).  Rows that the flags exclude keep
    whatever ``o`` / ``lse`` held."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    o = torch.empty_like(q) if o is None else o
    lse = torch.empty(Hq, T, dtype=torch.float32, device=q.device) if lse is None else lse
    workspace = _workspace(False, q, len(prompt_lens), len(resp_lens_flat), Hkv, workspace, o=o, reserve=o_lo is None)
    sums = _sums(workspace, q, len(prompt_lens), Hkv, stream) if flags & SP_FLAG_RESPONSE_ROWS else None
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), len(prompt_lens), _i32(prompt_lens), _i32(Gs),
            _i32(resp_lens_flat), Hq, Hkv, d, softmax_scale, _dtype_code(q), schedule, flags, None if o_lo is None else o_lo.data_ptr())
    room = (workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(lib.sp_attn_fwd_batched_ex(*args, *room) if sums is None else
           lib.sp_attn_fwd_batched_sums(*args, sums.data_ptr(), sums.numel(), *room))
    return o, lse


def sp_attn_bwd_batched_ex(q, k, v, o, lse, d_o, prompt_lens: Sequence[int], Gs: Sequence[int],
                           resp_lens_flat: Sequence[int], softmax_scale: float, flags: int, dq=None, dk=None, dv=None,
                           workspace=None, stream=None, stages: int = 7, o_lo=None):
    """sp_attn_bwd_batched with a flags word (SP_FLAG_RESPONSE_ROWS, SP_FLAG_ACCUMULATE_DKDV)."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    workspace = _workspace(True, q, len(prompt_lens), len(resp_lens_flat), Hkv, workspace, o=o, reserve=o_lo is not None)
    sums = _sums(workspace, q, len(prompt_lens), Hkv, stream)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(),
            dv.data_ptr(), len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq, Hkv, d, softmax_scale, _dtype_code(q),
            stages, flags, None if o_lo is None else o_lo.data_ptr())
    room = (workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(lib.sp_attn_bwd_batched_ex(*args, *room) if sums is None else
           lib.sp_attn_bwd_batched_sums(*args, sums.data_ptr(), sums.numel(), *room))
    return dq, dk, dv


def _loss_ws(T, n_groups, n_resp, device, workspace):
    if workspace is None:
        need = load_library().sp_attn_loss_workspace_bytes(T, n_groups, n_resp)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace


def sp_attn_logprob_fwd(logits, labels, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int],
                        logp=None, lse=None, workspace=None, stream=None):
    """Log-probability of labels[t] at every response row t of logits [T, V].  Returns (logp, lse);
    prompt rows keep whatever the output tensors held (zeros when allocated here)."""
    lib = load_library()
    T, V = logits.shape
    logp = torch.zeros(T, dtype=torch.float32, device=logits.device) if logp is None else logp
    lse = torch.zeros(T, dtype=torch.float32, device=logits.device) if lse is None else lse
    workspace = _loss_ws(T, len(prompt_lens), len(resp_lens_flat), logits.device, workspace)
    _check(lib.sp_attn_logprob_fwd(logits.data_ptr(), labels.data_ptr(), logp.data_ptr(), lse.data_ptr(), V,
                                   len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat),
                                   _dtype_code(logits), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return logp, lse


def sp_attn_logprob_bwd(logits, labels, lse, g, prompt_lens: Sequence[int], Gs: Sequence[int],
                        resp_lens_flat: Sequence[int], dlogits=None, workspace=None, stream=None):
    lib = load_library()
    T, V = logits.shape
    flags = 0
    if dlogits is None:
        # the launch itself zeroes the prompt rows when it covers every row of the tensor
        if logits.is_contiguous() and T == sum(prompt_lens) + sum(resp_lens_flat):
            dlogits, flags = torch.empty_like(logits), SP_FLAG_ZERO_PROMPT_ROWS
        else:
            dlogits = torch.zeros_like(logits)
    workspace = _loss_ws(T, len(prompt_lens), len(resp_lens_flat), logits.device, workspace)
    _check(lib.sp_attn_logprob_bwd_ex(logits.data_ptr(), labels.data_ptr(), lse.data_ptr(), g.data_ptr(),
                                      dlogits.data_ptr(), V, len(prompt_lens), _i32(prompt_lens), _i32(Gs),
                                      _i32(resp_lens_flat), _dtype_code(logits), flags, workspace.data_ptr(),
                                      workspace.numel(), _stream_ptr(stream)))
    return dlogits


def sp_attn_grpo_loss(logp, logp_old, logp_ref, adv, prompt_lens: Sequence[int], Gs: Sequence[int],
                      resp_lens_flat: Sequence[int], eps_low: float = 0.2, eps_high: float = 0.2, beta: float = 0.02,
                      g=None, workspace=None, stream=None):
    """GRPO objective over the response rows.  Returns (loss [1], g [T] = dloss/dlogp)."""
    lib = load_library()
    T = logp.shape[0]
    loss = torch.zeros(1, dtype=torch.float32, device=logp.device)
    g = torch.zeros(T, dtype=torch.float32, device=logp.device) if g is None else g
    workspace = _loss_ws(T, len(prompt_lens), len(resp_lens_flat), logp.device, workspace)
    _check(lib.sp_attn_grpo_loss(logp.data_ptr(), logp_old.data_ptr(), logp_ref.data_ptr(), adv.data_ptr(), eps_low,
                                 eps_high, beta, loss.data_ptr(), g.data_ptr(), len(prompt_lens), _i32(prompt_lens),
                                 _i32(Gs), _i32(resp_lens_flat), workspace.data_ptr(), workspace.numel(),
                                 _stream_ptr(stream)))
    return loss, g


def sp_attn_rope(x, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int], rope_base: float,
                 inverse: bool = False, out=None, workspace=None, stream=None):
    """Rotary embedding of x [T, H, d] at the restarted position indices; returns the rotated tensor
    (``out`` may be x itself)."""
    lib = load_library()
    T, H, d = x.shape
    out = torch.empty_like(x) if out is None else out
    if workspace is None:
        need = workspace_bytes(False, T, len(prompt_lens), len(resp_lens_flat), H, H, d, _dtype_code(x))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    _check(lib.sp_attn_rope(x.data_ptr(), out.data_ptr(), H, int(inverse), len(prompt_lens), _i32(prompt_lens),
                            _i32(Gs), _i32(resp_lens_flat), d, float(rope_base), _dtype_code(x),
                            workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return out


def sp_attn_rope_qk(q, k, prompt_lens: Sequence[int], Gs: Sequence[int], resp_lens_flat: Sequence[int], rope_base: float,
                    inverse: bool = False, q_out=None, k_out=None, workspace=None, stream=None):
    """Rotary embedding of q [T, Hq, d] and k [T, Hkv, d] in one launch; returns (q_out, k_out)."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    q_out = torch.empty_like(q) if q_out is None else q_out
    k_out = torch.empty_like(k) if k_out is None else k_out
    if workspace is None:
        need = workspace_bytes(False, T, len(prompt_lens), len(resp_lens_flat), Hq, Hq, d, _dtype_code(q))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    _check(lib.sp_attn_rope_qk(q.data_ptr(), q_out.data_ptr(), Hq, k.data_ptr(), k_out.data_ptr(), Hkv, int(inverse),
                               len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), d, float(rope_base),
                               _dtype_code(q), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return q_out, k_out


def sp_attn_bwd_batched(q, k, v, o, lse, d_o, prompt_lens: Sequence[int], Gs: Sequence[int],
                        resp_lens_flat: Sequence[int], softmax_scale: float, dq=None, dk=None, dv=None,
                        workspace=None, stream=None):
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    workspace = _workspace(True, q, len(prompt_lens), len(resp_lens_flat), Hkv, workspace, o=o)
    sums = _sums(workspace, q, len(prompt_lens), Hkv, stream)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(),
            dv.data_ptr(), len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq, Hkv, d, softmax_scale, _dtype_code(q))
    room = (workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(lib.sp_attn_bwd_batched(*args, *room) if sums is None else
           lib.sp_attn_bwd_batched_sums(*args, SP_BWD_STAGE_ALL, 0, None, sums.data_ptr(), sums.numel(), *room))
    return dq, dk, dv


def sp_attn_probe_atomic_add(buf, rows: int, heads: int, steps: int, n_blocks: int = 512, layout: int = 0, stream=None) -> int:
    """Enqueue the atomic-add measurement loop; returns the bytes the launch adds."""
    st = load_library().sp_attn_probe_atomic_add(buf.data_ptr(), rows, heads, steps, n_blocks, layout, _stream_ptr(stream))
    if st != SP_OK:
        raise SpAttnError(st, "sp_attn_probe_atomic_add: invalid argument or launch failure")
    return n_blocks * steps * 32768


def set_small_shape_steps(steps: int) -> None:
    """Threshold (mean 64-key steps per 256-row workgroup) below which calls take the 128-row kernel shape."""
    load_library().sp_attn_set_small_shape_steps(steps)


def sp_attn_mfma_ceiling(lds_operands: int, a, b, iters: int, out, n_blocks: int = 256, stream=None) -> float:
    """Enqueue the MFMA-only measurement loop; returns the FLOPs the launch executes."""
    lib = load_library()
    st = lib.sp_attn_mfma_ceiling(lds_operands, a.data_ptr(), b.data_ptr(), iters, n_blocks, out.data_ptr(),
                                  _stream_ptr(stream))
    if st != SP_OK:
        raise SpAttnError(st, "sp_attn_mfma_ceiling: invalid argument or launch failure")
    return float(n_blocks) * 8 * iters * 16 * 32768.0


def sp_attn_bwd_batched_static(q, k, v, o, lse, d_o, dq, dk, dv, prompt_lens: Sequence[int], Gs: Sequence[int],
                               resp_lens_flat: Sequence[int], softmax_scale: float, stream=None) -> None:
    """sp_attn_bwd_batched on the library's built-in device scratch: no workspace, and nothing is
    allocated (the caller passes every output)."""
    lib = load_library()
    T, Hq, d = q.shape
    _check(lib.sp_attn_bwd_batched_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                          d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                          len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq,
                                          k.shape[1], d, softmax_scale, _dtype_code(q), _stream_ptr(stream)))


def sp_attn_bwd_batched_stages(q, k, v, o, lse, d_o, prompt_lens: Sequence[int], Gs: Sequence[int],
                               resp_lens_flat: Sequence[int], softmax_scale: float, stages: int, workspace,
                               dq=None, dk=None, dv=None, stream=None) -> None:
    """Enqueue a subset of the backward stages (SP_BWD_STAGE_* bits).  The caller passes the
    workspace, because D written by the ROWSUM stage is read by the other two."""
    lib = load_library()
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    ptr = lambda x: None if x is None else x.data_ptr()
    sums = _sums(workspace, q, len(prompt_lens), Hkv, stream)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), ptr(o), lse.data_ptr(), d_o.data_ptr(), ptr(dq), ptr(dk), ptr(dv),
            len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat), Hq, Hkv, d, softmax_scale, _dtype_code(q), stages)
    room = (workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(lib.sp_attn_bwd_batched_stages(*args, *room) if sums is None else
           lib.sp_attn_bwd_batched_sums(*args, 0, None, sums.data_ptr(), sums.numel(), *room))


# ---- rollout: paged cache, attention of one new token per sequence, adjusted logits ----------------------------------

def _refuse(message: str):
    raise SpAttnError(SP_ERR_INVALID_ARG, message)


def _is(t, dtype, shape, index) -> bool:
    """Whether t is what a kernel takes its pointer for.  `index`: of the GPU, -1 for host memory."""
    return t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous()


def _need(name, t, dtype, shape, index):
    if not _is(t, dtype, shape, index):
        _refuse(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}; "
                f"expected {dtype} {tuple(shape)} on {'the host' if index < 0 else f'cuda:{index}'}, contiguous")


def _room(workspace, index):
    """Refuses a workspace whose bytes a kernel would not find behind its pointer."""
    if workspace is not None and (workspace.get_device() != index or not workspace.is_contiguous()):
        _refuse(f"workspace: {tuple(workspace.shape)} on {workspace.device}{'' if workspace.is_contiguous() else ', not contiguous'}; "
                f"expected contiguous memory on {'the host' if index < 0 else f'cuda:{index}'}")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _placed(f):
    """Runs f(raw stream, ...) on the device of its tensors (`index`) and on the caller's stream, so that what it allocates belongs there."""
    def run(index, stream, *args):
        if index < 0:
            _refuse("the tensors are not on a GPU")
        if stream is None:
            if index == _current_device():
                return f(_raw_stream(index), *args)
            with torch.cuda.device(index):
                return f(_raw_stream(index), *args)
        if stream.device_index != index:
            _refuse(f"the stream is on cuda:{stream.device_index}, the tensors are on cuda:{index}")
        with torch.cuda.stream(stream):
            return f(stream.cuda_stream, *args)
    return run


class KvCache:
    """A paged cache: k and v [n_pages, n_kv_heads, page_size, head_dim], contiguous, bf16 or float32.  A call takes the memory that they have
    then; their shape and type stay those of the construction."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 4:
            _refuse(f"k: {tuple(k.shape)}, expected [n_pages, n_kv_heads, page_size, head_dim]")
        self.index = k.get_device()
        _need("k", k, k.dtype, k.shape, self.index)
        _need("v", v, k.dtype, k.shape, self.index)
        self.k, self.v = k, v
        self.dtype, self.device = k.dtype, k.device
        n_pages, self.n_kv_heads, page_size, self.head_dim = k.shape
        self.code = _dtype_code(k)
        self._shape = k.shape
        self._struct = _KvCacheStruct(k.data_ptr(), v.data_ptr(), n_pages, page_size, self.n_kv_heads, self.head_dim, self.code)
        self._pointer = ctypes.pointer(self._struct)

    @property
    def _ref(self):
        k, v, struct = self.k, self.v, self._struct
        at_k, at_v = k.data_ptr(), v.data_ptr()
        if not (at_k == struct.k and at_v == struct.v and k.shape == v.shape == self._shape and k.dtype is v.dtype is self.dtype and
                k.is_contiguous() and v.is_contiguous()):
            _need("k", k, self.dtype, self._shape, self.index)
            _need("v", v, self.dtype, self._shape, self.index)
            struct.k, struct.v = at_k, at_v
        return self._pointer


class _AllLayersError(SpAttnError, AttributeError):
    """A call for one layer was given the caches of all of them."""


class KvLayers:
    """The caches of all layers of a model: k and v [n_layers, n_pages, n_kv_heads, page_size, head_dim], each layer contiguous, whose sequences have the
    same tables in every layer.  layers[i] is the KvCache of layer i.  Memory, shape and type as for KvCache."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 5 or k.shape[0] == 0:
            _refuse(f"k: {tuple(k.shape)}, expected [n_layers, n_pages, n_kv_heads, page_size, head_dim]")
        # (no attributes of a single layer's cache: a call for one layer refuses all of them)
        self.index, self._dtype, self.device = k.get_device(), k.dtype, k.device
        self._shape, self._strides = k.shape, k.stride()
        self._check(k, v)
        self.k, self.v = k, v
        self.n_layers, n_pages, heads, page_size, head_dim = k.shape
        self._stride = self._strides[0]
        self._struct = _KvCacheStruct(k.data_ptr(), v.data_ptr(), n_pages, page_size, heads, head_dim, _dtype_code(k))
        self._pointer = ctypes.pointer(self._struct)

    def __getattr__(self, name):
        if name in ("dtype", "code", "n_kv_heads", "head_dim"):
            raise _AllLayersError(SP_ERR_INVALID_ARG, "the call takes the cache of one layer: layers[i] of KvLayers")
        raise AttributeError(f"KvLayers has no attribute {name!r}")

    def __len__(self) -> int:
        return self.n_layers

    def __getitem__(self, i: int) -> KvCache:
        return KvCache(self.k[i], self.v[i])

    def _check(self, k, v):
        for name, t in (("k", k), ("v", v)):
            if t.shape != self._shape or t.stride() != self._strides or not t[0].is_contiguous() or (t.shape[0] > 1 and t.stride(0) < t[0].numel()):
                _refuse(f"{name}: {tuple(t.shape)} with strides {t.stride()}, expected {tuple(self._shape)} with strides {self._strides}, each layer contiguous "
                        "and behind the last")
            _need(name, t[0], self._dtype, self._shape[1:], self.index)

    @property
    def _ref(self):
        k, v, struct = self.k, self.v, self._struct
        at_k, at_v = k.data_ptr(), v.data_ptr()
        if not (at_k == struct.k and at_v == struct.v and k.shape == v.shape == self._shape and k.dtype is v.dtype is self._dtype and
                k.stride() == v.stride() == self._strides):
            self._check(k, v)
            struct.k, struct.v = at_k, at_v
        return self._pointer


class LogitRules:
    """How logits are adjusted ahead of a draw: bias (float32 [vocab] or None), then penalties, then the temperature."""

    def __init__(self, repetition: float = 1.0, presence: float = 0.0, frequency: float = 0.0, temperature: float = 1.0, bias=None):
        if bias is not None:
            if bias.dim() != 1:
                _refuse(f"bias: {tuple(bias.shape)}, expected [vocab]")
            _need("bias", bias, torch.float32, bias.shape, bias.get_device())
        self.bias = bias
        self._struct = _LogitRulesStruct(repetition, presence, frequency, temperature, None if bias is None else bias.data_ptr())
        self._ref = ctypes.pointer(self._struct)

    def _fits(self, vocab, index):
        if self.bias is not None:
            _need("bias", self.bias, torch.float32, (vocab,), index)
        self._struct.bias = _ptr(self.bias)            # where it lies now


def _ptr(t):
    return None if t is None else t.data_ptr()


def _token_stride(name, t, cache, heads) -> int:
    """Elements from token to token of [T, heads, d], whose heads are contiguous within a token."""
    d, shape = cache.head_dim, t.shape
    if t.dtype is not cache.dtype or t.get_device() != cache.index or shape[1:] != (heads, d):
        _refuse(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {cache.dtype} [tokens, {heads}, {d}] on {cache.device}")
    at, head, one = t.stride()
    if shape[0] and (one != 1 or (heads > 1 and head != d)):
        _refuse(f"{name}: the heads of a token are not contiguous (strides {t.stride()})")
    return at if shape[0] > 1 else heads * d


def sp_attn_cache_append(cache: KvCache, k, v, tables, lens, rope_base: float, q=None, new_lens: Optional[Sequence[int]] = None,
                         pos_base=None, q_out=None, k_out=None, lens_out=None, stream=None):
    """Append the rotated keys k and the values v of new tokens [T, n_kv_heads, d] to the cache.  Sequence s brings new_lens[s] tokens
    (host integers; None: one each), which become its tokens lens[s], lens[s] + 1, ... in the pages tables[s].  q [T, n_q_heads, d] is rotated
    along (into q_out), and the rotated keys also go to k_out where that is given.  k, v and q may be parts of one
    projection's output.  Returns (q_out, lens_out); q_out is None without q."""
    index, hkv, d, int32 = cache.index, cache.n_kv_heads, cache.head_dim, torch.int32
    ks, vs = _token_stride("k", k, cache, hkv), _token_stride("v", v, cache, hkv)
    T, n_seqs = k.shape[0], lens.shape[0]
    if v.shape[0] != T or T != (n_seqs if new_lens is None else sum(new_lens)) or (new_lens is not None and len(new_lens) != n_seqs):
        _refuse(f"{T} keys, {v.shape[0]} values and {n_seqs} sequences do not fit the new tokens")
    _need("lens", lens, int32, (n_seqs,), index)
    if tables.dim() != 2:
        _refuse(f"tables: {tuple(tables.shape)}, expected [sequences, pages]")
    _need("tables", tables, int32, (n_seqs, tables.shape[1]), index)
    if pos_base is not None:
        _need("pos_base", pos_base, int32, (n_seqs,), index)
    hq, qs = 0, 0
    if q is not None:
        hq = q.shape[1]
        qs = _token_stride("q", q, cache, hq)
        if q.shape[0] != T:
            _refuse(f"q has {q.shape[0]} tokens, k has {T}")
        if q_out is not None:
            _need("q_out", q_out, cache.dtype, (T, hq, d), index)
    elif q_out is not None:
        _refuse("q_out without q")
    if k_out is not None:
        _need("k_out", k_out, cache.dtype, (T, hkv, d), index)
    if lens_out is not None:
        _need("lens_out", lens_out, int32, (n_seqs,), index)
    return _append(index, stream, cache, q, qs, q_out, hq, k, ks, k_out, v, vs, n_seqs, new_lens, tables, lens, pos_base, lens_out, rope_base)


@_placed
def _append(raw, cache, q, qs, q_out, hq, k, ks, k_out, v, vs, n_seqs, new_lens, tables, lens, pos_base, lens_out, rope_base):
    if q is not None and q_out is None:
        q_out = torch.empty(k.shape[0], hq, cache.head_dim, dtype=cache.dtype, device=cache.device)
    if lens_out is None:
        lens_out = torch.empty_like(lens)
    if n_seqs == 0:
        return q_out, lens_out
    at = (_ptr(q), qs, _ptr(q_out), hq, k.data_ptr(), ks, _ptr(k_out), v.data_ptr(), vs)
    if k.shape[0] == 0:                    # the pointers of empty tensors are null, and no token is read or written
        at = (None, 0, None, 0, cache.k.data_ptr(), ks, None, cache.v.data_ptr(), vs)
    _check(load_library().sp_attn_cache_append(cache._ref, *at, n_seqs, None if new_lens is None else _i32(new_lens), tables.data_ptr(),
                                               tables.shape[1], lens.data_ptr(), _ptr(pos_base), lens_out.data_ptr(), rope_base, raw))
    return q_out, lens_out


@functools.lru_cache(maxsize=64)
def decode_workspace_bytes(n_groups: int, n_seqs: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype_code: int) -> int:
    return load_library().sp_attn_decode_workspace_bytes(n_groups, n_seqs, n_q_heads, n_kv_heads, head_dim, dtype_code)


def _pages_of(name, tables, lens, rows, index):
    """(pointer, width, pointer of the lengths) of a table, which may be None or have no columns."""
    if lens is not None:
        _need(name + "_lens", lens, torch.int32, (rows,), index)
    if tables is None:
        return None, 0, _ptr(lens)
    if tables.dim() != 2:
        _refuse(f"{name}_tables: {tuple(tables.shape)}, expected [rows, pages]")
    width = tables.shape[1]
    _need(name + "_tables", tables, torch.int32, (rows, width), index)
    return (tables.data_ptr() if width else None), width, _ptr(lens)


def sp_attn_decode(cache: KvCache, q, Gs: Optional[Sequence[int]], prompt_tables, prompt_lens, resp_tables, resp_lens, softmax_scale: float,
                   o=None, lse=None, workspace=None, stream=None):
    """Attention of one new token per sequence.  Row s of q [n_seqs, n_q_heads, d] attends to its group's prompt and to the first
    resp_lens[s] tokens of its own.  Gs: sequences of each group (host integers), None: one each.  prompt_tables [n_groups, width] and
    prompt_lens may be None (no shared prompts).  Returns (o, lse [n_q_heads, n_seqs])."""
    index = cache.index
    if q.dim() != 3:
        _refuse(f"q: {tuple(q.shape)}, expected [sequences, heads, {cache.head_dim}]")
    n_seqs, hq, d = q.shape
    _need("q", q, cache.dtype, (n_seqs, hq, cache.head_dim), index)
    n_groups = n_seqs if Gs is None else len(Gs)
    if (prompt_tables is None) != (prompt_lens is None):
        _refuse("prompt_tables and prompt_lens go together")
    prompt = _pages_of("prompt", prompt_tables, prompt_lens, n_groups, index)
    resp = _pages_of("resp", resp_tables, resp_lens, n_seqs, index)
    if o is not None:
        _need("o", o, cache.dtype, (n_seqs, hq, d), index)
    if lse is not None:
        _need("lse", lse, torch.float32, (hq, n_seqs), index)
    _room(workspace, index)
    return _decode(index, stream, cache, q, o, lse, hq, n_groups, n_seqs, Gs, prompt, resp, softmax_scale, workspace)


@_placed
def _decode(raw, cache, q, o, lse, hq, n_groups, n_seqs, Gs, prompt, resp, softmax_scale, workspace):
    lib = load_library()
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(hq, n_seqs, dtype=torch.float32, device=cache.device)
    if workspace is None:
        need = decode_workspace_bytes(n_groups, n_seqs, hq, cache.n_kv_heads, cache.head_dim, cache.code)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=cache.device)
    pt, pw, pl = prompt
    rt, rw, rl = resp
    _check(lib.sp_attn_decode(cache._ref, q.data_ptr(), o.data_ptr(), lse.data_ptr(), hq, n_groups, n_seqs, None if Gs is None else _i32(Gs),
                              pt, pw, pl if pw else None, rt, rw, rl, softmax_scale, workspace.data_ptr(), workspace.nbytes, raw))
    return o, lse


@functools.lru_cache(maxsize=64)
def tree_decode_workspace_bytes(n_groups: int, n_seqs: int, total_new: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype_code: int) -> int:
    return load_library().sp_attn_tree_decode_workspace_bytes(n_groups, n_seqs, total_new, n_q_heads, n_kv_heads, head_dim, dtype_code)


def sp_attn_tree_decode(cache: KvCache, q, Gs: Optional[Sequence[int]], new_lens: Sequence[int], ancestors, prompt_tables, prompt_lens, resp_tables,
                        resp_lens, softmax_scale: float, o=None, lse=None, workspace=None, stream=None):
    """Attention of new_lens[s] drafted tokens per sequence (host integers).  Row t of q [T, n_q_heads, d], sequence behind sequence, attends to its group's
    prompt, to its sequence's first resp_lens[s] - new_lens[s] tokens, and to those of its drafted tokens, the last of these resp_lens[s], whose bits are set in row t of
    ancestors [T, words] (int32 or uint32, bit m % 32 of word m / 32: drafted token m); None: to its own and those ahead of it.  The rest as
    sp_attn_decode.  Returns (o, lse [n_q_heads, T])."""
    index = cache.index
    if q.dim() != 3:
        _refuse(f"q: {tuple(q.shape)}, expected [tokens, heads, {cache.head_dim}]")
    T, hq, d = q.shape
    n_seqs = len(new_lens)
    _need("q", q, cache.dtype, (T, hq, cache.head_dim), index)
    if T != sum(new_lens):
        _refuse(f"q has {T} tokens, new_lens add up to {sum(new_lens)}")
    n_groups = n_seqs if Gs is None else len(Gs)
    if (prompt_tables is None) != (prompt_lens is None):
        _refuse("prompt_tables and prompt_lens go together")
    rows = _mask_rows(ancestors, T, index)
    prompt = _pages_of("prompt", prompt_tables, prompt_lens, n_groups, index)
    resp = _pages_of("resp", resp_tables, resp_lens, n_seqs, index)
    if o is not None:
        _need("o", o, cache.dtype, (T, hq, d), index)
    if lse is not None:
        _need("lse", lse, torch.float32, (hq, T), index)
    _room(workspace, index)
    return _tree_decode(index, stream, cache, q, o, lse, n_groups, n_seqs, Gs, new_lens, rows, prompt, resp, softmax_scale, workspace)


@_placed
def _tree_decode(raw, cache, q, o, lse, n_groups, n_seqs, Gs, new_lens, mask, prompt, resp, softmax_scale, workspace):
    T, hq, _ = q.shape
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(hq, T, dtype=torch.float32, device=cache.device)
    if workspace is None:
        need = tree_decode_workspace_bytes(n_groups, n_seqs, T, hq, cache.n_kv_heads, cache.head_dim, cache.code)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=cache.device)
    pt, pw, pl = prompt
    rt, rw, rl = resp
    at = (q.data_ptr(), o.data_ptr(), lse.data_ptr()) if T else (cache.k.data_ptr(),) * 3      # the pointers of empty tensors are null, and no row is read or written
    ancestors, words = mask
    _check(load_library().sp_attn_tree_decode(cache._ref, *at, hq, n_groups, n_seqs, None if Gs is None else _i32(Gs), _i32(new_lens),
                                              ancestors, words if ancestors else 0, pt, pw, pl if pw else None, rt, rw, rl, softmax_scale,
                                              workspace.data_ptr(), workspace.nbytes, raw))
    return o, lse


def _layers(cache):
    """(number of layers, elements from one to the next) of a KvCache or of KvLayers."""
    return (cache.n_layers, cache._stride) if isinstance(cache, KvLayers) else (1, 0)


def _rows_of(name, t, dtype, rows, index):
    """Width of [rows, width]."""
    if t.dim() != 2:
        _refuse(f"{name}: {tuple(t.shape)}, expected two dimensions")
    _need(name, t, dtype, (rows, t.shape[1]), index)
    return t.shape[1]


def sp_attn_cache_keep(cache, tables, lens, kept, n_kept, lens_out=None, stream=None):
    """Of the tokens behind the first lens[s] of sequence s, those numbered kept[s, :n_kept[s]] (ascending) become its next ones, in every layer of the cache
    (KvCache or KvLayers).  Returns lens_out, lens + n_kept."""
    index, int32, n_seqs = cache.index, torch.int32, lens.shape[0]
    _need("lens", lens, int32, (n_seqs,), index)
    _need("n_kept", n_kept, int32, (n_seqs,), index)
    _rows_of("tables", tables, int32, n_seqs, index)
    _rows_of("kept", kept, int32, n_seqs, index)
    if lens_out is not None:
        _need("lens_out", lens_out, int32, (n_seqs,), index)
    return _keep(index, stream, cache, tables, lens, kept, n_kept, lens_out)


@_placed
def _keep(raw, cache, tables, lens, kept, n_kept, lens_out):
    n_seqs = lens.shape[0]
    if lens_out is None:
        lens_out = torch.empty_like(lens)
    if n_seqs:
        _check(load_library().sp_attn_cache_keep(cache._ref, *_layers(cache), n_seqs, tables.data_ptr(), tables.shape[1], lens.data_ptr(),
                                                 kept.data_ptr() if kept.shape[1] else None, kept.shape[1], n_kept.data_ptr(), lens_out.data_ptr(), raw))
    return lens_out


@functools.lru_cache(maxsize=64)
def pages_workspace_bytes(n_pages: int, n_seqs: int) -> int:
    return load_library().sp_attn_pages_workspace_bytes(n_pages, n_seqs)


def _pages_workspace(n_pages, n_seqs, device, workspace):
    return torch.empty(max(256, pages_workspace_bytes(n_pages, n_seqs)), dtype=torch.uint8, device=device) if workspace is None else workspace


def sp_attn_pages_fit(refs, page_size: int, tables, lens, missing=None, workspace=None, stream=None):
    """Fits tables [n_seqs, width] to sequences of lens[s] tokens: pages behind go back, missing ones ahead come from the free ones, those with refs [n_pages] of 0, lowest
    first.  tables and refs change in place.  Returns missing [1], how many places got no page."""
    index, int32 = refs.get_device(), torch.int32
    if refs.dim() != 1:
        _refuse(f"refs: {tuple(refs.shape)}, expected [n_pages]")
    _need("refs", refs, int32, refs.shape, index)
    n_seqs = lens.shape[0]
    _need("lens", lens, int32, (n_seqs,), index)
    _rows_of("tables", tables, int32, n_seqs, index)
    if missing is not None:
        _need("missing", missing, int32, (1,), index)
    _room(workspace, index)
    return _fit(index, stream, refs, page_size, tables, lens, missing, workspace)


@_placed
def _fit(raw, refs, page_size, tables, lens, missing, workspace):
    n_seqs = lens.shape[0]
    if missing is None:
        missing = torch.empty(1, dtype=torch.int32, device=refs.device)
    if n_seqs == 0:
        return missing.zero_()
    workspace = _pages_workspace(refs.shape[0], n_seqs, refs.device, workspace)
    _check(load_library().sp_attn_pages_fit(refs.data_ptr(), refs.shape[0], page_size, n_seqs, tables.data_ptr(), tables.shape[1], lens.data_ptr(),
                                            missing.data_ptr(), workspace.data_ptr(), workspace.nbytes, raw))
    return missing


def sp_attn_cache_fork(cache, refs, parents, src_tables, src_lens, tables, lens_out=None, workspace=None, stream=None):
    """Sequence s of tables [n_seqs, width] becomes a copy of sequence parents[s] of src_tables, in every layer of the cache (KvCache or KvLayers): whole pages are shared, the
    last tokens copied to a free page.  tables and refs [n_pages] change in place.  Returns lens_out (-1 where no page was left; rows whose parent is none keep what
    it held, -1 when it is allocated here)."""
    index, int32 = cache.index, torch.int32
    _need("refs", refs, int32, (cache._shape[-4],), index)
    n_seqs, n_src = parents.shape[0], src_lens.shape[0]
    _need("parents", parents, int32, (n_seqs,), index)
    _need("src_lens", src_lens, int32, (n_src,), index)
    _rows_of("src_tables", src_tables, int32, n_src, index)
    _rows_of("tables", tables, int32, n_seqs, index)
    if lens_out is not None:
        _need("lens_out", lens_out, int32, (n_seqs,), index)
    _room(workspace, index)
    return _fork(index, stream, cache, refs, parents, src_tables, src_lens, tables, lens_out, workspace)


@_placed
def _fork(raw, cache, refs, parents, src_tables, src_lens, tables, lens_out, workspace):
    n_seqs, flags = parents.shape[0], 0
    if lens_out is None:
        lens_out, flags = torch.empty_like(parents), SP_FLAG_MARK_ORPHANS
    if n_seqs == 0:
        return lens_out
    workspace = _pages_workspace(refs.shape[0], n_seqs, cache.device, workspace)
    _check(load_library().sp_attn_cache_fork(cache._ref, *_layers(cache), refs.data_ptr(), n_seqs, parents.data_ptr(), src_lens.shape[0], src_tables.data_ptr(),
                                             src_tables.shape[1], src_lens.data_ptr(), tables.data_ptr(), tables.shape[1], lens_out.data_ptr(), flags,
                                             workspace.data_ptr(), workspace.nbytes, raw))
    return lens_out


def _logit_stride(name, t, shape, dtype, index) -> int:
    """Elements from row to row of logits, whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        _refuse(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtype} {tuple(shape)} beside the logits")
    if t.stride(1) != 1 and t.shape[1] > 1:
        _refuse(f"{name}: the elements of a row are not contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _mask_rows(mask, rows, index):
    if mask is None:
        return None, 0
    if mask.dtype not in (torch.int32, torch.uint32) or mask.dim() != 2:
        _refuse(f"mask: {mask.dtype} {tuple(mask.shape)}, expected rows of int32 or uint32 words")
    _need("mask", mask, mask.dtype, (rows, mask.shape[1]), index)
    if rows and not mask.shape[1]:                                       # (its null address would read as no mask)
        _refuse(f"mask: {tuple(mask.shape)}, rows of no words")
    return mask.data_ptr(), mask.shape[1]


def _history(name, tokens, lens, rows, index):
    """(pointer, stride, pointer of the lengths) of rows of token ids, which may be missing."""
    if tokens is None and lens is None:
        return None, 0, None
    if tokens is None or lens is None:
        _refuse(f"{name}_tokens and {name}_lens go together")
    if tokens.dim() != 2:
        _refuse(f"{name}_tokens: {tuple(tokens.shape)}, expected [rows, tokens]")
    stride = tokens.shape[1]
    _need(name + "_tokens", tokens, torch.int32, (rows, stride), index)
    _need(name + "_lens", lens, torch.int32, (rows,), index)
    return (tokens.data_ptr(), stride, lens.data_ptr()) if stride else (None, 0, None)


def sp_attn_adjust_logits(logits, rules: LogitRules, Gs: Optional[Sequence[int]], prompt_tokens, prompt_lens, resp_tokens, resp_lens,
                          mask=None, out=None, stream=None):
    """Adjusted logits [n_seqs, vocab] of one row per sequence.  Its history is the first prompt_lens[g] ids of its group's row of
    prompt_tokens [n_groups, .] and the first resp_lens[s] ids of its row of resp_tokens [n_seqs, .] (either pair may be None).  mask [n_seqs, words]:
    bit v % 32 of word v / 32 allows id v.  ``out`` may be logits itself."""
    index = logits.get_device()
    n_seqs, vocab = logits.shape
    n_groups = n_seqs if Gs is None else len(Gs)
    stride = _logit_stride("logits", logits, logits.shape, logits.dtype, index)
    out_stride = vocab if out is None else _logit_stride("out", out, logits.shape, logits.dtype, index)
    rules._fits(vocab, index)
    rows = _mask_rows(mask, n_seqs, index)
    prompt, resp = _history("prompt", prompt_tokens, prompt_lens, n_groups, index), _history("resp", resp_tokens, resp_lens, n_seqs, index)
    return _adjust(index, stream, logits, stride, out, out_stride, rules, rows, n_groups, n_seqs, Gs, prompt, resp)


@_placed
def _adjust(raw, logits, stride, out, out_stride, rules, mask, n_groups, n_seqs, Gs, prompt, resp):
    vocab = logits.shape[1]
    if out is None:
        out = torch.empty(n_seqs, vocab, dtype=logits.dtype, device=logits.device)
    _check(load_library().sp_attn_adjust_logits(logits.data_ptr(), stride, out.data_ptr(), out_stride, vocab, rules._ref, *mask, n_groups, n_seqs,
                                                None if Gs is None else _i32(Gs), *prompt, *resp, _dtype_code(logits), raw))
    return out


def _adjusted_args(logits, labels, tokens, rules, prompt_lens, Gs, resp_lens_flat, mask, workspace):
    """What the forward and the backward check alike; returns the device's index and the mask's pointer and stride."""
    if len(Gs) != len(prompt_lens) or sum(Gs) != len(resp_lens_flat) or min(Gs, default=0) < 0:      # the library takes no lengths of these lists
        _refuse(f"{len(prompt_lens)} prompts, groups of {list(Gs)} responses and {len(resp_lens_flat)} lengths of responses do not fit")
    index = logits.get_device()
    T, V = logits.shape
    _need("logits", logits, logits.dtype, (T, V), index)
    if T != sum(prompt_lens) + sum(resp_lens_flat):
        _refuse(f"logits have {T} rows, the pack has {sum(prompt_lens) + sum(resp_lens_flat)}")
    _need("labels", labels, torch.int32, (T,), index)
    _need("tokens", tokens, torch.int32, (T,), index)
    rules._fits(V, index)
    _room(workspace, index)
    return index, _mask_rows(mask, T, index)


@functools.lru_cache(maxsize=64)
def _adjusted_workspace_bytes(T, n_groups, n_resp, V) -> int:
    return load_library().sp_attn_adjusted_logprob_workspace_bytes(T, n_groups, n_resp, V)


def _adjusted_workspace(logits, prompt_lens, resp_lens_flat, workspace):
    if workspace is not None:
        return workspace
    T, V = logits.shape
    need = _adjusted_workspace_bytes(T, len(prompt_lens), len(resp_lens_flat), V)
    return torch.empty(max(256, need), dtype=torch.uint8, device=logits.device)


def sp_attn_adjusted_logprob_fwd(logits, labels, tokens, rules: LogitRules, prompt_lens: Sequence[int], Gs: Sequence[int],
                                 resp_lens_flat: Sequence[int], mask=None, flags: int = 0, logp=None, lse=None, workspace=None, stream=None):
    """Log-probability of labels[t] under the adjusted distribution at every response row t of logits [T, V]; tokens [T] are the pack's ids.
    mask [T, words] as in sp_attn_adjust_logits.  Returns (logp, lse); prompt rows keep whatever the output tensors held (zeros when
    allocated here)."""
    index, rows = _adjusted_args(logits, labels, tokens, rules, prompt_lens, Gs, resp_lens_flat, mask, workspace)
    for name, t in (("logp", logp), ("lse", lse)):
        if t is not None:
            _need(name, t, torch.float32, (logits.shape[0],), index)
    return _adjusted_fwd(index, stream, logits, labels, tokens, rules, prompt_lens, Gs, resp_lens_flat, rows, flags, logp, lse, workspace)


@_placed
def _adjusted_fwd(raw, logits, labels, tokens, rules, prompt_lens, Gs, resp_lens_flat, mask, flags, logp, lse, workspace):
    T, V = logits.shape
    if logp is None or lse is None:
        if logp is None and lse is None:
            flags |= SP_FLAG_ZERO_PROMPT_ROWS
            logp, lse = (torch.empty(T, dtype=torch.float32, device=logits.device) for _ in range(2))
        else:
            zeros = torch.zeros(T, dtype=torch.float32, device=logits.device)
            logp, lse = zeros if logp is None else logp, zeros if lse is None else lse
    workspace = _adjusted_workspace(logits, prompt_lens, resp_lens_flat, workspace)
    _check(load_library().sp_attn_adjusted_logprob_fwd(logits.data_ptr(), labels.data_ptr(), tokens.data_ptr(), logp.data_ptr(), lse.data_ptr(), V,
                                                       rules._ref, *mask, len(prompt_lens), _i32(prompt_lens), _i32(Gs), _i32(resp_lens_flat),
                                                       _dtype_code(logits), flags, workspace.data_ptr(), workspace.nbytes, raw))
    return logp, lse


def sp_attn_adjusted_logprob_bwd(logits, labels, tokens, lse, g, rules: LogitRules, prompt_lens: Sequence[int], Gs: Sequence[int],
                                 resp_lens_flat: Sequence[int], mask=None, flags: int = 0, dlogits=None, workspace=None, stream=None):
    """Gradient with respect to the raw logits of sum_t g[t] logp[t], logp of sp_attn_adjusted_logprob_fwd.  Prompt rows of dlogits are zero
    when it is allocated here, otherwise they keep what they held (SP_FLAG_ZERO_PROMPT_ROWS: zero).  ``dlogits`` may be logits itself."""
    index, rows = _adjusted_args(logits, labels, tokens, rules, prompt_lens, Gs, resp_lens_flat, mask, workspace)
    T, V = logits.shape
    _need("lse", lse, torch.float32, (T,), index)
    _need("g", g, torch.float32, (T,), index)
    if dlogits is None:
        flags |= SP_FLAG_ZERO_PROMPT_ROWS
    else:
        _need("dlogits", dlogits, logits.dtype, (T, V), index)
    return _adjusted_bwd(index, stream, logits, labels, tokens, lse, g, rules, prompt_lens, Gs, resp_lens_flat, rows, flags, dlogits, workspace)


@_placed
def _adjusted_bwd(raw, logits, labels, tokens, lse, g, rules, prompt_lens, Gs, resp_lens_flat, mask, flags, dlogits, workspace):
    if dlogits is None:
        dlogits = torch.empty_like(logits)
    workspace = _adjusted_workspace(logits, prompt_lens, resp_lens_flat, workspace)
    _check(load_library().sp_attn_adjusted_logprob_bwd(logits.data_ptr(), labels.data_ptr(), tokens.data_ptr(), lse.data_ptr(), g.data_ptr(),
                                                       dlogits.data_ptr(), logits.shape[1], rules._ref, *mask, len(prompt_lens), _i32(prompt_lens),
                                                       _i32(Gs), _i32(resp_lens_flat), _dtype_code(logits), flags, workspace.data_ptr(),
                                                       workspace.nbytes, raw))
    return dlogits
