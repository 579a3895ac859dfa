"""Thin Python binding of libdepsync.so (argument marshalling only).

Every step of a chain runs in the library's HIP kernels; this module only turns torch
tensors into device pointers and streams into hipStream_t handles, and mirrors the names of
include/depsync.h.  There is no fallback: if the shared library is missing or a call fails,
an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdepsync.so")

# enums of include/depsync.h
ROWSYNC, TILESYNC, STRIDEDSYNC, AUTOSYNC = 0, 1, 2, 3
MODE_FINE, MODE_STREAMSYNC, MODE_PLAIN, MODE_FUSED = 0, 1, 2, 3
MID_NONE, MID_GELU, MID_RELU, MID_SWIGLU, MID_CAUSAL_ATTN = 0, 1, 2, 3, 4
BF16, FP16 = 0, 1
(TILE_AUTO, TILE_256x256, TILE_256x128, TILE_128x256, TILE_128x128, TILE_64x128, TILE_64x64,
 TILE_256x192, TILE_128x192, TILE_256x64, TILE_64x64_DEEP, TILE_64x192, TILE_128x192_DEEP, TILE_128x128_DEEP) = range(14)
TILE_192x192 = 15
W_ROWS, W_KBLOCKED = 0, 1
FLAG_NO_REORDER, FLAG_COUNT, FLAG_REVERSE_ORDER, FLAG_HW_ORDER, FLAG_TRACE, FLAG_QUEUE_ORDER = 1, 2, 4, 8, 16, 32
OK, EINVAL, ENOMEM, EHIP, ETIMEOUT, ENOTIMPL, ELIMIT = 0, -1, -2, -3, -4, -5, -6

EXPORTS = [
    "sync_policy_create", "sync_policy_destroy", "dep_chain_reset", "depsync_last_status", "depsync_read_trace",
    "dep_gemm_chain", "dep_conv_chain", "depsync_gemm_chain_plan", "depsync_conv_chain_plan",
    "depsync_row_major", "depsync_policy_sem", "depsync_policy_value", "depsync_wave_model",
    "depsync_sync_count", "depsync_simulate_chain", "depsync_strerror", "depsync_last_hip_error",
    "depsync_tile_shape", "depsync_device_info", "depsync_gemm_chain_autotune", "depsync_conv_chain_autotune",
    "depsync_gemm_chain_tuned", "depsync_conv_chain_tuned", "depsync_gemm_chain_set_tuned", "depsync_conv_chain_set_tuned",
    "depsync_mfma_calibration", "dep_copy_chain", "depsync_copy_chain_plan",
    "dep_conv_chain_n", "depsync_conv_chain_n_plan", "depsync_conv_chain_n_autotune", "depsync_workspace_bytes",
    "depsync_gemm_chain_check_waits", "depsync_conv_chain_n_check_waits", "dep_gemm_chain_static",
    "depsync_gemm_chain_autotune_policy", "depsync_conv_chain_n_autotune_policy", "depsync_gemm_chain_policy",
    "depsync_conv_chain_n_policy", "depsync_gemm_chain_launch_form", "depsync_conv_chain_n_launch_form",
    "dep_tree_attn", "depsync_tree_attn_workspace", "dep_cache_append", "dep_cache_weights", "dep_cache_evict",
    "depsync_cache_evict_workspace",
    "dep_qk_norm_rope", "dep_tree_attn8", "depsync_tree_attn8_workspace", "dep_cache_append8", "dep_verify_drafts", "depsync_verify_drafts_workspace",
]


class DepsyncError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = _lib().depsync_strerror(status).decode()
        if status == EHIP:
            msg += f" [hip error {_lib().depsync_last_hip_error()}]"
        super().__init__(f"{what}: {msg} ({status})")


class PolicyParams(ctypes.Structure):
    _fields_ = [("stride", ctypes.c_uint32), ("count", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("spin_limit", ctypes.c_uint32), ("delay_tile", ctypes.c_uint32),
                ("delay_iters", ctypes.c_uint32), ("ksplit", ctypes.c_uint32)]


class Status(ctypes.Structure):
    _fields_ = [("timed_out", ctypes.c_int32), ("first_timeout", ctypes.c_int32),
                ("posts", ctypes.c_uint32), ("waits", ctypes.c_uint32),
                ("polling_waits", ctypes.c_uint32), ("launches", ctypes.c_uint32)]


class TraceRec(ctypes.Structure):
    _fields_ = [("rel", ctypes.c_uint32), ("where", ctypes.c_uint32), ("tx", ctypes.c_uint32), ("ty", ctypes.c_uint32),
                ("t_enter", ctypes.c_uint64), ("t_start", ctypes.c_uint64), ("t_ready", ctypes.c_uint64), ("t_end", ctypes.c_uint64)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("tile_prod", ctypes.c_int32), ("tile_mid", ctypes.c_int32), ("tile_cons", ctypes.c_int32),
                ("prod_grid_x", ctypes.c_int32), ("prod_grid_y", ctypes.c_int32),
                ("mid_grid_x", ctypes.c_int32), ("mid_grid_y", ctypes.c_int32),
                ("cons_grid_x", ctypes.c_int32), ("cons_grid_y", ctypes.c_int32),
                ("n_prod", ctypes.c_int32), ("n_mid", ctypes.c_int32), ("n_cons", ctypes.c_int32),
                ("n_sems", ctypes.c_int32), ("slots", ctypes.c_int32),
                ("waves_streamsync", ctypes.c_int32), ("waves_fine", ctypes.c_int32),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class GemmChainDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("K1", ctypes.c_int32), ("N1", ctypes.c_int32), ("N2", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("mid", ctypes.c_int32),
                ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W1t", ctypes.c_void_p), ("ldw1", ctypes.c_int64),
                ("H", ctypes.c_void_p), ("ldh", ctypes.c_int64),
                ("W2t", ctypes.c_void_p), ("ldw2", ctypes.c_int64),
                ("Y", ctypes.c_void_p), ("ldy", ctypes.c_int64),
                ("T", ctypes.c_void_p), ("ldt", ctypes.c_int64),
                ("batch", ctypes.c_int32), ("seq", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("tile_prod", ctypes.c_int32), ("tile_cons", ctypes.c_int32), ("w_layout", ctypes.c_int32),
                ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("ld_cache", ctypes.c_int64),
                ("cached", ctypes.c_int32)]


class ConvChainDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("C", ctypes.c_int32),
                ("K1", ctypes.c_int32), ("K2", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("inp", ctypes.c_void_p), ("w1", ctypes.c_void_p), ("mid", ctypes.c_void_p),
                ("w2", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("tile_prod", ctypes.c_int32), ("tile_cons", ctypes.c_int32)]


class ConvChainNDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("C", ctypes.c_int32),
                ("n", ctypes.c_int32), ("K", ctypes.c_int32 * 4), ("dtype", ctypes.c_int32),
                ("inp", ctypes.c_void_p), ("w", ctypes.c_void_p * 4), ("out", ctypes.c_void_p * 4),
                ("tile_prod", ctypes.c_int32), ("tile_cons", ctypes.c_int32)]


class CopyChainDesc(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("mid", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("bytes", ctypes.c_uint64), ("tile_bytes", ctypes.c_uint32)]


def _fields(**groups):
    """ctypes fields in the header's order: name -> "i" (int32), "l" (int64), "p" (pointer), "f" (float)."""
    kinds = {"i": ctypes.c_int32, "l": ctypes.c_int64, "p": ctypes.c_void_p, "f": ctypes.c_float}
    return [(n, kinds[k]) for n, k in groups.items()]


class TreeAttnDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", heads="i", kv_heads="i", head_dim="i", dtype="i", capacity="i", max_cached="i",
                       q="p", q_batch="l", q_token="l", q_head="l",
                       k_new="p", v_new="p", new_batch="l", new_token="l", new_head="l",
                       k_cache="p", v_cache="p", cache_batch="l", cache_token="l", cache_head="l",
                       cached="p", drafted="p", tree="p", tree_batch="l", scale="f",
                       out="p", out_batch="l", out_token="l", out_head="l", lse="p")


class CacheAppendDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", kv_heads="i", head_dim="i", dtype="i", capacity="i", n_max="i",
                       k_new="p", v_new="p", new_batch="l", new_token="l", new_head="l",
                       k_cache="p", v_cache="p", cache_batch="l", cache_token="l", cache_head="l",
                       cached="p", cached_out="p", accepted="p", n_accepted="p", weights="p", pos="p", start="p", n_out="p")


class CacheWeightsDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", heads="i", kv_heads="i", head_dim="i", dtype="i", capacity="i", max_cached="i", n_max="i",
                       q="p", q_batch="l", q_token="l", q_head="l", lse="p",
                       k_cache="p", cache_batch="l", cache_token="l", cache_head="l",
                       cached="p", accepted="p", n_accepted="p", scale="f", weights="p")


class CacheEvictDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", kv_heads="i", head_dim="i", dtype="i", capacity="i", max_cached="i", budget="i", recent="i",
                       k_cache="p", v_cache="p", cache_batch="l", cache_token="l", cache_head="l",
                       weights="p", pos="p", cached="p", cached_out="p", capacity_out="i",
                       k_out="p", v_out="p", out_batch="l", out_token="l", out_head="l", weights_out="p", pos_out="p")


class TreeAttn8Desc(ctypes.Structure):
    _fields_ = [("attn", TreeAttnDesc)] + _fields(block="i", k_scale="p", v_scale="p", k_tail="p", v_tail="p", tail_batch="l", tail_token="l", tail_head="l")


class CacheAppend8Desc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", kv_heads="i", head_dim="i", dtype="i", capacity="i", block="i", n_max="i",
                       k_new="p", v_new="p", new_batch="l", new_token="l", new_head="l",
                       k_cache="p", v_cache="p", cache_batch="l", cache_token="l", cache_head="l", k_scale="p", v_scale="p",
                       k_tail="p", v_tail="p", tail_batch="l", tail_token="l", tail_head="l",
                       cached="p", cached_out="p", accepted="p", n_accepted="p", n_out="p")


class QkNormRopeDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", heads="i", kv_heads="i", head_dim="i", dtype="i", rotary_dim="i", interleaved="i", norm="i", eps="f",
                       q="p", q_batch="l", q_token="l", q_head="l", k="p", k_batch="l", k_token="l", k_head="l",
                       q_out="p", q_out_batch="l", q_out_token="l", q_out_head="l", k_out="p", k_out_batch="l", k_out_token="l", k_out_head="l",
                       q_gain="p", k_gain="p", freq="p", start="p", depth="p", depth_batch="l", drafted="p")


class VerifyDraftsDesc(ctypes.Structure):
    _fields_ = _fields(batch="i", tokens="i", vocab="i", p="p", p_batch="l", p_token="l", q="p", q_batch="l", q_token="l",
                       ids="p", parents="p", parents_batch="l", drafted="p", u="p", accepted="p", n_accepted="p", next="p")


_LIB = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it first (python -m paper_2305_13450_amd.build or "
                "__graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int
        L.sync_policy_create.argtypes = [i32, ctypes.POINTER(PolicyParams), ctypes.POINTER(vp)]
        L.sync_policy_destroy.argtypes = [vp]
        L.dep_chain_reset.argtypes = [vp, vp]
        L.depsync_last_status.argtypes = [vp, ctypes.POINTER(Status)]
        L.depsync_read_trace.argtypes = [vp, ctypes.POINTER(TraceRec), i32]
        L.dep_gemm_chain.argtypes = [ctypes.POINTER(GemmChainDesc), vp, i32, vp, vp]
        L.dep_conv_chain.argtypes = [ctypes.POINTER(ConvChainDesc), vp, i32, vp, vp]
        L.depsync_gemm_chain_plan.argtypes = [ctypes.POINTER(GemmChainDesc), vp, i32, ctypes.POINTER(PlanInfo)]
        L.depsync_conv_chain_plan.argtypes = [ctypes.POINTER(ConvChainDesc), vp, i32, ctypes.POINTER(PlanInfo)]
        L.depsync_gemm_chain_autotune.argtypes = [ctypes.POINTER(GemmChainDesc), vp, vp, i32, ctypes.POINTER(i32)]
        L.depsync_conv_chain_autotune.argtypes = [ctypes.POINTER(ConvChainDesc), vp, vp, i32, ctypes.POINTER(i32)]
        L.dep_conv_chain_n.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, i32, vp, vp]
        L.depsync_conv_chain_n_plan.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, i32, ctypes.POINTER(PlanInfo)]
        L.depsync_conv_chain_n_autotune.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, vp, i32, ctypes.POINTER(i32)]
        L.dep_copy_chain.argtypes = [ctypes.POINTER(CopyChainDesc), vp, i32, vp, vp]
        L.depsync_copy_chain_plan.argtypes = [ctypes.POINTER(CopyChainDesc), vp, i32, ctypes.POINTER(PlanInfo)]
        L.depsync_mfma_calibration.argtypes = [i32, i32, ctypes.POINTER(ctypes.c_double)]
        L.depsync_gemm_chain_tuned.argtypes = [ctypes.POINTER(GemmChainDesc), vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.depsync_conv_chain_tuned.argtypes = [ctypes.POINTER(ConvChainDesc), vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.depsync_gemm_chain_set_tuned.argtypes = [ctypes.POINTER(GemmChainDesc), vp, i32, i32]
        L.depsync_conv_chain_set_tuned.argtypes = [ctypes.POINTER(ConvChainDesc), vp, i32, i32]
        i32p = ctypes.POINTER(i32)
        L.depsync_gemm_chain_launch_form.argtypes = [ctypes.POINTER(GemmChainDesc), vp, i32, i32, i32p, i32p]
        L.depsync_conv_chain_n_launch_form.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, i32, i32, i32p, i32p]
        i64p = ctypes.POINTER(ctypes.c_int64)
        L.depsync_gemm_chain_check_waits.argtypes = [ctypes.POINTER(GemmChainDesc), i32, ctypes.POINTER(PolicyParams), i32, i64p]
        L.depsync_conv_chain_n_check_waits.argtypes = [ctypes.POINTER(ConvChainNDesc), i32, ctypes.POINTER(PolicyParams), i32, i64p]
        f3 = ctypes.POINTER(ctypes.c_float)
        L.depsync_gemm_chain_autotune_policy.argtypes = [ctypes.POINTER(GemmChainDesc), vp, vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), f3]
        L.depsync_conv_chain_n_autotune_policy.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), f3]
        L.depsync_gemm_chain_policy.argtypes = [ctypes.POINTER(GemmChainDesc), vp, ctypes.POINTER(i32)]
        L.depsync_conv_chain_n_policy.argtypes = [ctypes.POINTER(ConvChainNDesc), vp, ctypes.POINTER(i32)]
        L.dep_gemm_chain_static.argtypes = [ctypes.POINTER(GemmChainDesc), i32, ctypes.POINTER(PolicyParams), vp]
        szp = ctypes.POINTER(ctypes.c_size_t)
        # (descriptors come by reference or packed into bytes)
        L.dep_tree_attn.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.depsync_tree_attn_workspace.argtypes = [vp, i32, szp]
        L.dep_cache_append.argtypes = [vp, vp]
        L.dep_cache_weights.argtypes = [vp, vp]
        L.dep_cache_evict.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.depsync_cache_evict_workspace.argtypes = [vp, szp]
        L.dep_qk_norm_rope.argtypes = [vp, vp]
        L.dep_tree_attn8.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.depsync_tree_attn8_workspace.argtypes = [vp, i32, szp]
        L.dep_cache_append8.argtypes = [vp, vp]
        L.dep_verify_drafts.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.depsync_verify_drafts_workspace.argtypes = [vp, szp]
        L.depsync_row_major.argtypes = [i32] * 4
        L.depsync_policy_sem.argtypes = [i32] * 6
        L.depsync_policy_value.argtypes = [i32] * 4
        L.depsync_wave_model.argtypes = [i32, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double)]
        L.depsync_sync_count.argtypes = [i32] * 6
        L.depsync_simulate_chain.argtypes = [i32, i32, i32, ctypes.c_double, i32, i32, ctypes.c_double, i32, i32]
        L.depsync_simulate_chain.restype = ctypes.c_double
        L.depsync_strerror.argtypes = [i32]
        L.depsync_strerror.restype = ctypes.c_char_p
        L.depsync_last_hip_error.argtypes = []
        L.depsync_tile_shape.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.depsync_device_info.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(i32)]
        _LIB = L
    return _LIB


def _check(status: int, what: str) -> None:
    if status != OK:
        raise DepsyncError(status, what)


def _stream_handle(stream) -> Optional[int]:
    """torch.cuda.Stream | raw handle | None -> hipStream_t as an integer (None = NULL)."""
    if stream is None:
        return None
    if hasattr(stream, "cuda_stream"):
        return int(stream.cuda_stream) or None
    return int(stream) or None


def _tile_pair(tile):
    """A macro-tile id for every stage, or a (producer, consumer) pair of ids."""
    if isinstance(tile, (tuple, list)):
        prod, cons = tile
        return int(prod), int(cons)
    return int(tile), int(tile)


_CODES = {}


def _dtype_code(t) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        import torch
        _CODES.update({torch.bfloat16: BF16, torch.float16: FP16})
        code = _CODES.get(t.dtype)
        if code is None:
            raise TypeError(f"unsupported element type {t.dtype}")
    return code


def _dev2d(t, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with contiguous rows")
    return t.data_ptr(), t.stride(0)


class SyncPolicy:
    """Owner of a sync_policy_t (policy kind + semaphore workspace)."""

    def __init__(self, kind: int, stride: int = 0, count: int = 0, flags: int = 0, spin_limit: int = 0,
                 delay_tile: int = 0, delay_iters: int = 0, ksplit: int = 0):
        self.kind = kind
        params = PolicyParams(stride, count, flags, spin_limit, delay_tile, delay_iters, ksplit)
        h = ctypes.c_void_p()
        _check(_lib().sync_policy_create(kind, ctypes.byref(params), ctypes.byref(h)), "sync_policy_create")
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("policy already destroyed")
        return self._h

    def destroy(self):
        if self._h is not None:
            _check(_lib().sync_policy_destroy(self._h), "sync_policy_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def reset(self, stream=None):
        _check(_lib().dep_chain_reset(self.handle, _stream_handle(stream)), "dep_chain_reset")

    def read_trace(self, n_tiles: int):
        """Per-tile timing records of the last chain run with FLAG_TRACE (list of TraceRec)."""
        buf = (TraceRec * n_tiles)()
        n = _lib().depsync_read_trace(self.handle, buf, n_tiles)
        if n < 0:
            raise DepsyncError(n, "depsync_read_trace")
        return list(buf[:n])

    def status(self, raise_on_timeout: bool = True) -> Status:
        st = Status()
        rc = _lib().depsync_last_status(self.handle, ctypes.byref(st))
        if rc == ETIMEOUT and not raise_on_timeout:
            return st
        _check(rc, "depsync_last_status")
        return st


def sync_policy_create(kind: int, **params) -> SyncPolicy:
    return SyncPolicy(kind, **params)


def pack_weights_kblocked(Wt):
    """[N x K] (K contiguous) -> the K-blocked layout [K/64][N][64]: a pure re-arrangement."""
    n, k = Wt.shape
    if k % 64:
        raise ValueError("K must be a multiple of 64")
    return Wt.reshape(n, k // 64, 64).permute(1, 0, 2).contiguous()


def _dev_w(t, name: str):
    """A weight operand: 2-D [N x K] row-major, or 3-D [K/64][N][64] (K-blocked).  -> (ptr, ld, N, K, blocked)"""
    if t.dim() == 3:
        if not t.is_cuda or not t.is_contiguous() or t.shape[2] != 64:
            raise ValueError(f"{name}: K-blocked weights must be a contiguous [K/64, N, 64] device tensor")
        return t.data_ptr(), 0, t.shape[1], t.shape[0] * 64, True
    ptr, ld = _dev2d(t, name)
    return ptr, ld, t.shape[0], t.shape[1], False


def _gemm_desc(X, W1t, H, W2t, Y, mid, tile, T=None, batch=0, seq=0, heads=0, head_dim=0,
               k_cache=None, v_cache=None) -> GemmChainDesc:
    d = GemmChainDesc()
    d.X, d.ldx = _dev2d(X, "X")
    d.W1t, d.ldw1, w1n, w1k, b1 = _dev_w(W1t, "W1t")
    d.H, d.ldh = _dev2d(H, "H")
    d.W2t, d.ldw2, w2n, w2k, b2 = _dev_w(W2t, "W2t")
    if b1 != b2:
        raise ValueError("both weight operands must use the same layout")
    d.w_layout = W_KBLOCKED if b1 else W_ROWS
    d.Y, d.ldy = _dev2d(Y, "Y")
    d.M, d.K1 = X.shape
    d.N1 = H.shape[1]
    d.N2 = Y.shape[1]
    d.dtype = _dtype_code(X)
    for t in (W1t, H, W2t, Y):
        if t.dtype != X.dtype:
            raise TypeError("all tensors of a chain must share one element type")
    d.mid = mid
    if T is not None:
        d.T, d.ldt = _dev2d(T, "T")
    d.batch, d.seq, d.heads, d.head_dim = batch, seq, heads, head_dim
    if k_cache is not None or v_cache is not None:
        # [batch, cached, heads*head_dim] device tensors of earlier tokens' keys and values
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            if t is None or not t.is_cuda or t.dim() != 3 or t.stride(2) != 1 or t.dtype != X.dtype:
                raise ValueError(f"{name} must be a 3-D device tensor of the chain's element type")
            if t.shape[0] != batch or t.stride(0) != t.shape[1] * t.stride(1):
                raise ValueError(f"{name}: one block of rows per sequence, equally spaced")
        if k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
            raise ValueError("k_cache and v_cache must have the same shape and strides")
        d.k_cache, d.v_cache = k_cache.data_ptr(), v_cache.data_ptr()
        d.ld_cache, d.cached = k_cache.stride(1), k_cache.shape[1]
    d.tile_prod, d.tile_cons = _tile_pair(tile)
    rows1 = 2 * d.N1 if mid == MID_SWIGLU else d.N1
    k2 = heads * head_dim if mid == MID_CAUSAL_ATTN else d.N1
    if (w1n, w1k) != (rows1, d.K1) or (w2n, w2k) != (d.N2, k2) or H.shape[0] != d.M or Y.shape[0] != d.M:
        raise ValueError("operand shapes do not form a chain")
    return d


def dep_gemm_chain(X, W1t, H, W2t, Y, policy: SyncPolicy, mode: int = MODE_FINE, mid: int = MID_GELU,
                   tile: int = TILE_AUTO, stream_producer=None, stream_consumer=None, T=None,
                   batch: int = 0, seq: int = 0, heads: int = 0, head_dim: int = 0,
                   k_cache=None, v_cache=None) -> None:
    """Enqueue Y = mid(X W1) W2 with W1t = W1^T [N1 x K1] and W2t = W2^T [N2 x K2] (row-major)."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, tile, T, batch, seq, heads, head_dim, k_cache, v_cache)
    _check(_lib().dep_gemm_chain(ctypes.byref(d), policy.handle, mode, _stream_handle(stream_producer),
                                 _stream_handle(stream_consumer)), "dep_gemm_chain")


def dep_gemm_chain_static(X, W1t, H, W2t, Y, kind: int, mid: int = MID_GELU, tile: int = TILE_AUTO, stream=None,
                          T=None, batch: int = 0, seq: int = 0, heads: int = 0, head_dim: int = 0,
                          k_cache=None, v_cache=None, **params) -> None:
    """The chain in one dispatch on `stream` with the library's fixed device workspace: no policy
    object, no allocation.  `params`: fields of PolicyParams (flags, ksplit, ...)."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, tile, T, batch, seq, heads, head_dim, k_cache, v_cache)
    pp = PolicyParams(**params)
    _check(_lib().dep_gemm_chain_static(ctypes.byref(d), kind, ctypes.byref(pp), _stream_handle(stream)),
           "dep_gemm_chain_static")


def gemm_chain_plan(X, W1t, H, W2t, Y, policy: Optional[SyncPolicy], mid: int = MID_GELU, tile: int = TILE_AUTO,
                    n_cu: int = 0, **attn) -> PlanInfo:
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, tile, **attn)
    info = PlanInfo()
    _check(_lib().depsync_gemm_chain_plan(ctypes.byref(d), policy.handle if policy else None, n_cu,
                                          ctypes.byref(info)), "depsync_gemm_chain_plan")
    return info


def gemm_chain_autotune(X, W1t, H, W2t, Y, policy: SyncPolicy, mid: int = MID_GELU, stream=None, reps: int = 3,
                        **attn) -> int:
    """Time every macro-tile shape on this chain and make the fastest the library's choice for it."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, TILE_AUTO, **attn)
    tile = ctypes.c_int(0)
    _check(_lib().depsync_gemm_chain_autotune(ctypes.byref(d), policy.handle, _stream_handle(stream), reps,
                                              ctypes.byref(tile)), "depsync_gemm_chain_autotune")
    return tile.value


def conv_chain_autotune(x, w1, mid, w2, out, policy: SyncPolicy, stream=None, reps: int = 3) -> int:
    d = _conv_desc(x, w1, mid, w2, out, TILE_AUTO)
    tile = ctypes.c_int(0)
    _check(_lib().depsync_conv_chain_autotune(ctypes.byref(d), policy.handle, _stream_handle(stream), reps,
                                              ctypes.byref(tile)), "depsync_conv_chain_autotune")
    return tile.value


def gemm_chain_autotune_policy(X, W1t, H, W2t, Y, policy: SyncPolicy, mid: int = MID_GELU, stream=None, reps: int = 3, **attn):
    """Autotune the chain under every policy kind and remember the fastest for its shape (what AUTOSYNC
    policies resolve to).  Returns (kind, tile, [us under ROWSYNC, TILESYNC, STRIDEDSYNC; -1 = cannot run])."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, TILE_AUTO, **attn)
    kind, tile, us = ctypes.c_int(-1), ctypes.c_int(0), (ctypes.c_float * 3)()
    _check(_lib().depsync_gemm_chain_autotune_policy(ctypes.byref(d), policy.handle, _stream_handle(stream), reps,
                                                     ctypes.byref(kind), ctypes.byref(tile), us), "depsync_gemm_chain_autotune_policy")
    return kind.value, tile.value, list(us)


def conv_chain_n_autotune_policy(x, ws, outs, policy: SyncPolicy, stream=None, reps: int = 3):
    d = _conv_n_desc(x, ws, outs, TILE_AUTO)
    kind, tile, us = ctypes.c_int(-1), ctypes.c_int(0), (ctypes.c_float * 3)()
    _check(_lib().depsync_conv_chain_n_autotune_policy(ctypes.byref(d), policy.handle, _stream_handle(stream), reps,
                                                       ctypes.byref(kind), ctypes.byref(tile), us), "depsync_conv_chain_n_autotune_policy")
    return kind.value, tile.value, list(us)


def gemm_chain_policy(X, W1t, H, W2t, Y, policy: SyncPolicy, mid: int = MID_GELU, **attn) -> int:
    """The policy kind a chain of this shape runs under with `policy` (what AUTOSYNC resolves to)."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, TILE_AUTO, **attn)
    kind = ctypes.c_int(-1)
    _check(_lib().depsync_gemm_chain_policy(ctypes.byref(d), policy.handle, ctypes.byref(kind)), "depsync_gemm_chain_policy")
    return kind.value


TUNED_NO_SPLIT, TUNED_HW_ORDER = 1, 2


def gemm_chain_tuned(X, W1t, H, W2t, Y, policy: SyncPolicy, mid: int = MID_GELU, **attn):
    """(tile, flags) the library remembers for this chain; tile 0 when it remembers nothing."""
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, TILE_AUTO, **attn)
    tile, flags = ctypes.c_int(0), ctypes.c_int(0)
    _check(_lib().depsync_gemm_chain_tuned(ctypes.byref(d), policy.handle, ctypes.byref(tile), ctypes.byref(flags)),
           "depsync_gemm_chain_tuned")
    return tile.value, flags.value


def gemm_chain_set_tuned(X, W1t, H, W2t, Y, policy: SyncPolicy, tile: int, flags: int = 0, mid: int = MID_GELU, **attn):
    d = _gemm_desc(X, W1t, H, W2t, Y, mid, TILE_AUTO, **attn)
    _check(_lib().depsync_gemm_chain_set_tuned(ctypes.byref(d), policy.handle, tile, flags), "depsync_gemm_chain_set_tuned")


def conv_chain_tuned(x, w1, mid, w2, out, policy: SyncPolicy):
    d = _conv_desc(x, w1, mid, w2, out, TILE_AUTO)
    tile, flags = ctypes.c_int(0), ctypes.c_int(0)
    _check(_lib().depsync_conv_chain_tuned(ctypes.byref(d), policy.handle, ctypes.byref(tile), ctypes.byref(flags)),
           "depsync_conv_chain_tuned")
    return tile.value, flags.value


def conv_chain_set_tuned(x, w1, mid, w2, out, policy: SyncPolicy, tile: int, flags: int = 0):
    d = _conv_desc(x, w1, mid, w2, out, TILE_AUTO)
    _check(_lib().depsync_conv_chain_set_tuned(ctypes.byref(d), policy.handle, tile, flags), "depsync_conv_chain_set_tuned")


def _conv_desc(x, w1, mid, w2, out, tile) -> ConvChainDesc:
    for t, name in ((x, "x"), (w1, "w1"), (mid, "mid"), (w2, "w2"), (out, "out")):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-D device tensor")
        if t.dtype != x.dtype:
            raise TypeError("all tensors of a chain must share one element type")
    d = ConvChainDesc()
    d.B, d.H, d.W, d.C = x.shape
    d.K1, d.K2 = w1.shape[0], w2.shape[0]
    if (tuple(w1.shape) != (d.K1, 3, 3, d.C) or tuple(w2.shape) != (d.K2, 3, 3, d.K1)
            or tuple(mid.shape) != (d.B, d.H, d.W, d.K1) or tuple(out.shape) != (d.B, d.H, d.W, d.K2)):
        raise ValueError("operand shapes do not form a conv chain")
    d.dtype = _dtype_code(x)
    d.inp, d.w1, d.mid, d.w2, d.out = x.data_ptr(), w1.data_ptr(), mid.data_ptr(), w2.data_ptr(), out.data_ptr()
    d.tile_prod, d.tile_cons = _tile_pair(tile)
    return d


def dep_conv_chain(x, w1, mid, w2, out, policy: SyncPolicy, mode: int = MODE_FINE, tile: int = TILE_AUTO,
                   stream_producer=None, stream_consumer=None) -> None:
    """Enqueue out = conv3x3(relu(conv3x3(x, w1)), w2); NHWC activations, [K,3,3,C] weights."""
    d = _conv_desc(x, w1, mid, w2, out, tile)
    _check(_lib().dep_conv_chain(ctypes.byref(d), policy.handle, mode, _stream_handle(stream_producer),
                                 _stream_handle(stream_consumer)), "dep_conv_chain")


def conv_chain_plan(x, w1, mid, w2, out, policy: Optional[SyncPolicy], tile: int = TILE_AUTO, n_cu: int = 0) -> PlanInfo:
    d = _conv_desc(x, w1, mid, w2, out, tile)
    info = PlanInfo()
    _check(_lib().depsync_conv_chain_plan(ctypes.byref(d), policy.handle if policy else None, n_cu,
                                          ctypes.byref(info)), "depsync_conv_chain_plan")
    return info


def _conv_n_desc(x, ws, outs, tile) -> ConvChainNDesc:
    n = len(ws)
    if n != len(outs) or not 2 <= n <= 4:
        raise ValueError("a conv chain has 2 to 4 convolutions, one output buffer each")
    for t in [x, *ws, *outs]:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
    d = ConvChainNDesc()
    d.B, d.H, d.W, d.C = x.shape
    d.n = n
    d.dtype = _dtype_code(x)
    d.inp = x.data_ptr()
    cin = d.C
    for i, (w, o) in enumerate(zip(ws, outs)):
        if tuple(w.shape[1:]) != (3, 3, cin) or tuple(o.shape) != (d.B, d.H, d.W, w.shape[0]) or w.dtype != x.dtype or o.dtype != x.dtype:
            raise ValueError(f"conv {i}: weights [K,3,3,{cin}] and output [B,H,W,K] of the input's type expected")
        d.K[i], d.w[i], d.out[i] = w.shape[0], w.data_ptr(), o.data_ptr()
        cin = w.shape[0]
    d.tile_prod, d.tile_cons = _tile_pair(tile)
    return d


def dep_conv_chain_n(x, ws, outs, policy: SyncPolicy, mode: int = MODE_FINE, tile: int = TILE_AUTO,
                     stream_producer=None, stream_consumer=None) -> None:
    """Enqueue 2..4 chained 3x3 convolutions, ReLU between them: outs[i] = conv(relu-ed outs[i-1], ws[i])."""
    d = _conv_n_desc(x, ws, outs, tile)
    _check(_lib().dep_conv_chain_n(ctypes.byref(d), policy.handle, mode, _stream_handle(stream_producer),
                                   _stream_handle(stream_consumer)), "dep_conv_chain_n")


def conv_chain_n_plan(x, ws, outs, policy: Optional[SyncPolicy], tile: int = TILE_AUTO, n_cu: int = 0) -> PlanInfo:
    d = _conv_n_desc(x, ws, outs, tile)
    info = PlanInfo()
    _check(_lib().depsync_conv_chain_n_plan(ctypes.byref(d), policy.handle if policy else None, n_cu,
                                            ctypes.byref(info)), "depsync_conv_chain_n_plan")
    return info


def conv_chain_n_autotune(x, ws, outs, policy: SyncPolicy, stream=None, reps: int = 3) -> int:
    d = _conv_n_desc(x, ws, outs, TILE_AUTO)
    tile = ctypes.c_int(0)
    _check(_lib().depsync_conv_chain_n_autotune(ctypes.byref(d), policy.handle, _stream_handle(stream), reps,
                                                ctypes.byref(tile)), "depsync_conv_chain_n_autotune")
    return tile.value


def _copy_desc(src, mid, dst, tile_bytes: int) -> CopyChainDesc:
    n = src.numel() * src.element_size()
    for t, name in ((src, "src"), (mid, "mid"), (dst, "dst")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous device tensor")
        if t.numel() * t.element_size() != n:
            raise ValueError("src, mid and dst must have the same size in bytes")
    d = CopyChainDesc()
    d.src, d.mid, d.dst = src.data_ptr(), mid.data_ptr(), dst.data_ptr()
    d.bytes, d.tile_bytes = n, tile_bytes
    return d


def dep_copy_chain(src, mid, dst, policy: SyncPolicy, mode: int = MODE_FINE, tile_bytes: int = 0,
                   stream_producer=None, stream_consumer=None) -> None:
    """Enqueue mid = src then dst = mid as two dependent tiled stages (the synchronisation-overhead chain)."""
    d = _copy_desc(src, mid, dst, tile_bytes)
    _check(_lib().dep_copy_chain(ctypes.byref(d), policy.handle, mode, _stream_handle(stream_producer),
                                 _stream_handle(stream_consumer)), "dep_copy_chain")


def copy_chain_plan(src, mid, dst, policy: SyncPolicy, tile_bytes: int = 0, n_cu: int = 0) -> PlanInfo:
    d = _copy_desc(src, mid, dst, tile_bytes)
    info = PlanInfo()
    _check(_lib().depsync_copy_chain_plan(ctypes.byref(d), policy.handle, n_cu, ctypes.byref(info)),
           "depsync_copy_chain_plan")
    return info


def launch_form(desc, policy: Optional[SyncPolicy], mode: int, n_cu: int = 0) -> tuple:
    """(kernel launches, tiles named by the block index) of a GeMM or N-convolution chain in this mode."""
    f = _lib().depsync_gemm_chain_launch_form if isinstance(desc, GemmChainDesc) else _lib().depsync_conv_chain_n_launch_form
    n, hw = ctypes.c_int(0), ctypes.c_int(0)
    _check(f(ctypes.byref(desc), policy.handle if policy else None, mode, n_cu, ctypes.byref(n), ctypes.byref(hw)), "launch_form")
    return n.value, bool(hw.value)


def gemm_chain_check_waits(desc: GemmChainDesc, kind: int, n_cu: int = 0, **params) -> int:
    """(row tile, K part) pairs of the planned chain with an operand slice no wait covers (0 = sound)."""
    pp = PolicyParams(**params)
    n = ctypes.c_int64(-1)
    _check(_lib().depsync_gemm_chain_check_waits(ctypes.byref(desc), kind, ctypes.byref(pp), n_cu, ctypes.byref(n)),
           "depsync_gemm_chain_check_waits")
    return n.value


def conv_chain_n_check_waits(desc: ConvChainNDesc, kind: int, n_cu: int = 0, **params) -> int:
    pp = PolicyParams(**params)
    n = ctypes.c_int64(-1)
    _check(_lib().depsync_conv_chain_n_check_waits(ctypes.byref(desc), kind, ctypes.byref(pp), n_cu, ctypes.byref(n)),
           "depsync_conv_chain_n_check_waits")
    return n.value


# ---- the cache of token generation ----------------------------------------------------------

# These calls are short, so their descriptors are packed in one go (in the header's order, as the classes above have it) and each tensor is
# asked once for what is needed: 35 fields set one by one and the former checks took 23 us a call, three times the two launches.
# They take part in a torch program's order: without a stream they run on torch's current one on the tensors' device (the chains above: on the default stream).

_TORCH = None


def _torch():
    """torch, imported at the first call (nothing else of this module needs it)."""
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


_P_TREE = struct.Struct("8i P3q 2P3q 2P3q 3Pq f4x P3q P")
_P_APPEND = struct.Struct("7i4x 2P3q 2P3q 8P")
_P_WEIGHTS = struct.Struct("9i4x P3q P P3q 3P f4x P")
_P_EVICT = struct.Struct("8i 2P3q 4P i4x 2P3q 2P")


def _t4(t, name: str, dtype, device: int, shape=None):
    """Pointer and the first three strides of a [batch, token, head, head_dim] tensor on this device with contiguous rows."""
    s = t.stride()
    if t.get_device() != device or device < 0 or len(s) != 4 or s[3] != 1:
        raise ValueError(f"{name} must be a 4-D tensor with contiguous rows on the device of the others")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype} where {dtype} is needed (all 16-bit tensors of a call share one element type)")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)} where {tuple(shape)} is needed")
    return t.data_ptr(), s[0], s[1], s[2]


def _pair(a, b, name: str, dtype, device: int, shape):
    """The pointers of two tensors alike (keys and values), and their strides."""
    s = a.stride()
    if s == b.stride() and a.shape == shape == b.shape and a.dtype is dtype is b.dtype and a.get_device() == device == b.get_device() and s[3] == 1 and device >= 0:
        return a.data_ptr(), b.data_ptr(), s[0], s[1], s[2]
    pa, s0, s1, s2 = _t4(a, "k_" + name, dtype, device, shape)
    pb, *sb = _t4(b, "v_" + name, dtype, device, shape)
    if sb != [s0, s1, s2] and any(x != y and n > 1 for x, y, n in zip(sb, (s0, s1, s2), shape)):   # (those of dimensions of size 1 are not read)
        raise ValueError(f"k_{name} and v_{name} must have the same strides")
    return pa, pb, s0, s1, s2


def _arr(t, name: str, dtype, device: int, shape) -> int:
    """Pointer of a contiguous tensor of this shape and type on this device; None -> 0."""
    if t is None:
        return 0
    if t.get_device() != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of {dtype} and shape {tuple(shape)} on the device of the others")
    return t.data_ptr()


def _current_or(stream, device: int):
    """The handle of `stream`, or of torch's current stream on this device where it is None: what made the tensors was enqueued there."""
    return _torch()._C._cuda_getCurrentRawStream(device) or None if stream is None else _stream_handle(stream)


def _call(device: int, what: str, f, *args) -> None:
    """f(*args) with this device current, and its status checked."""
    torch = _TORCH or _torch()
    if device == torch._C._cuda_getDevice():
        rc = f(*args)
    else:
        with torch.cuda.device(device):
            rc = f(*args)
    if rc != OK:
        raise DepsyncError(rc, what)


def _workspace(nbytes: int, given, device: int, stream):
    """`given`, or memory that torch's allocator ties to `stream` (a hipStream_t): (tensor to keep, pointer, bytes)."""
    torch = _torch()
    if given is not None:
        if given.get_device() != device or not given.is_contiguous():
            raise ValueError("the workspace must be a contiguous tensor on the device of the others")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if nbytes == 0:
        return None, None, 0
    if (stream or 0) == torch._C._cuda_getCurrentRawStream(device):
        t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    else:
        own = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
        with torch.cuda.stream(own):
            t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), nbytes


def tree_mask(parents):
    """The `tree` words of dep_tree_attn for drafted tokens with these parents: an integer tensor [T] or [B, T] in host memory, -1 (or any
    negative value) for a root, every parent before its children.  Each token sees itself and its ancestors.  -> int64 [.., T, ceil(T / 64)]"""
    torch = _torch()
    p = torch.as_tensor(parents)
    if p.is_cuda or p.dim() not in (1, 2) or p.shape[-1] < 1:
        raise ValueError("parents must be a host tensor [tokens] or [batch, tokens]")
    flat = p.reshape(-1, p.shape[-1]).tolist()
    n = p.shape[-1]
    rows = []
    for seq in flat:
        seen = []
        for t, parent in enumerate(seq):
            if parent >= t:
                raise ValueError(f"token {t}: its parent {parent} must come before it")
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << t)
        for bits in seen:
            words = [bits >> 64 * w & (1 << 64) - 1 for w in range((n + 63) // 64)]
            rows.append([w - (1 << 64) if w >> 63 else w for w in words])
    return torch.tensor(rows, dtype=torch.int64).reshape(*p.shape, -1)


def _tree_attn_desc(q, k_new, v_new, k_cache, v_cache, cached, out, lse, tree, drafted, scale, max_cached, held=None):
    """(descriptor, device) of a call.  held: the type of the cache's numbers where it is not the others'."""
    torch = _torch()
    device, dtype = q.get_device(), q.dtype
    code = _dtype_code(q)
    if q.dim() != 4 or k_new.dim() != 4:
        raise ValueError("q and k_new must be [batch, tokens, heads, head_dim]")
    B, T, Hq, D = q.shape
    Hk = k_new.shape[2]
    new = _pair(k_new, v_new, "new", dtype, device, (B, T, Hk, D))
    cap, cache, lengths = 0, (0, 0, 0, 0, 0), 0
    if k_cache is not None:
        if v_cache is None or cached is None or k_cache.dim() != 4:
            raise ValueError("a cache is k_cache and v_cache [batch, capacity, kv_heads, head_dim], and cached")
        cap = k_cache.shape[1]
        cache = _pair(k_cache, v_cache, "cache", held or dtype, device, (B, cap, Hk, D))
        lengths = _arr(cached, "cached", torch.int32, device, (B,))
    tree_ptr, tree_batch = 0, 0
    if tree is not None:
        words = (T, (T + 63) // 64)
        if tree.dim() == 2:
            tree_ptr = _arr(tree, "tree", torch.int64, device, words)
        else:
            tree_ptr, tree_batch = _arr(tree, "tree", torch.int64, device, (B, *words)), words[0] * words[1]
    return _P_TREE.pack(B, T, Hq, Hk, D, code, cap, max_cached or 0, *_t4(q, "q", dtype, device), *new, *cache, lengths,
                        _arr(drafted, "drafted", torch.int32, device, (B,)), tree_ptr, tree_batch, scale or 0.0,
                        *_t4(out, "out", dtype, device, (B, T, Hq, D)), _arr(lse, "lse", torch.float32, device, (B, T, Hq))), device


def _bytes(what: str, device: int, f, *args) -> int:
    """What a workspace query says."""
    need = ctypes.c_size_t(0)
    _call(device, what, f, *args, ctypes.byref(need))
    return need.value


@functools.lru_cache(maxsize=4096)
def _tree_attn_bytes(device: int, sizes: bytes) -> int:
    """The workspace of dep_tree_attn, by the descriptor's eight sizes: all that it depends on beside the device."""
    return _bytes("dep_tree_attn", device, _lib().depsync_tree_attn_workspace, sizes + bytes(_P_TREE.size - len(sizes)), 0)


def dep_tree_attn(q, k_new, v_new, k_cache, v_cache, cached, out, lse=None, tree=None, drafted=None, scale: Optional[float] = None,
                  max_cached: Optional[int] = None, workspace=None, stream=None) -> None:
    """Enqueue out = softmax(scale q k^T) v of drafted tokens over a cache and, as `tree` (see tree_mask) says, one another.

    q, out [B, T, Hq, D]; k_new, v_new [B, T, Hk, D]; k_cache, v_cache [B, capacity, Hk, D] (None: no cache) of which sequence b has
    cached[b] rows (int32).  drafted[b] (int32): the tokens that sequence b has; the others' rows of out and lse are left alone.
    lse [B, T, Hq] (float32) receives the logarithm of each row's sum.  scale: None or 0 is 1 / sqrt(D).  max_cached: the most rows that a sequence has, where the host knows.
    stream: a torch stream or handle (0: the default stream); None: torch's current stream on the tensors' device."""
    d, device = _tree_attn_desc(q, k_new, v_new, k_cache, v_cache, cached, out, lse, tree, drafted, scale, max_cached)
    stream = _current_or(stream, device)
    need = 0 if workspace is not None else _tree_attn_bytes(device, d[:32])
    keep, ptr, size = _workspace(need, workspace, device, stream)
    _call(device, "dep_tree_attn", _lib().dep_tree_attn, d, ptr, size, stream)


def tree_attn_workspace(q, k_new, v_new, k_cache, v_cache, cached, out, lse=None, tree=None, drafted=None, scale: Optional[float] = None,
                        max_cached: Optional[int] = None, n_cu: int = 0) -> int:
    """Bytes of workspace that dep_tree_attn with these arguments needs."""
    d, device = _tree_attn_desc(q, k_new, v_new, k_cache, v_cache, cached, out, lse, tree, drafted, scale, max_cached)
    return _bytes("depsync_tree_attn_workspace", device, _lib().depsync_tree_attn_workspace, d, n_cu)


def _accepted(B: int, tokens: int, accepted, n_accepted, device: int):
    torch = _torch()
    if accepted is not None and accepted.dim() != 2:
        raise ValueError("accepted must be [batch, n_max]")
    n_max = tokens if accepted is None else accepted.shape[1]
    return n_max, _arr(accepted, "accepted", torch.int32, device, (B, n_max)), _arr(n_accepted, "n_accepted", torch.int32, device, (B,))


def dep_cache_append(k_new, v_new, k_cache, v_cache, cached, cached_out, accepted=None, n_accepted=None, weights=None, pos=None, start=None,
                     stream=None, n_out=None) -> None:
    """Enqueue: the keys and values of drafted tokens accepted[b, :n_accepted[b]] (int32; None: the first ones) go to rows cached[b].. of the cache,
    their weights [B, Hk, capacity] (float32) become 0, their positions (int32, same shape) start[b].., and cached_out = cached + n.  n_out[b] (int32) receives n, which is
    less than n_accepted[b] where the capacity was reached: what dep_cache_weights then takes for n_accepted.  stream: as for dep_tree_attn."""
    torch = _torch()
    device, dtype = k_new.get_device(), k_new.dtype
    code = _dtype_code(k_new)
    if k_new.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("k_new and k_cache must be [batch, tokens or capacity, kv_heads, head_dim]")
    B, T, Hk, D = k_new.shape
    cap = k_cache.shape[1]
    i32 = torch.int32
    n_max, acc, n_acc = _accepted(B, T, accepted, n_accepted, device)
    d = _P_APPEND.pack(B, T, Hk, D, code, cap, n_max, *_pair(k_new, v_new, "new", dtype, device, (B, T, Hk, D)),
                       *_pair(k_cache, v_cache, "cache", dtype, device, (B, cap, Hk, D)), _arr(cached, "cached", i32, device, (B,)),
                       _arr(cached_out, "cached_out", i32, device, (B,)), acc, n_acc, _arr(weights, "weights", torch.float32, device, (B, Hk, cap)),
                       _arr(pos, "pos", i32, device, (B, Hk, cap)), _arr(start, "start", i32, device, (B,)), _arr(n_out, "n_out", i32, device, (B,)))
    _call(device, "dep_cache_append", _lib().dep_cache_append, d, _current_or(stream, device))


def dep_cache_weights(q, lse, k_cache, cached, weights, accepted=None, n_accepted=None, scale: Optional[float] = None,
                      max_cached: Optional[int] = None, stream=None) -> None:
    """Enqueue weights[b, h, k] += the attention weight that cached row k received from the accepted tokens, whose own rows are the last
    of cached[b] (n_accepted: the append's n_out, where that may have dropped tokens at the capacity).  q [B, T, Hq, D] and lse [B, T, Hq] are
    dep_tree_attn's; weights is [B, Hk, capacity] (float32).  stream: as there."""
    torch = _torch()
    device, dtype = q.get_device(), q.dtype
    code = _dtype_code(q)
    if q.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q and k_cache must be [batch, tokens or capacity, heads, head_dim]")
    B, T, Hq, D = q.shape
    cap, Hk = k_cache.shape[1:3]
    n_max, acc, n_acc = _accepted(B, T, accepted, n_accepted, device)
    d = _P_WEIGHTS.pack(B, T, Hq, Hk, D, code, cap, max_cached or 0, n_max, *_t4(q, "q", dtype, device), _arr(lse, "lse", torch.float32, device, (B, T, Hq)),
                        *_t4(k_cache, "k_cache", dtype, device, (B, cap, Hk, D)), _arr(cached, "cached", torch.int32, device, (B,)), acc, n_acc,
                        scale or 0.0, _arr(weights, "weights", torch.float32, device, (B, Hk, cap)))
    _call(device, "dep_cache_weights", _lib().dep_cache_weights, d, _current_or(stream, device))


def _cache_evict_desc(k_cache, v_cache, weights, pos, cached, cached_out, budget, recent, max_cached, k_out, v_out, weights_out, pos_out):
    """(descriptor, device) of a call."""
    torch = _torch()
    device, dtype = k_cache.get_device(), k_cache.dtype
    code = _dtype_code(k_cache)
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [batch, capacity, kv_heads, head_dim]")
    B, cap, Hk, D = k_cache.shape
    f32, i32 = torch.float32, torch.int32
    given = [x is not None for x in (k_out, v_out, weights_out, pos_out)]
    if any(given) != all(given):
        raise DepsyncError(EINVAL, "dep_cache_evict: k_out, v_out, weights_out and pos_out go together")
    cap_out, outs, rows_out = 0, (0, 0, 0, 0, 0), (0, 0)
    if k_out is not None:
        if k_out.dim() != 4:
            raise ValueError("k_out must be [batch, capacity, kv_heads, head_dim]")
        cap_out = k_out.shape[1]
        outs = _pair(k_out, v_out, "out", dtype, device, (B, cap_out, Hk, D))
        rows_out = _arr(weights_out, "weights_out", f32, device, (B, Hk, cap_out)), _arr(pos_out, "pos_out", i32, device, (B, Hk, cap_out))
    return _P_EVICT.pack(B, Hk, D, code, cap, max_cached or 0, budget, recent, *_pair(k_cache, v_cache, "cache", dtype, device, (B, cap, Hk, D)),
                         _arr(weights, "weights", f32, device, (B, Hk, cap)), _arr(pos, "pos", i32, device, (B, Hk, cap)),
                         _arr(cached, "cached", i32, device, (B,)), _arr(cached_out, "cached_out", i32, device, (B,)), cap_out, *outs, *rows_out), device


@functools.lru_cache(maxsize=4096)
def _evict_bytes(sizes: bytes, other: bool) -> int:
    """The workspace of dep_cache_evict, by the descriptor's eight sizes and whether other buffers are given: all that it depends on."""
    d = CacheEvictDesc.from_buffer_copy(sizes + bytes(_P_EVICT.size - len(sizes)))
    d.k_out = 16 if other else None
    need = ctypes.c_size_t(0)
    _check(_lib().depsync_cache_evict_workspace(ctypes.byref(d), ctypes.byref(need)), "dep_cache_evict")
    return need.value


def dep_cache_evict(k_cache, v_cache, weights, pos, cached, cached_out, budget: int, recent: int = 0, max_cached: Optional[int] = None,
                    k_out=None, v_out=None, weights_out=None, pos_out=None, workspace=None, stream=None) -> None:
    """Enqueue: every sequence and head keeps `budget` rows: the `recent` newest by position, then the heaviest, among equals the lowest row.
    In place kept rows behind the budget fill the places of those that go; into k_out .. pos_out (all four) the kept rows go in their order.
    cached_out = min(cached, budget).  stream: as for dep_tree_attn."""
    d, device = _cache_evict_desc(k_cache, v_cache, weights, pos, cached, cached_out, budget, recent, max_cached, k_out, v_out, weights_out, pos_out)
    stream = _current_or(stream, device)
    need = 0 if workspace is not None else _evict_bytes(d[:32], k_out is not None)
    keep, ptr, size = _workspace(need, workspace, device, stream)
    _call(device, "dep_cache_evict", _lib().dep_cache_evict, d, ptr, size, stream)


def cache_evict_workspace(k_cache, v_cache, weights, pos, cached, cached_out, budget: int, recent: int = 0, max_cached: Optional[int] = None,
                          k_out=None, v_out=None, weights_out=None, pos_out=None) -> int:
    """Bytes of workspace that dep_cache_evict with these arguments needs."""
    d, device = _cache_evict_desc(k_cache, v_cache, weights, pos, cached, cached_out, budget, recent, max_cached, k_out, v_out, weights_out, pos_out)
    return _bytes("depsync_cache_evict_workspace", device, _lib().depsync_cache_evict_workspace, d)


# ---- a round of drafts over a cache of 8 bits ------------------------------------------------

_P_TREE8 = struct.Struct("i4x 4P3q")
_P_APPEND8 = struct.Struct("8i 2P3q 2P3q 2P 2P3q 5P")
_P_NORM = struct.Struct("9if P3q P3q P3q P3q 5PqP")
_P_VERIFY = struct.Struct("3i4x P2q P2q 2PqP P 3P")


def _scales(k_scale, v_scale, device: int, shape):
    f32 = _torch().float32
    return _arr(k_scale, "k_scale", f32, device, shape), _arr(v_scale, "v_scale", f32, device, shape)


def _held8(k_cache, k_scale, v_scale, k_tail, v_tail, dtype, device: int):
    """(rows of a block, pointers of the scales, pointers and strides of the rows in 16 bits) of a cache of 8 bits."""
    if k_cache.dim() != 4 or k_tail.dim() != 4:
        raise ValueError("k_cache must be [batch, capacity, kv_heads, head_dim] and k_tail [batch, block, kv_heads, head_dim]")
    B, cap, Hk, D = k_cache.shape
    block = k_tail.shape[1]
    if block not in (32, 64, 128) or cap < block or cap % block:
        raise ValueError(f"blocks of {block} rows in a capacity of {cap}: blocks have 32, 64 or 128, and the capacity is a multiple")
    return block, *_scales(k_scale, v_scale, device, (B, Hk, cap // block)), *_pair(k_tail, v_tail, "tail", dtype, device, (B, block, Hk, D))


def _tree_attn8_desc(q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, out, lse, tree, drafted, scale, max_cached):
    """(descriptor, device) of a call."""
    if k_cache is None:
        raise ValueError("k_cache is missing: without a cache dep_tree_attn does it")
    d, device = _tree_attn_desc(q, k_new, v_new, k_cache, v_cache, cached, out, lse, tree, drafted, scale, max_cached, _torch().float8_e4m3fn)
    return d + _P_TREE8.pack(*_held8(k_cache, k_scale, v_scale, k_tail, v_tail, q.dtype, device)), device


@functools.lru_cache(maxsize=4096)
def _tree_attn8_bytes(device: int, sizes: bytes, block: bytes) -> int:
    """The workspace of dep_tree_attn8, by the descriptor's sizes: all that it depends on beside the device."""
    d = sizes + bytes(_P_TREE.size - len(sizes)) + block + bytes(_P_TREE8.size - len(block))
    return _bytes("dep_tree_attn8", device, _lib().depsync_tree_attn8_workspace, d, 0)


def dep_tree_attn8(q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, out, lse=None, tree=None, drafted=None,
                   scale: Optional[float] = None, max_cached: Optional[int] = None, workspace=None, stream=None) -> None:
    """Enqueue what dep_tree_attn does over a cache of 8 bits: the rows of full blocks in k_cache, v_cache [B, capacity, Hk, D] (float8_e4m3fn) with
    k_scale, v_scale [B, Hk, capacity / block] (float32), the rows behind them, cached % block of them, in k_tail, v_tail [B, block, Hk, D] (q's type)."""
    d, device = _tree_attn8_desc(q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, out, lse, tree, drafted, scale, max_cached)
    stream = _current_or(stream, device)
    need = 0 if workspace is not None else _tree_attn8_bytes(device, d[:32], d[_P_TREE.size:_P_TREE.size + 4])
    keep, ptr, size = _workspace(need, workspace, device, stream)
    _call(device, "dep_tree_attn8", _lib().dep_tree_attn8, d, ptr, size, stream)


def tree_attn8_workspace(q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, out, lse=None, tree=None, drafted=None,
                         scale: Optional[float] = None, max_cached: Optional[int] = None, n_cu: int = 0) -> int:
    """Bytes of workspace that dep_tree_attn8 with these arguments needs."""
    d, device = _tree_attn8_desc(q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, out, lse, tree, drafted, scale, max_cached)
    return _bytes("depsync_tree_attn8_workspace", device, _lib().depsync_tree_attn8_workspace, d, n_cu)


def dep_cache_append8(k_new, v_new, k_cache, v_cache, k_scale, v_scale, k_tail, v_tail, cached, cached_out, accepted=None, n_accepted=None,
                      n_out=None, stream=None) -> None:
    """Enqueue: drafted tokens accepted[b, :n_accepted[b]] (int32; None: the first ones) become rows cached[b].. of a cache of 8 bits (see dep_tree_attn8):
    blocks that are full now go into 8 bits with a scale of their own, the rows behind them into the tails.  cached_out = cached + n; n_out[b] (int32)
    receives n, which is less than n_accepted[b] where the capacity was reached."""
    torch = _torch()
    device, dtype = k_new.get_device(), k_new.dtype
    code = _dtype_code(k_new)
    if k_new.dim() != 4:
        raise ValueError("k_new must be [batch, tokens, kv_heads, head_dim]")
    B, T, Hk, D = k_new.shape
    block, ks, vs, *tail = _held8(k_cache, k_scale, v_scale, k_tail, v_tail, dtype, device)
    cap = k_cache.shape[1]
    i32 = torch.int32
    n_max, acc, n_acc = _accepted(B, T, accepted, n_accepted, device)
    d = _P_APPEND8.pack(B, T, Hk, D, code, cap, block, n_max, *_pair(k_new, v_new, "new", dtype, device, (B, T, Hk, D)),
                        *_pair(k_cache, v_cache, "cache", torch.float8_e4m3fn, device, (B, cap, Hk, D)), ks, vs, *tail, _arr(cached, "cached", i32, device, (B,)),
                        _arr(cached_out, "cached_out", i32, device, (B,)), acc, n_acc, _arr(n_out, "n_out", i32, device, (B,)))
    _call(device, "dep_cache_append8", _lib().dep_cache_append8, d, _current_or(stream, device))


def rope_frequencies(angles, device=None):
    """The `freq` of dep_qk_norm_rope for rotations by angles[i] radians a position (a float64 tensor or list of numbers below 2^100 in magnitude, in host memory or not): int64 [len],
    turns as fractions of 2^64.  On `device`, by default that of the angles.  Worked out exactly on the host, once for a model: angles in device memory are waited for."""
    from fractions import Fraction
    torch = _torch()
    t = torch.as_tensor(angles, dtype=torch.float64)
    if t.dim() != 1 or not bool((t.abs() < 2.0 ** 100).all()):
        raise ValueError("angles must be one finite number below 2^100 for each pair")
    turn = Fraction(2 * 314159265358979323846264338327950288419716939937510, 10 ** 50)   # 2 pi to 50 places: a turn is off by 2^-66 at most
    words = [round(Fraction(x) / turn * 2 ** 64) % 2 ** 64 for x in t.tolist()]
    return torch.tensor([w - 2 ** 64 if w >> 63 else w for w in words], dtype=torch.int64, device=t.device if device is None else device)


def dep_qk_norm_rope(q, k, freq=None, q_gain=None, k_gain=None, q_out=None, k_out=None, start=None, depth=None, drafted=None, eps: float = 1e-6,
                     norm: bool = True, interleaved: bool = False, stream=None) -> None:
    """Enqueue: every row x of q [B, T, Hq, D] and k [B, T, Hk, D] becomes x / sqrt(mean(x^2) + eps) * gain (norm False: x * gain), and the first 2 len(freq)
    numbers of that are rotated in pairs, pair i by position * freq[i] (see rope_frequencies; None: no rotation): i and i + len(freq), or, interleaved, 2 i and 2 i + 1.

    q_gain, k_gain [D] (float32; None: ones).  q_out, k_out: None is in place.  The position of token t is start[b] + depth[b, t] (int32 [B] and [B, T] or [T]; None: 0, and t).
    drafted[b] (int32): the tokens that sequence b has; the others' rows are left alone.  stream: as for dep_tree_attn."""
    torch = _torch()
    device, dtype = q.get_device(), q.dtype
    code = _dtype_code(q)
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [batch, tokens, heads, head_dim]")
    B, T, Hq, D = q.shape
    Hk = k.shape[2]
    qp, kp = _t4(q, "q", dtype, device), _t4(k, "k", dtype, device, (B, T, Hk, D))
    R, fp = 0, 0
    if freq is not None:
        if freq.dim() != 1:
            raise ValueError("freq must be one number for each pair")
        R, fp = 2 * freq.shape[0], _arr(freq, "freq", torch.int64, device, freq.shape)
    depth_ptr, depth_batch = 0, 0
    if depth is not None:
        depth_batch = T if depth.dim() == 2 else 0
        depth_ptr = _arr(depth, "depth", torch.int32, device, (B, T) if depth_batch else (T,))
    f32, i32 = torch.float32, torch.int32
    d = _P_NORM.pack(B, T, Hq, Hk, D, code, R, bool(interleaved), bool(norm), eps, *qp, *kp,
                     *(qp if q_out is None else _t4(q_out, "q_out", dtype, device, (B, T, Hq, D))),
                     *(kp if k_out is None else _t4(k_out, "k_out", dtype, device, (B, T, Hk, D))),
                     _arr(q_gain, "q_gain", f32, device, (D,)), _arr(k_gain, "k_gain", f32, device, (D,)), fp,
                     _arr(start, "start", i32, device, (B,)), depth_ptr, depth_batch, _arr(drafted, "drafted", i32, device, (B,)))
    _call(device, "dep_qk_norm_rope", _lib().dep_qk_norm_rope, d, _current_or(stream, device))


def _probabilities(t, name: str, device: int, shape):
    """Pointer and strides of a [batch, tokens, vocab] tensor of 32-bit numbers with contiguous rows; None -> zeros."""
    if t is None:
        return 0, 0, 0
    if t.get_device() != device or t.dtype is not _torch().float32 or t.shape != shape or (t.stride(2) != 1 and shape[2] > 1):
        raise ValueError(f"{name} must be a float32 tensor of shape {tuple(shape)} with contiguous rows on the device of the others")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _verify_desc(p, ids, u, accepted, n_accepted, next, q, parents, drafted):
    """(descriptor, device) of a call."""
    torch = _torch()
    device = p.get_device()
    if p.dim() != 3 or device < 0:
        raise ValueError("p must be a [batch, tokens, vocab] tensor on a GPU")
    B, T, V = p.shape
    i32 = torch.int32
    parents_ptr, parents_batch = 0, 0
    if parents is not None:
        parents_batch = T if parents.dim() == 2 else 0
        parents_ptr = _arr(parents, "parents", i32, device, (B, T) if parents_batch else (T,))
    return _P_VERIFY.pack(B, T, V, *_probabilities(p, "p", device, p.shape), *_probabilities(q, "q", device, p.shape), _arr(ids, "ids", i32, device, (B, T)),
                          parents_ptr, parents_batch, _arr(drafted, "drafted", i32, device, (B,)), _arr(u, "u", torch.float32, device, (B, T)),
                          _arr(accepted, "accepted", i32, device, (B, T)), _arr(n_accepted, "n_accepted", i32, device, (B,)),
                          _arr(next, "next", i32, device, (B,))), device


def dep_verify_drafts(p, ids, u, accepted, n_accepted, next, q=None, parents=None, drafted=None, workspace=None, stream=None) -> None:
    """Enqueue: which drafted tokens stay, and the token that follows them.  Token 0 of a sequence is known and stays; p [B, T, V] (float32) are the target's probabilities
    behind each token, q (same shape) those by which the draft drew each token's children (None: they were not drawn), ids [B, T] (int32) the tokens, parents [B, T] or [T]
    (int32; None: a chain) the tree, u [B, T] (float32) random numbers from [0, 1): u[:, 0] draws the next token, the others decide about theirs.

    accepted [B, T], n_accepted [B] and next [B] (int32) receive the tokens that stay (0 first), their number, and the next token: what the appends take.
    drafted[b] (int32): the tokens that sequence b has (None: all; 0: nothing to verify).  stream: as for dep_tree_attn."""
    d, device = _verify_desc(p, ids, u, accepted, n_accepted, next, q, parents, drafted)
    stream = _current_or(stream, device)
    need = 0 if workspace is not None else _verify_bytes(d)
    keep, ptr, size = _workspace(need, workspace, device, stream)
    _call(device, "dep_verify_drafts", _lib().dep_verify_drafts, d, ptr, size, stream)


def _verify_bytes(d: bytes) -> int:
    need = ctypes.c_size_t(0)
    _check(_lib().depsync_verify_drafts_workspace(d, ctypes.byref(need)), "dep_verify_drafts")
    return need.value


def verify_drafts_workspace(p, ids, u, accepted, n_accepted, next, q=None, parents=None, drafted=None) -> int:
    """Bytes of workspace that dep_verify_drafts with these arguments needs."""
    return _verify_bytes(_verify_desc(p, ids, u, accepted, n_accepted, next, q, parents, drafted)[0])


# ---- host mirrors -------------------------------------------------------------------------

def row_major(tile_x, tile_y, grid_x, grid_y) -> int:
    return _lib().depsync_row_major(tile_x, tile_y, grid_x, grid_y)


def policy_sem(kind, tile_x, tile_y, grid_x, grid_y, stride=0) -> int:
    return _lib().depsync_policy_sem(kind, tile_x, tile_y, grid_x, grid_y, stride)


def policy_value(kind, grid_x, grid_y, stride=0) -> int:
    return _lib().depsync_policy_value(kind, grid_x, grid_y, stride)


def wave_model(n_tiles, occupancy, n_cu):
    w, u = ctypes.c_int(), ctypes.c_double()
    _check(_lib().depsync_wave_model(n_tiles, occupancy, n_cu, ctypes.byref(w), ctypes.byref(u)), "depsync_wave_model")
    return w.value, u.value


def sync_count(kind, prod_grid, cons_grid, prod_rows_per_cons_row=1) -> int:
    return _lib().depsync_sync_count(kind, prod_grid[0], prod_grid[1], cons_grid[0], cons_grid[1],
                                     prod_rows_per_cons_row)


def mfma_calibration(zero_operands: bool = False, milliseconds: int = 200) -> float:
    """TFLOP/s a register-only bf16 MFMA loop sustains on this device (zero or random operands)."""
    out = ctypes.c_double(0.0)
    _check(_lib().depsync_mfma_calibration(int(zero_operands), milliseconds, ctypes.byref(out)), "depsync_mfma_calibration")
    return out.value


def simulate_chain(slots, prod_grid, d1, cons_grid, d2, halo=0, stream_sync=False) -> float:
    return _lib().depsync_simulate_chain(slots, prod_grid[0], prod_grid[1], d1, cons_grid[0], cons_grid[1], d2,
                                         halo, int(stream_sync))


def tile_shape(tile):
    r, c = ctypes.c_int(), ctypes.c_int()
    _check(_lib().depsync_tile_shape(tile, ctypes.byref(r), ctypes.byref(c)), "depsync_tile_shape")
    return r.value, c.value


def workspace_bytes() -> int:
    """Device memory a policy's workspace takes (split-K partial tiles not included)."""
    f = _lib().depsync_workspace_bytes
    f.restype = ctypes.c_size_t
    return int(f())


def device_info():
    n, k = ctypes.c_int(), ctypes.c_int()
    _check(_lib().depsync_device_info(ctypes.byref(n), ctypes.byref(k)), "depsync_device_info")
    return n.value, k.value
