"""Binding of the COVER C ABI (``include/cover.h``): ctypes, and a native form of the calls a
decoding step makes (``csrc/host.cpp``).

Argument marshalling only: torch supplies device memory and the stream; every step of the
computation runs in the HIP kernels of ``libcover.so``.  There is no fallback -- if the
libraries have not been built, or a call is rejected, an exception is raised.  A call goes to
its native form first; that makes it, or hands back what fails a check or is out of the
ordinary (None) to the Python form below it, which raises the error.

``stream`` is a torch stream or a HIP handle (None: the current stream): the kernels run on it, and what a
call allocates comes from its memory.  The caller orders it behind the work that made the inputs, and the
use of the results behind it.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

from .build import HOST, LIB

COVER_OK, COVER_ERR_INVALID, COVER_ERR_UNSUPPORTED, COVER_ERR_HIP = 0, -1, -2, -3
COVER_F32, COVER_BF16 = 0, 1
COVER_MAX_L = 65536
COVER_MAX_LR = 16384
COVER_RECT_RECORD = 68

EXPORTED = ("cover_attn_cached", "cover_attn_cached_plan", "cover_attn_cached_splits",
            "cover_attn_fwd", "cover_attn_rect", "cover_attn_stats", "cover_attn_stats_noalloc",
            "cover_attn_stats_workspace", "cover_cache_load", "cover_cache_store",
            "cover_debug_status", "cover_decode_update", "cover_rms_norm", "cover_rope", "cover_rope_freq",
            "cover_select_seeds", "cover_status_str", "cover_token_sample", "cover_token_stats",
            "cover_version")
# status bits of the contract checks that COVER_DEBUG=1 enables (cover_debug_status)
COVER_DEBUG_SEED_COUNT, COVER_DEBUG_SEED_RANGE, COVER_DEBUG_SEED_DUPLICATE = 1, 2, 4
COVER_DEBUG_SELECT_NONFINITE, COVER_DEBUG_SELECT_NEGATIVE = 8, 16
COVER_DEBUG_STORE_DUPLICATE = 32
COVER_NORM_MAX_D = 32768
COVER_CACHED_MAX_LQ = 2048
# how rope_freq scales frequencies (cover_rope_scaling)
ROPE_SCALING = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


class CoverError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_str(status)} ({status})")
        self.status = status


class AttnDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("L", ctypes.c_int32), ("d", ctypes.c_int32), ("max_seeds", ctypes.c_int32),
                ("dtype", ctypes.c_int), ("scale", ctypes.c_float),
                ("q_sb", ctypes.c_int64), ("q_sh", ctypes.c_int64), ("q_sl", ctypes.c_int64),
                ("kv_sb", ctypes.c_int64), ("kv_sh", ctypes.c_int64), ("kv_sl", ctypes.c_int64)]


class SelectDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Lr", ctypes.c_int32), ("max_seeds", ctypes.c_int32),
                ("pos_offset", ctypes.c_int32)]


class TokenDesc(ctypes.Structure):
    _fields_ = [("R", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int),
                ("row_stride", ctypes.c_int64)]


class UpdateDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Lr", ctypes.c_int32), ("max_seeds", ctypes.c_int32),
                ("pos_offset", ctypes.c_int32), ("mask_id", ctypes.c_int32),
                ("draft_cap", ctypes.c_int32), ("remask_budget", ctypes.c_int32),
                ("tau", ctypes.c_float), ("min_draft", ctypes.c_int32)]


class RectDesc(ctypes.Structure):
    _fields_ = [("attn", AttnDesc), ("q_off", ctypes.c_int32), ("Lq", ctypes.c_int32),
                ("n_split", ctypes.c_int32)]


class StatsDesc(ctypes.Structure):
    _fields_ = [("attn", AttnDesc), ("r0", ctypes.c_int32), ("Lr", ctypes.c_int32)]


def _fields(ints: str, reals: str, strides: str, dtype: bool = True):
    return ([(n, ctypes.c_int32) for n in ints.split()] + ([("dtype", ctypes.c_int)] if dtype else [])
            + [(n, ctypes.c_float) for n in reals.split()] + [(n, ctypes.c_int64) for n in strides.split()])


class NormDesc(ctypes.Structure):
    _fields_ = _fields("R D", "eps", "x_stride res_stride res_out_stride out_stride")


class RopeDesc(ctypes.Structure):
    _fields_ = _fields("B L Hq Hkv d rot interleaved", "attention_factor",
                       "pos_sb q_sb q_sh q_sl qo_sb qo_sh qo_sl k_sb k_sh k_sl ko_sb ko_sh ko_sl")


class CacheDesc(ctypes.Structure):
    _fields_ = _fields("B H N L d first", "", "k_sb k_sh k_sl v_sb v_sh v_sl c_sb c_sh c_sl s_sb s_sh")


class CachedDesc(ctypes.Structure):
    _fields_ = _fields("B Hq Hkv L Lq d max_seeds q_off n_split", "scale",
                       "q_sb q_sh q_sl o_sb o_sh o_sl k_sb k_sh k_sl v_sb v_sh v_sl c_sb c_sh c_sl s_sb s_sh", False)


def attn_stats_workspace(B: int, Hq: int, Lr: int) -> int:
    """Floats of workspace a cover_attn_stats call of this size asks for (the library's
    cover_attn_stats_workspace)."""
    n = lib().cover_attn_stats_workspace(int(B), int(Hq), int(Lr))
    if n < 0:
        raise ValueError("negative size")
    return int(n)


_lib = None
_lib_path = LIB
_host = None


def use_library(path: str) -> None:
    """Load the library from `path` instead of libcover.so (the in-tree timing build of the
    same sources, for measurements).  Must come before the first call."""
    global _lib_path
    if _lib is not None and path != _lib_path:
        raise RuntimeError("the COVER library is already loaded")
    _lib_path = path


def host():
    """The calls' native forms (csrc/host.cpp, built in-tree) on the loaded library."""
    global _host
    if _host is None:
        import importlib.machinery
        import importlib.util

        if not os.path.exists(HOST):
            raise RuntimeError(f"the binding's native part is not built ({HOST}); run "
                               "`python -m paper_2602_06161_amd.build` or __graft_entry__.build()")
        loader = importlib.machinery.ExtensionFileLoader("_cover_host", HOST)
        m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_cover_host", loader))
        loader.exec_module(m)
        L = lib()
        m.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.cover_attn_fwd, L.cover_select_seeds, L.cover_token_stats, L.cover_token_sample,
            L.cover_attn_stats, L.cover_attn_stats_workspace, L.cover_decode_update)))
        m.bind_layer(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.cover_rms_norm, L.cover_rope, L.cover_cache_store, L.cover_cache_load, L.cover_attn_cached,
            L.cover_attn_cached_splits)))
        _host = m
    return _host


def lib():
    """Load libcover.so (built in-tree); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_lib_path):
            raise RuntimeError(f"COVER HIP library not built ({_lib_path}); run "
                               "`python -m paper_2602_06161_amd.build` or __graft_entry__.build()")
        L = ctypes.CDLL(_lib_path)
        P = ctypes.c_void_p
        L.cover_attn_fwd.argtypes = [P, P, P, P, P, P, P, P, P, ctypes.POINTER(AttnDesc), P]
        L.cover_attn_fwd.restype = ctypes.c_int
        L.cover_select_seeds.argtypes = [P, P, P, P, P, P, P, ctypes.POINTER(SelectDesc), P]
        L.cover_select_seeds.restype = ctypes.c_int
        L.cover_token_stats.argtypes = [P, P, P, P, P, ctypes.POINTER(TokenDesc), P]
        L.cover_attn_rect.argtypes = [P, P, P, P, P, P, P, P, P, P, ctypes.POINTER(RectDesc), P]
        L.cover_attn_rect.restype = ctypes.c_int
        L.cover_decode_update.argtypes = [P, P, P, P, P, P, P, P, P, P, P,
                                          ctypes.POINTER(UpdateDesc), P]
        L.cover_decode_update.restype = ctypes.c_int
        L.cover_token_stats.restype = ctypes.c_int
        L.cover_token_sample.argtypes = [P, ctypes.c_float, ctypes.c_uint64, ctypes.c_uint32, P, P,
                                         ctypes.POINTER(TokenDesc), P]
        L.cover_token_sample.restype = ctypes.c_int
        L.cover_attn_stats.argtypes = [P, P, P, P, P, P, P, P, P, P, P, ctypes.POINTER(StatsDesc), P]
        L.cover_attn_stats.restype = ctypes.c_int
        L.cover_attn_stats_noalloc.argtypes = [P, P, P, P, P, P, P, P, P, P,
                                               ctypes.POINTER(StatsDesc), P]
        L.cover_attn_stats_noalloc.restype = ctypes.c_int
        L.cover_attn_stats_workspace.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        L.cover_attn_stats_workspace.restype = ctypes.c_int64
        L.cover_rms_norm.argtypes = [P] * 6 + [ctypes.POINTER(NormDesc), P]
        L.cover_rope.argtypes = [P] * 6 + [ctypes.POINTER(RopeDesc), P]
        L.cover_rope_freq.argtypes = [P, ctypes.c_int32, ctypes.c_double, ctypes.c_int] + [ctypes.c_double] * 4
        L.cover_cache_store.argtypes = [P] * 7 + [ctypes.POINTER(CacheDesc), P]
        L.cover_cache_load.argtypes = [P] * 7 + [ctypes.POINTER(CacheDesc), P]
        L.cover_attn_cached.argtypes = [P] * 14 + [ctypes.POINTER(CachedDesc), P]
        L.cover_attn_cached_splits.argtypes = [ctypes.c_int32] * 5
        L.cover_attn_cached_plan.argtypes = [ctypes.c_int32] * 7 + [ctypes.POINTER(ctypes.c_int32)] * 2
        L.cover_attn_cached_plan.restype = ctypes.c_int
        for f in (L.cover_rms_norm, L.cover_rope, L.cover_rope_freq, L.cover_cache_store, L.cover_cache_load,
                  L.cover_attn_cached):
            f.restype = ctypes.c_int
        L.cover_attn_cached_splits.restype = ctypes.c_int32
        L.cover_status_str.argtypes = [ctypes.c_int]
        L.cover_status_str.restype = ctypes.c_char_p
        L.cover_version.argtypes = []
        L.cover_version.restype = ctypes.c_int32
        L.cover_debug_status.argtypes = [ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, P]
        L.cover_debug_status.restype = ctypes.c_int
        _lib = L
    return _lib


def status_str(s: int) -> str:
    return lib().cover_status_str(s).decode()


def version() -> int:
    return lib().cover_version()


def debug_status(clear: bool = False, stream=None) -> int:
    """The contract-violation bits recorded under COVER_DEBUG=1 on the current GPU (waits
    for `stream`); optionally reset them."""
    v = ctypes.c_int32(0)
    st = lib().cover_debug_status(ctypes.byref(v), 1 if clear else 0, _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_debug_status")
    return v.value


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _raw_stream(stream) -> int:
    """The HIP stream handle `stream` stands for (None: the current stream; without an initialised
    GPU 0, which nothing uses: no tensor is on a GPU then)."""
    if stream is None:
        if not torch.cuda.is_initialized():
            return 0
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _other(stream):
    """`stream` as a torch stream where it is not the current one, else None."""
    if not torch.cuda.is_initialized():
        return None
    raw = stream if isinstance(stream, int) else stream.cuda_stream
    if raw == torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()):
        return None
    if not isinstance(stream, int):
        return stream
    return torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()


def _run_on(stream, call, *args, **kw):
    """call(*args, **kw) with `stream` as the current one.  What the call allocates comes from that stream's
    memory (what the caller's stream has freed may still be in use there), and is not given out again before the
    caller's stream, too, has passed the point where it is dropped."""
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        done = call(*args, **kw)
    given = {id(x) for x in (*args, *kw.values())}
    for t in done:
        if t is not None and id(t) not in given:
            t.record_stream(here)
    return done


def attn_desc(q: torch.Tensor, k: torch.Tensor, max_seeds: int, scale: float = 0.0) -> AttnDesc:
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    dt = {torch.float32: COVER_F32, torch.bfloat16: COVER_BF16}.get(q.dtype)
    if dt is None:
        raise TypeError(f"unsupported dtype {q.dtype}")
    return AttnDesc(B, Hq, Hkv, L, d, max_seeds, dt, float(scale),
                    q.stride(0), q.stride(1), q.stride(2), k.stride(0), k.stride(1), k.stride(2))


def cover_attn_fwd(q, k_live, v_live, k_cache, v_cache, seed_idx=None, n_seed=None, out=None,
                   lse=None, scale: float = 0.0, stream=None, want_lse: bool = True):
    """COVER attention of one layer.  Tensors on the GPU: q [B,Hq,L,d]; k/v [B,Hkv,L,d]
    (head dim contiguous, all four K/V tensors with identical strides); seed_idx int32
    [B,max_seeds]; n_seed int32 [B].  Returns (out, lse)."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_attn_fwd, q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed, out, lse, scale,
                       want_lse=want_lse)
    done = (_host or host()).attn_fwd(q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed, out, lse,
                                       scale, want_lse, _raw_stream(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_attn_fwd")
    for t in (k_live, v_live, k_cache, v_cache):
        if t.shape != k_live.shape or t.stride() != k_live.stride() or t.dtype != q.dtype:
            raise ValueError("k_live, v_live, k_cache, v_cache need equal shape, strides and dtype")
    if q.stride(-1) != 1 or k_live.stride(-1) != 1:
        raise ValueError("head dimension must be contiguous")
    max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
    if seed_idx is not None and (seed_idx.dtype != torch.int32 or n_seed is None
                                 or n_seed.dtype != torch.int32 or not seed_idx.is_contiguous()):
        raise ValueError("seed_idx and n_seed must be contiguous int32 tensors")
    B, Hq, L, d = q.shape
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.stride() != q.stride() or out.dtype != q.dtype:
        raise ValueError("out must match q's shape, strides and dtype")
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, L), device=q.device, dtype=torch.float32)
    desc = attn_desc(q, k_live, max_seeds, scale)
    st = lib().cover_attn_fwd(_ptr(q), _ptr(k_live), _ptr(v_live), _ptr(k_cache), _ptr(v_cache),
                              _ptr(seed_idx), _ptr(n_seed), _ptr(out), _ptr(lse),
                              ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_attn_fwd")
    return out, lse


def rect_workspace(B: int, Hq: int, Lq: int, n_split: int) -> int:
    """Floats of workspace cover_attn_rect needs (COVER_ATTN_RECT_WORKSPACE): none for the
    single launch (n_split == 1)."""
    return B * Hq * n_split * Lq * COVER_RECT_RECORD if n_split > 1 else 0


def rect_splits(B: int, Hq: int, Lq: int, L: int) -> int:
    """Key splits.  1 (the single launch: one workgroup per 32 query rows, its waves split the
    keys) unless the sequence is long and the block leaves most CUs idle: that kernel reads
    all of a head's K and V through one CU per 32 rows, about 100 GB/s per CU, so past 2048
    keys with fewer than 256 workgroups the keys are split across workgroups instead (1 to 8
    rounds of 256 workgroups of at least 128 keys each, merged by a second launch)."""
    if L <= 2048 or B * Hq * ((Lq + 31) // 32) >= 256:
        return 1
    tiles, stages = B * Hq * ((Lq + 31) // 32), -(-L // 32)
    # rounds of 256 workgroups, each as long as its stages and about 18 stages' worth of start
    # and merge; 24 for the second launch.  The candidates fill 1 to 8 rounds.
    best, least = 1, stages + 18
    for rounds in range(1, 9):
        n = min(256 * rounds // tiles, 256, -(-L // 128))
        if n > 1:
            length = -(-stages // n)
            n = -(-stages // length)  # the fewest splits of that length
            cost = -(-tiles * n // 256) * (length + 18) + 24
            if cost < least:
                best, least = n, cost
    return best


def _rect_plan(B: int, Hq: int, Lq: int, L: int, n_split, workspace):
    """(n_split, floats of workspace) of a call; without an n_split of the caller's as many splits
    as rect_splits says, or as a smaller workspace of the caller's holds (two at least)."""
    if n_split is None:
        n_split = rect_splits(B, Hq, Lq, L)
        if workspace is not None and n_split > 2:
            n_split = min(n_split, max(2, workspace.numel() // (B * Hq * Lq * COVER_RECT_RECORD)))
    return n_split, rect_workspace(B, Hq, Lq, n_split)


def cover_attn_rect(q, k_live, v_live, k_cache, v_cache, q_off: int, seed_idx=None, n_seed=None,
                    out=None, lse=None, scale: float = 0.0, n_split=None, workspace=None,
                    want_lse: bool = True, stream=None):
    """COVER attention of the query block [q_off, q_off + Lq) against all L keys.  q
    [B,Hq,Lq,d] bf16; k/v [B,Hkv,L,d] (equal strides); seeds as for cover_attn_fwd (absolute
    positions).  Returns (out [B,Hq,Lq,d], lse [B,Hq,Lq])."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_attn_rect, q, k_live, v_live, k_cache, v_cache, q_off, seed_idx, n_seed, out, lse,
                       scale, n_split, workspace, want_lse)
    for t in (k_live, v_live, k_cache, v_cache):
        if t.shape != k_live.shape or t.stride() != k_live.stride() or t.dtype != q.dtype:
            raise ValueError("k_live, v_live, k_cache, v_cache need equal shape, strides and dtype")
    if q.stride(-1) != 1 or k_live.stride(-1) != 1:
        raise ValueError("head dimension must be contiguous")
    max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
    if seed_idx is not None and (seed_idx.dtype != torch.int32 or n_seed is None
                                 or n_seed.dtype != torch.int32 or not seed_idx.is_contiguous()):
        raise ValueError("seed_idx and n_seed must be contiguous int32 tensors")
    B, Hq, Lq, d = q.shape
    L = k_live.shape[2]
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.stride() != q.stride() or out.dtype != q.dtype:
        raise ValueError("out must match q's shape, strides and dtype")
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, Lq), device=q.device, dtype=torch.float32)
    n_split, need = _rect_plan(B, Hq, Lq, L, n_split, workspace)
    if need == 0:
        workspace = None  # not used by the single launch
    elif workspace is None:
        workspace = torch.empty(need, device=q.device, dtype=torch.float32)
    if workspace is not None and (workspace.dtype != torch.float32 or workspace.numel() < need
                                  or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous fp32 with at least {need} elements")
    ad = attn_desc(q, k_live, max_seeds, scale)
    ad.L = L
    desc = RectDesc(ad, q_off, Lq, n_split)
    st = lib().cover_attn_rect(_ptr(q), _ptr(k_live), _ptr(v_live), _ptr(k_cache), _ptr(v_cache),
                               _ptr(seed_idx), _ptr(n_seed), _ptr(out), _ptr(lse), _ptr(workspace),
                               ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_attn_rect")
    return out, lse


def cover_select_seeds(logp, d_in, d_out, flags, max_seeds: int, pos_offset: int = 0,
                       seed_idx=None, n_seed=None, score=None, want_score: bool = True,
                       stream=None):
    """Stability-aware seed selection.  logp/d_in/d_out fp32 [B,Lr], flags uint8 [B,Lr] on the
    GPU (contiguous).  Returns (seed_idx int32 [B,max_seeds], n_seed int32 [B], score fp64
    [B,Lr] or None)."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_select_seeds, logp, d_in, d_out, flags, max_seeds, pos_offset, seed_idx, n_seed,
                       score, want_score)
    done = (_host or host()).select_seeds(logp, d_in, d_out, flags, max_seeds, pos_offset, seed_idx,
                                           n_seed, score, want_score, _raw_stream(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_select_seeds")
    B, Lr = logp.shape
    for t, dt in ((logp, torch.float32), (d_in, torch.float32), (d_out, torch.float32),
                  (flags, torch.uint8)):
        if t.shape != (B, Lr) or t.dtype != dt or not t.is_contiguous():
            raise ValueError("selection inputs must be contiguous [B,Lr] (fp32 x3, uint8 flags)")
    dev = logp.device
    if seed_idx is None:
        seed_idx = torch.empty((B, max_seeds), device=dev, dtype=torch.int32)
    if n_seed is None:
        n_seed = torch.empty((B,), device=dev, dtype=torch.int32)
    if score is None and want_score:
        score = torch.empty((B, Lr), device=dev, dtype=torch.float64)
    desc = SelectDesc(B, Lr, max_seeds, pos_offset)
    st = lib().cover_select_seeds(_ptr(logp), _ptr(d_in), _ptr(d_out), _ptr(flags),
                                  _ptr(seed_idx), _ptr(n_seed), _ptr(score), ctypes.byref(desc),
                                  _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_select_seeds")
    return seed_idx, n_seed, score


def cover_decode_update(tokens, argmax, conf, seed_idx, n_seed, remask_count, mask_id: int,
                        tau: float, draft_cap: int, remask_budget: int, pos_offset: int = 0,
                        flags=None, drafted=None, counts=None, want_outputs: bool = True,
                        last_unmask=None, flipflops=None, min_draft: int = 0, stream=None):
    """One step's decoding-state update, in place on tokens and remask_count (int32 [B,Lr]);
    argmax int32 / conf fp32 [B,Lr]; seed_idx int32 [B,max_seeds], n_seed int32 [B] (may be
    None: no seeds).  Returns (flags uint8, drafted uint8, counts int32 [B,5]), allocated
    unless given (None when want_outputs is False).  With last_unmask (int32 [B,Lr], in
    place) the step's flip-flop events go to flipflops (int32 [B], allocated unless given),
    returned as a fourth element."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_decode_update, tokens, argmax, conf, seed_idx, n_seed, remask_count, mask_id, tau,
                       draft_cap, remask_budget, pos_offset, flags, drafted, counts, want_outputs, last_unmask,
                       flipflops, min_draft)
    if last_unmask is None and flipflops is None:
        done = (_host or host()).decode_update(tokens, argmax, conf, seed_idx, n_seed, remask_count, mask_id,
                                                tau, draft_cap, remask_budget, pos_offset, flags,
                                                drafted, counts, want_outputs, min_draft, _raw_stream(stream))
        if done.__class__ is tuple:
            return done
        if done is not None:
            raise CoverError(done, "cover_decode_update")
    B, Lr = tokens.shape
    for t, dt in ((tokens, torch.int32), (argmax, torch.int32), (conf, torch.float32),
                  (remask_count, torch.int32)):
        if t.shape != (B, Lr) or t.dtype != dt or not t.is_contiguous():
            raise ValueError("update inputs must be contiguous [B,Lr] (int32 x3, fp32 conf)")
    max_seeds = 0
    if seed_idx is not None:
        if seed_idx.dim() != 2 or seed_idx.shape[0] != B or seed_idx.dtype != torch.int32 or \
                not seed_idx.is_contiguous() or n_seed is None or n_seed.shape != (B,) or \
                n_seed.dtype != torch.int32:
            raise ValueError("seed_idx must be contiguous int32 [B,max_seeds], n_seed int32 [B]")
        max_seeds = seed_idx.shape[1]
    dev = tokens.device
    if want_outputs:
        flags = torch.empty((B, Lr), device=dev, dtype=torch.uint8) if flags is None else flags
        drafted = torch.empty((B, Lr), device=dev, dtype=torch.uint8) if drafted is None else drafted
        counts = torch.empty((B, 5), device=dev, dtype=torch.int32) if counts is None else counts
    for t, shape, dt in ((flags, (B, Lr), torch.uint8), (drafted, (B, Lr), torch.uint8),
                         (counts, (B, 5), torch.int32), (last_unmask, (B, Lr), torch.int32),
                         (flipflops, (B,), torch.int32)):
        if t is not None and (t.shape != shape or t.dtype != dt or not t.is_contiguous()):
            raise ValueError("flags/drafted must be contiguous uint8 [B,Lr], counts int32 [B,5], "
                             "last_unmask int32 [B,Lr], flipflops int32 [B]")
    if last_unmask is not None and flipflops is None:
        flipflops = torch.empty((B,), device=dev, dtype=torch.int32)
    desc = UpdateDesc(B, Lr, max_seeds, pos_offset, mask_id, draft_cap, remask_budget, tau,
                      min_draft)
    st = lib().cover_decode_update(_ptr(tokens), _ptr(argmax), _ptr(conf),
                                   _ptr(seed_idx) if max_seeds else None,
                                   _ptr(n_seed) if max_seeds else None, _ptr(remask_count),
                                   _ptr(flags), _ptr(drafted), _ptr(counts), _ptr(last_unmask),
                                   _ptr(flipflops), ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_decode_update")
    if last_unmask is not None:
        return flags, drafted, counts, flipflops
    return flags, drafted, counts


def cover_token_sample(logits, temperature: float, seed: int, step: int, want_prob: bool = True,
                       stream=None):
    """Temperature sampling per row of logits [R, V] (bf16 or fp32, last dimension
    contiguous, row stride a multiple of 16 bytes).  Returns (token int32 [R], prob fp32 [R]
    or None)."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_token_sample, logits, temperature, seed, step, want_prob)
    done = (_host or host()).token_sample(logits, temperature, seed, step, want_prob, _raw_stream(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_token_sample")
    R, V = logits.shape
    dt = {torch.float32: COVER_F32, torch.bfloat16: COVER_BF16}.get(logits.dtype)
    if dt is None or logits.stride(-1) != 1:
        raise ValueError("logits must be bf16 or fp32 with a contiguous last dimension")
    token = torch.empty(R, device=logits.device, dtype=torch.int32)
    prob = torch.empty(R, device=logits.device, dtype=torch.float32) if want_prob else None
    desc = TokenDesc(R, V, dt, logits.stride(0))
    st = lib().cover_token_sample(_ptr(logits), float(temperature), int(seed) & (2**64 - 1),
                                  int(step) & 0xFFFFFFFF, _ptr(token), _ptr(prob),
                                  ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_token_sample")
    return token, prob


def cover_token_stats(logits, tokens=None, want_logp: bool = True, want_conf: bool = True,
                      want_argmax: bool = True, stream=None):
    """Per-row log p(token), max probability and argmax of logits [R, V] (bf16 or fp32, last
    dimension contiguous, row stride a multiple of 16 bytes).  Returns (logp, conf, argmax),
    each None when not requested."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_token_stats, logits, tokens, want_logp, want_conf, want_argmax)
    done = (_host or host()).token_stats(logits, tokens, want_logp, want_conf, want_argmax, _raw_stream(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_token_stats")
    R, V = logits.shape
    dt = {torch.float32: COVER_F32, torch.bfloat16: COVER_BF16}.get(logits.dtype)
    if dt is None or logits.stride(-1) != 1:
        raise ValueError("logits must be bf16 or fp32 with a contiguous last dimension")
    if want_logp and (tokens is None or tokens.dtype != torch.int32 or tokens.shape != (R,)
                      or not tokens.is_contiguous()):
        raise ValueError("tokens must be a contiguous int32 [R] tensor")
    dev = logits.device
    logp = torch.empty(R, device=dev, dtype=torch.float32) if want_logp else None
    conf = torch.empty(R, device=dev, dtype=torch.float32) if want_conf else None
    amax = torch.empty(R, device=dev, dtype=torch.int32) if want_argmax else None
    desc = TokenDesc(R, V, dt, logits.stride(0))
    st = lib().cover_token_stats(_ptr(logits), _ptr(tokens if want_logp else None), _ptr(logp),
                                 _ptr(conf), _ptr(amax), ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_token_stats")
    return logp, conf, amax


def cover_attn_stats(q, k_live, k_cache, seed_idx, n_seed, lse, masked, drafted, r0: int,
                     scale: float = 0.0, workspace=None, stream=None):
    """d_in, d_out [B, Lr] over the region [r0, r0+Lr) (Lr = masked.shape[1]) from the corrected
    attention weights of cover_attn_fwd (lse from that call).  bf16 q/k; masked, drafted
    uint8 [B, Lr]."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_attn_stats, q, k_live, k_cache, seed_idx, n_seed, lse, masked, drafted, r0, scale,
                       workspace)
    done = (_host or host()).attn_stats(q, k_live, k_cache, seed_idx, n_seed, lse, masked, drafted, r0,
                                         scale, workspace, _raw_stream(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_attn_stats")
    B, Hq, L, d = q.shape
    Lr = masked.shape[1]
    for t in (k_live, k_cache):
        if t.shape != k_live.shape or t.stride() != k_live.stride() or t.dtype != q.dtype:
            raise ValueError("k_live and k_cache need equal shape, strides and dtype")
    for t in (masked, drafted):
        if t.shape != (B, Lr) or t.dtype != torch.uint8 or not t.is_contiguous():
            raise ValueError("masked / drafted must be contiguous uint8 [B, Lr]")
    if lse.shape != (B, Hq, L) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be contiguous fp32 [B, Hq, L]")
    max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
    dev = q.device
    d_in = torch.empty((B, Lr), device=dev, dtype=torch.float32)
    d_out = torch.empty((B, Lr), device=dev, dtype=torch.float32)
    need = attn_stats_workspace(B, Hq, Lr)
    if workspace is None:
        workspace = torch.empty(max(1, need), device=dev, dtype=torch.float32)
    elif (workspace.dtype != torch.float32 or not workspace.is_contiguous()
          or workspace.numel() < need or workspace.device != dev):
        raise ValueError(f"workspace must be a contiguous fp32 tensor of at least {need} floats "
                         f"on {dev}")
    desc = StatsDesc(attn_desc(q, k_live, max_seeds, scale), int(r0), int(Lr))
    st = lib().cover_attn_stats(_ptr(q), _ptr(k_live), _ptr(k_cache), _ptr(seed_idx),
                                _ptr(n_seed), _ptr(lse), _ptr(masked), _ptr(drafted), _ptr(d_in),
                                _ptr(d_out), _ptr(workspace), ctypes.byref(desc), _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_attn_stats")
    return d_in, d_out


COVER_STATS_SCRATCH_FLOATS = 1 << 20


def cover_attn_stats_noalloc(q, k_live, k_cache, seed_idx, n_seed, lse, masked, drafted,
                             r0: int, d_in, d_out, scale: float = 0.0, stream=None):
    """cover_attn_stats with the library's own per-GPU workspace: nothing is allocated, so the
    outputs d_in, d_out (contiguous fp32 [B, Lr]) are the caller's."""
    B, Hq, L, d = q.shape
    Lr = masked.shape[1]
    for t in (k_live, k_cache):
        if t.shape != k_live.shape or t.stride() != k_live.stride() or t.dtype != q.dtype:
            raise ValueError("k_live and k_cache need equal shape, strides and dtype")
    for t in (masked, drafted):
        if t.shape != (B, Lr) or t.dtype != torch.uint8 or not t.is_contiguous():
            raise ValueError("masked / drafted must be contiguous uint8 [B, Lr]")
    if lse.shape != (B, Hq, L) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be contiguous fp32 [B, Hq, L]")
    for t in (d_in, d_out):
        if t.shape != (B, Lr) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("d_in / d_out must be contiguous fp32 [B, Lr]")
    max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
    desc = StatsDesc(attn_desc(q, k_live, max_seeds, scale), int(r0), int(Lr))
    st = lib().cover_attn_stats_noalloc(_ptr(q), _ptr(k_live), _ptr(k_cache), _ptr(seed_idx),
                                        _ptr(n_seed), _ptr(lse), _ptr(masked), _ptr(drafted),
                                        _ptr(d_in), _ptr(d_out), ctypes.byref(desc),
                                        _stream(stream))
    if st != COVER_OK:
        raise CoverError(st, "cover_attn_stats_noalloc")
    return d_in, d_out


# ---- the layer's operators around the attention, with the 8-bit cache -------------------------------
def _place(stream):
    """The HIP stream handle `stream` stands for and the current GPU (0 and -1 without an initialised
    one: no tensor is on a GPU then)."""
    if not torch.cuda.is_initialized():
        return 0, -1
    dev = torch._C._cuda_getDevice()
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev), dev
    return (stream if isinstance(stream, int) else stream.cuda_stream), dev


def _on_gpu(**tensors):
    for name, t in tensors.items():
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device.index != torch.cuda.current_device():
            raise ValueError(f"{name} must be a tensor on the current GPU")


def _dtype(t, name: str) -> int:
    dt = {torch.float32: COVER_F32, torch.bfloat16: COVER_BF16}.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be bf16 or fp32, not {t.dtype}")
    return dt


def _empty_rows(R: int, D: int, dtype, device):
    """[R, D] whose rows start at multiples of 16 bytes."""
    per = 16 // dtype.itemsize
    return torch.empty((R, -(-D // per) * per), dtype=dtype, device=device)[:, :D]


def _int32(n, name: str) -> int:
    if not -2**31 <= int(n) < 2**31:
        raise ValueError(f"{name} must be a 32-bit integer")
    return int(n)


def _check(st: int, what: str) -> None:
    if st != COVER_OK:
        raise CoverError(st, what)


def cover_rms_norm(x, weight=None, residual=None, eps: float = 1e-6, quantize: bool = False, out=None,
                   residual_out=None, scale=None, stream=None):
    """Residual addition and root-mean-square norm of x [R, D] (bf16 or fp32; last dimension
    contiguous).  The rows of x, residual and the outputs start at multiples of 16 bytes, and so does weight [D]
    (contiguous, x's type): a contiguous [R, D] qualifies where D elements are a multiple of 16 bytes, other D need
    rows that are padded.  Returns (out, residual_out, scale): out [R, D] in
    x's type, or with quantize the codes (float8_e4m3fn) and scale fp32 [R] of its e4m3 form; residual_out
    = x + residual rounded to x's type (None without a residual).  residual_out may be x or residual, and
    out (without quantize) may be x."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_rms_norm, x, weight, residual, eps, quantize, out, residual_out, scale)
    done = (_host or host()).rms_norm(x, weight, residual, eps, quantize, out, residual_out, scale, *_place(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_rms_norm")
    _on_gpu(x=x, weight=weight, residual=residual, out=out, residual_out=residual_out, scale=scale)
    dt = _dtype(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [R, D]")
    R, D = x.shape
    if weight is not None and (weight.shape != (D,) or weight.dtype != x.dtype or not weight.is_contiguous()):
        raise ValueError("weight must be contiguous [D] of x's type")
    if not quantize and scale is not None:
        raise ValueError("scale is for quantize=True")
    if residual is None and residual_out is not None:
        raise ValueError("residual_out needs a residual")
    codes = torch.float8_e4m3fn if quantize else x.dtype
    if out is None:
        out = _empty_rows(R, D, codes, x.device)
    if residual is not None and residual_out is None:
        residual_out = _empty_rows(R, D, x.dtype, x.device)
    if quantize and scale is None:
        scale = torch.empty(R, device=x.device, dtype=torch.float32)
    for t, kind in ((x, x.dtype), (residual, x.dtype), (residual_out, x.dtype), (out, codes)):
        if t is not None and (t.shape != (R, D) or t.dtype != kind or (D > 1 and t.stride(1) != 1)):
            raise ValueError("x, residual, residual_out and out must be [R, D] of x's type (out float8_e4m3fn with "
                             "quantize) with a contiguous last dimension")
    if scale is not None and (scale.shape != (R,) or scale.dtype != torch.float32 or not scale.is_contiguous()):
        raise ValueError("scale must be contiguous fp32 [R]")
    step = lambda t: 0 if t is None else t.stride(0)  # noqa: E731
    desc = NormDesc(R, D, dt, float(eps), step(x), step(residual), step(residual_out), step(out))
    _check(lib().cover_rms_norm(_ptr(x), _ptr(residual), _ptr(weight), _ptr(residual_out), _ptr(out), _ptr(scale),
                                ctypes.byref(desc), _stream(stream)), "cover_rms_norm")
    return out, residual_out, scale


def rope_freq(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
              original_length: float = 0.0, low: float = 1.0, high: float = 32.0, device=None):
    """The frequencies cover_rope takes, fp64 [rot / 2] in turns per position: base^(-2 i / rot) / (2 pi),
    scaled for longer contexts by `scaling`: "plain", "linear" (positions interpolated by factor), "base" (the
    base raised so that the slowest frequency is interpolated) or "parts" (only frequencies with few turns
    over original_length are; between low and high turns in part)."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling must be one of {', '.join(ROPE_SCALING)}")
    freq = torch.empty(max(int(rot), 0) // 2, dtype=torch.float64, device="cpu")
    _check(lib().cover_rope_freq(_ptr(freq), int(rot), float(base), ROPE_SCALING[scaling], float(factor),
                                 float(original_length), float(low), float(high)), "cover_rope_freq")
    return freq if device is None else freq.to(device)


def cover_rope(q, k, pos, freq, interleaved: bool = False, attention_factor: float = 1.0, q_out=None, k_out=None,
               stream=None):
    """Rotary positions of q [B,Hq,L,d] and k [B,Hkv,L,d] (bf16 or fp32, head dimension contiguous; k may
    be None; strides and first elements multiples of 16 bytes).  pos int32 [B,L] or [L]; freq fp64 [rot / 2] on the GPU (rope_freq).  Returns (q_out, k_out),
    allocated unless given; they may be q and k themselves."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_rope, q, k, pos, freq, interleaved, attention_factor, q_out, k_out)
    done = (_host or host()).rope(q, k, pos, freq, interleaved, attention_factor, q_out, k_out, *_place(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_rope")
    _on_gpu(q=q, k=k, pos=pos, freq=freq, q_out=q_out, k_out=k_out)
    dt = _dtype(q, "q")
    if q.dim() != 4:
        raise ValueError("q must be [B,Hq,L,d]")
    B, Hq, L, d = q.shape
    if k is None and k_out is not None:
        raise ValueError("k_out needs k")
    if k is not None and (k.dim() != 4 or k.shape[0] != B or k.shape[2:] != q.shape[2:] or k.dtype != q.dtype):
        raise ValueError("k must be [B,Hkv,L,d] of q's type")
    if pos.dtype != torch.int32 or tuple(pos.shape) not in ((B, L), (L,)) or (L > 1 and pos.stride(-1) != 1):
        raise ValueError("pos must be int32 [B,L] or [L], its last dimension contiguous")
    if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError("freq must be contiguous fp64 [rot / 2]")
    if q_out is None:
        q_out = torch.empty_like(q)
    if k is not None and k_out is None:
        k_out = torch.empty_like(k)
    for t, like in ((q, q), (k, k), (q_out, q), (k_out, k)):
        if t is not None and (t.shape != like.shape or t.dtype != q.dtype or t.stride(3) != 1):
            raise ValueError("q_out and k_out must match q and k in shape and type, head dimensions be contiguous")
    s3 = lambda t: (0, 0, 0) if t is None else t.stride()[:3]  # noqa: E731
    desc = RopeDesc(B, L, Hq, 0 if k is None else k.shape[1], d, 2 * freq.shape[0], int(bool(interleaved)), dt,
                    float(attention_factor), pos.stride(0) if pos.dim() == 2 else 0, *s3(q), *s3(q_out), *s3(k),
                    *s3(k_out))
    _check(lib().cover_rope(_ptr(q), _ptr(k), _ptr(pos), _ptr(freq), _ptr(q_out), _ptr(k_out), ctypes.byref(desc),
                            _stream(stream)), "cover_rope")
    return q_out, k_out


def _check_cache(B, H, d, k_cache, v_cache, k_scale, v_scale) -> int:
    """Checks the cache's four tensors; returns the positions they hold."""
    for t in (k_cache, v_cache):
        if t.dim() != 4 or t.dtype != torch.float8_e4m3fn or t.shape != k_cache.shape or \
                t.stride() != k_cache.stride() or t.stride(3) != 1 or (t.shape[0], t.shape[1], t.shape[3]) != (B, H, d):
            raise ValueError("k_cache and v_cache must be float8_e4m3fn [B,Hkv,L,d] of equal strides, head dimension "
                             "contiguous")
    L = k_cache.shape[2]
    for t in (k_scale, v_scale):
        if t.shape != (B, H, L) or t.dtype != torch.float32 or t.stride() != k_scale.stride() or \
                (L > 1 and t.stride(2) != 1):
            raise ValueError("k_scale and v_scale must be fp32 [B,Hkv,L] of equal strides, positions contiguous")
    return L


def _cache_rows(pos, B: int, N: int):
    """(pos or None, first) of a call on N rows: an int is the position of row 0."""
    if isinstance(pos, int):
        return None, _int32(pos, "pos")
    _on_gpu(pos=pos)
    if pos.dtype != torch.int32 or pos.shape != (B, N) or not pos.is_contiguous():
        raise ValueError("pos must be an int or contiguous int32 [B,N]")
    return pos, 0


def cover_cache_store(k, v, pos, k_cache, v_cache, k_scale, v_scale, stream=None):
    """Write k, v [B,Hkv,N,d] (bf16 or fp32, head dimension contiguous) into the 8-bit cache: k_cache, v_cache
    float8_e4m3fn [B,Hkv,L,d], k_scale, v_scale fp32 [B,Hkv,L].  pos: int32 [B,N], the rows' positions (distinct;
    those outside [0, L) are skipped), or an int, the position of row 0.  Returns the four cache tensors."""
    done = (_host or host()).cache_store(k, v, pos, k_cache, v_cache, k_scale, v_scale, *_place(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_cache_store")
    _on_gpu(k=k, v=v, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale)
    dt = _dtype(k, "k")
    if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or k.stride(3) != 1 or v.stride(3) != 1:
        raise ValueError("k and v must be [B,Hkv,N,d] of one type, head dimension contiguous")
    B, H, N, d = k.shape
    L = _check_cache(B, H, d, k_cache, v_cache, k_scale, v_scale)
    pos, first = _cache_rows(pos, B, N)
    desc = CacheDesc(B, H, N, L, d, first, dt, *k.stride()[:3], *v.stride()[:3], *k_cache.stride()[:3],
                     *k_scale.stride()[:2])
    _check(lib().cover_cache_store(_ptr(k), _ptr(v), _ptr(pos), _ptr(k_cache), _ptr(v_cache), _ptr(k_scale),
                                   _ptr(v_scale), ctypes.byref(desc), _stream(stream)), "cover_cache_store")
    return k_cache, v_cache, k_scale, v_scale


def cover_cache_load(k_cache, v_cache, k_scale, v_scale, pos, n=None, k=None, v=None, dtype=torch.bfloat16,
                     stream=None):
    """Read rows of the 8-bit cache back.  pos: int32 [B,N] (rows whose position is outside [0, L) are zeros), or
    an int, the position of the first of n rows.  Returns (k, v) [B,Hkv,N,d] of `dtype` (bf16 or fp32), or the
    caller's tensors."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_cache_load, k_cache, v_cache, k_scale, v_scale, pos, n, k, v, dtype)
    done = (_host or host()).cache_load(k_cache, v_cache, k_scale, v_scale, pos, n, k, v, dtype is torch.bfloat16,
                                        *_place(stream)) if dtype in (torch.bfloat16, torch.float32) else None
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_cache_load")
    _on_gpu(k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, k=k, v=v)
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [B,Hkv,L,d]")
    B, H, _, d = k_cache.shape
    L = _check_cache(B, H, d, k_cache, v_cache, k_scale, v_scale)
    N = pos.shape[-1] if isinstance(pos, torch.Tensor) and pos.dim() == 2 else n
    if N is None or N < 0 or (n is not None and n != N):
        raise ValueError("n rows are needed where pos is an int; with a list of positions n is its width")
    pos, first = _cache_rows(pos, B, N)
    if k is None:
        k = torch.empty((B, H, N, d), device=k_cache.device, dtype=dtype)
    if v is None:
        v = torch.empty((B, H, N, d), device=k_cache.device, dtype=dtype)
    dt = _dtype(k, "k")
    for t in (k, v):
        if t.shape != (B, H, N, d) or t.dtype != dtype or t.stride(3) != 1:
            raise ValueError("k and v must be [B,Hkv,N,d] of `dtype`, head dimension contiguous")
    desc = CacheDesc(B, H, N, L, d, first, dt, *k.stride()[:3], *v.stride()[:3], *k_cache.stride()[:3],
                     *k_scale.stride()[:2])
    _check(lib().cover_cache_load(_ptr(k), _ptr(v), _ptr(pos), _ptr(k_cache), _ptr(v_cache), _ptr(k_scale),
                                  _ptr(v_scale), ctypes.byref(desc), _stream(stream)), "cover_cache_load")
    return k, v


def attn_cached_splits(B: int, Hq: int, Hkv: int, L: int, Lq: int) -> int:
    """The n_split that suits a cover_attn_cached call of these sizes."""
    return int(lib().cover_attn_cached_splits(int(B), int(Hq), int(Hkv), int(L), int(Lq)))


def attn_cached_plan(B: int, Hq: int, Hkv: int, L: int, Lq: int, d: int, n_split=None):
    """(key ranges, query rows per workgroup) of a cover_attn_cached call of these sizes (n_split None: the one that
    suits it)."""
    if n_split is None:
        n_split = attn_cached_splits(B, Hq, Hkv, L, Lq)
    ranges, rows = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().cover_attn_cached_plan(int(B), int(Hq), int(Hkv), int(L), int(Lq), int(d), _int32(n_split, "n_split"),
                                        ctypes.byref(ranges), ctypes.byref(rows)), "cover_attn_cached_plan")
    return ranges.value, rows.value


def attn_cached_workspace(B: int, Hq: int, Lq: int, d: int, n_split: int) -> int:
    """Floats of workspace cover_attn_cached needs (COVER_ATTN_CACHED_WORKSPACE)."""
    return B * Hq * n_split * Lq * (d + 4) if n_split > 1 else 0


def cover_attn_cached(q, k_live, v_live, k_cache, v_cache, k_scale, v_scale, q_off, seed_idx=None, n_seed=None,
                      kv_len=None, out=None, lse=None, scale: float = 0.0, n_split=None, workspace=None,
                      want_lse: bool = True, stream=None):
    """COVER attention of a block of Lq query rows against the 8-bit cache and the block's own rows.  q
    [B,Hq,Lq,d], k_live, v_live [B,Hkv,Lq,d] bf16 (head dimension contiguous); the cache as for
    cover_cache_store; q_off: the block's first position, an int or int32 [B]; kv_len int32 [B]: keys of each
    batch row (None: all L); seeds as for cover_attn_fwd (absolute positions).  Rows at or past kv_len are not
    written.  Returns (out [B,Hq,Lq,d], lse [B,Hq,Lq])."""
    if stream is not None and (other := _other(stream)) is not None:
        return _run_on(other, cover_attn_cached, q, k_live, v_live, k_cache, v_cache, k_scale, v_scale, q_off,
                       seed_idx, n_seed, kv_len, out, lse, scale, n_split, workspace, want_lse)
    done = (_host or host()).attn_cached(q, k_live, v_live, k_cache, v_cache, k_scale, v_scale, q_off, seed_idx, n_seed,
                                         kv_len, out, lse, scale, n_split, workspace, want_lse,
                                         *_place(stream))
    if done.__class__ is tuple:
        return done
    if done is not None:
        raise CoverError(done, "cover_attn_cached")
    off = q_off if isinstance(q_off, torch.Tensor) else None
    _on_gpu(q=q, k_live=k_live, v_live=v_live, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale,
            q_off=off, seed_idx=seed_idx, n_seed=n_seed, kv_len=kv_len, out=out, lse=lse, workspace=workspace)
    if q.dtype != torch.bfloat16:
        raise TypeError(f"q must be bf16, not {q.dtype}")
    if q.dim() != 4 or k_live.dim() != 4:
        raise ValueError("q must be [B,Hq,Lq,d], k_live [B,Hkv,Lq,d]")
    B, Hq, Lq, d = q.shape
    Hkv = k_live.shape[1]
    for t in (k_live, v_live):
        if t.shape != (B, Hkv, Lq, d) or t.dtype != q.dtype or t.stride(3) != 1:
            raise ValueError("k_live and v_live must be bf16 [B,Hkv,Lq,d], head dimension contiguous")
    if q.stride(3) != 1:
        raise ValueError("head dimension must be contiguous")
    L = _check_cache(B, Hkv, d, k_cache, v_cache, k_scale, v_scale)
    for name, t in (("q_off", off), ("kv_len", kv_len)):
        if t is not None and (t.shape != (B,) or t.dtype != torch.int32 or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous int32 [B]")
    max_seeds = 0
    if seed_idx is not None:
        if seed_idx.dim() != 2 or seed_idx.shape[0] != B or seed_idx.dtype != torch.int32 or \
                not seed_idx.is_contiguous() or n_seed is None or n_seed.shape != (B,) or n_seed.dtype != torch.int32 \
                or not n_seed.is_contiguous():
            raise ValueError("seed_idx must be contiguous int32 [B,max_seeds], n_seed int32 [B]")
        max_seeds = seed_idx.shape[1]
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.dtype != q.dtype or out.stride(3) != 1:
        raise ValueError("out must match q's shape and dtype, its head dimension be contiguous")
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, Lq), device=q.device, dtype=torch.float32)
    if lse is not None and (lse.shape != (B, Hq, Lq) or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous fp32 [B,Hq,Lq]")
    if n_split is None:
        n_split = attn_cached_splits(B, Hq, Hkv, L, Lq)
        if workspace is not None and B * Lq and n_split > 1:  # as many ranges as the caller's workspace holds
            n_split = max(1, min(n_split, workspace.numel() // (B * Hq * Lq * (d + 4))))
    need = attn_cached_workspace(B, Hq, Lq, d, min(n_split, 256))
    if need == 0:
        workspace = None
    elif workspace is None:
        workspace = torch.empty(need, device=q.device, dtype=torch.float32)
    if workspace is not None and (workspace.dtype != torch.float32 or workspace.numel() < need
                                  or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous fp32 with at least {need} elements")
    desc = CachedDesc(B, Hq, Hkv, L, Lq, d, max_seeds, 0 if off is not None else _int32(q_off, "q_off"),
                      _int32(n_split, "n_split"), float(scale),
                      *q.stride()[:3], *out.stride()[:3], *k_live.stride()[:3], *v_live.stride()[:3],
                      *k_cache.stride()[:3], *k_scale.stride()[:2])
    _check(lib().cover_attn_cached(_ptr(q), _ptr(k_live), _ptr(v_live), _ptr(k_cache), _ptr(v_cache), _ptr(k_scale),
                                   _ptr(v_scale), _ptr(off), _ptr(kv_len), _ptr(seed_idx), _ptr(n_seed), _ptr(out),
                                   _ptr(lse), _ptr(workspace), ctypes.byref(desc), _stream(stream)),
           "cover_attn_cached")
    return out, lse


def attn_flops(B: int, Hq: int, L: int, d: int) -> int:
    """Algorithmic flops of one call: QK^T plus PV, 2 flops per multiply-add, non-causal."""
    return 4 * B * Hq * L * L * d


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)


class PreparedAttn:
    """A cover_attn_fwd call with its arguments marshalled once, for tight loops: calling it
    re-launches the kernel on the same tensors (their contents may change between calls)."""

    def __init__(self, q, k_live, v_live, k_cache, v_cache, seed_idx=None, n_seed=None, out=None,
                 lse=None, scale: float = 0.0, stream=None):
        self.out, self.lse = cover_attn_fwd(q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed,
                                            out=out, lse=lse, scale=scale, stream=stream)
        self._keep = (q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed, self.out, self.lse)
        max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
        self._desc = attn_desc(q, k_live, max_seeds, scale)
        self._args = (_ptr(q), _ptr(k_live), _ptr(v_live), _ptr(k_cache), _ptr(v_cache),
                      _ptr(seed_idx), _ptr(n_seed), _ptr(self.out), _ptr(self.lse),
                      ctypes.byref(self._desc), _stream(stream))
        self._fn = lib().cover_attn_fwd

    def __call__(self):
        st = self._fn(*self._args)
        if st != COVER_OK:
            raise CoverError(st, "cover_attn_fwd")


class PreparedRect:
    """A cover_attn_rect call with its arguments marshalled once (see PreparedAttn)."""

    def __init__(self, q, k_live, v_live, k_cache, v_cache, q_off: int, seed_idx=None,
                 n_seed=None, out=None, lse=None, scale: float = 0.0, n_split=None, workspace=None,
                 stream=None):
        B, Hq, Lq, d = q.shape
        L = k_live.shape[2]
        n_split, need = _rect_plan(B, Hq, Lq, L, n_split, workspace)
        if need and workspace is None:
            with torch.cuda.stream(None if stream is None else _other(stream)):
                workspace = torch.empty(need, device=q.device, dtype=torch.float32)
        self.out, self.lse = cover_attn_rect(q, k_live, v_live, k_cache, v_cache, q_off, seed_idx,
                                             n_seed, out=out, lse=lse, scale=scale, n_split=n_split,
                                             workspace=workspace, stream=stream)
        self.n_split = n_split
        ws = workspace if need else None
        self._keep = (q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed, self.out, self.lse, ws)
        max_seeds = 0 if seed_idx is None else seed_idx.shape[-1]
        ad = attn_desc(q, k_live, max_seeds, scale)
        ad.L = L
        self._desc = RectDesc(ad, q_off, Lq, n_split)
        self._args = (_ptr(q), _ptr(k_live), _ptr(v_live), _ptr(k_cache), _ptr(v_cache),
                      _ptr(seed_idx), _ptr(n_seed), _ptr(self.out), _ptr(self.lse), _ptr(ws),
                      ctypes.byref(self._desc), _stream(stream))
        self._fn = lib().cover_attn_rect

    def __call__(self):
        st = self._fn(*self._args)
        if st != COVER_OK:
            raise CoverError(st, "cover_attn_rect")


class PreparedSelect:
    """A cover_select_seeds call with its arguments marshalled once (see PreparedAttn)."""

    def __init__(self, logp, d_in, d_out, flags, max_seeds: int, pos_offset: int = 0,
                 seed_idx=None, n_seed=None, score=None, want_score: bool = True, stream=None):
        self.seed_idx, self.n_seed, self.score = cover_select_seeds(
            logp, d_in, d_out, flags, max_seeds, pos_offset, seed_idx=seed_idx, n_seed=n_seed,
            score=score, want_score=want_score, stream=stream)
        self._keep = (logp, d_in, d_out, flags, self.seed_idx, self.n_seed, self.score)
        self._desc = SelectDesc(logp.shape[0], logp.shape[1], max_seeds, pos_offset)
        self._args = (_ptr(logp), _ptr(d_in), _ptr(d_out), _ptr(flags), _ptr(self.seed_idx),
                      _ptr(self.n_seed), _ptr(self.score), ctypes.byref(self._desc),
                      _stream(stream))
        self._fn = lib().cover_select_seeds

    def __call__(self):
        st = self._fn(*self._args)
        if st != COVER_OK:
            raise CoverError(st, "cover_select_seeds")
