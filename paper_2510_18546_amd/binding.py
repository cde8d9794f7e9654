"""ctypes binding over the C ABI of libefficientnav.so (include/efficientnav.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels. torch supplies device memory and the stream; there is no fallback
of any kind: a missing library raises.
"""
from __future__ import annotations

import array
import ctypes as C
import os
import sys
import weakref
from typing import Optional, Sequence, Tuple

import numpy as np

from . import build as _build

EN_F32, EN_BF16, EN_I8 = 0, 1, 2
STATUS = {0: "EN_OK", 1: "EN_ERR_INVALID_ARG", 2: "EN_ERR_OUT_OF_RANGE", 3: "EN_ERR_DUPLICATE",
          4: "EN_ERR_CAPACITY", 5: "EN_ERR_UNSUPPORTED", 6: "EN_ERR_DEVICE"}

EXPORTS = [
    "kv_pool_create", "kv_pool_set_scales", "kv_pool_set_len", "kv_pool_append", "kv_pool_destroy", "segment_select",
    "segment_select_scored", "en_plan_get_info", "en_plan_query", "en_plan_set_splits",
    "en_plan_values_from_pool",
    "en_plan_destroy", "en_context_bytes", "gather_rope", "gather_rope_queries", "en_workspace_bytes",
    "segmented_prefill_attention", "segmented_prefill_attention_prepared", "segment_attention_mass",
    "segment_cluster_assign",
    "segment_cluster_assign_rows",
    "en_decode_workspace_bytes", "segmented_decode_step", "segmented_decode_step_static", "en_timing_enable",
    "en_timing_collect", "en_last_error", "en_ceiling_mfma_bf16", "en_ceiling_read_stream",
    "kv_tier_slot_bytes", "kv_tier_create", "kv_tier_pool", "kv_tier_put", "kv_tier_append",
    "kv_tier_select_scored",
    "kv_tier_fetch", "kv_tier_fence", "kv_tier_prefetch", "kv_tier_get_stats", "kv_tier_residency",
    "kv_tier_destroy",
    "en_tree_workspace_bytes", "segmented_tree_attention", "token_rules_apply", "en_tree_accept_workspace_bytes",
    "token_tree_accept", "segmented_tree_commit",
]
TREE_MAX_NODES = 64


class EnError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"{STATUS.get(code, code)}: {text}")
        self.code = code


class PoolDesc(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("capacity", C.c_int32), ("n_kv_heads", C.c_int32),
                ("n_q_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("max_ctx", C.c_int32), ("reserved", C.c_int32), ("rope_base", C.c_double)]


class PlanInfo(C.Structure):
    _fields_ = [("n_agents", C.c_int32), ("n_new", C.c_int32), ("max_segments", C.c_int32),
                ("ctx_stride", C.c_int32), ("max_ctx_len", C.c_int32), ("n_splits", C.c_int32),
                ("total_pairs", C.c_int64), ("total_cached", C.c_int64)]


class TierStats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("fetches", "requested", "hits", "prefetched", "misses", "loads",
                                         "bytes_loaded", "evictions")]


class _TokenRules(C.Structure):
    _fields_ = [("penalties_dev", C.c_void_p), ("history_dev", C.c_void_p), ("history_len_dev", C.c_void_p),
                ("bias_dev", C.c_void_p), ("mask_dev", C.c_void_p), ("bias_agent_stride", C.c_int64),
                ("mask_agent_stride", C.c_int64), ("mask_node_stride", C.c_int64), ("history_stride", C.c_int32),
                ("reserved", C.c_int32)]


_lib = None


def load(path: Optional[str] = None) -> C.CDLL:
    """Load the built library; build it first only if nothing has been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or _build.LIB_PATH
    if not os.path.exists(path):
        _build.build()
    lib = C.CDLL(path)
    # arrays of the host are passed by address (see _ip): a typed pointer object costs a microsecond to make
    vp = i32p = f32p = C.c_void_p
    lib.kv_pool_create.argtypes = [C.POINTER(PoolDesc), vp, vp, i32p, C.POINTER(vp)]
    lib.kv_pool_set_scales.argtypes = [vp, vp, vp]
    lib.kv_pool_set_len.argtypes = [vp, C.c_int32, C.c_int32]
    lib.kv_pool_append.argtypes = [vp, C.c_int32, vp, vp, C.c_int32, vp]
    lib.kv_pool_destroy.argtypes = [vp]
    lib.segment_select.argtypes = [vp, C.c_int32, i32p, i32p, C.c_int32, C.POINTER(vp)]
    lib.segment_select_scored.argtypes = [vp, f32p, C.c_float, C.c_int64, C.c_int32,
                                          i32p, i32p, C.POINTER(vp)]
    lib.en_plan_get_info.argtypes = [vp, C.POINTER(PlanInfo)]
    lib.en_plan_query.argtypes = [vp, C.c_int32, i32p, i32p]
    lib.en_plan_set_splits.argtypes = [vp, C.c_int32]
    lib.en_plan_values_from_pool.argtypes = [vp, C.c_int32]
    lib.en_plan_destroy.argtypes = [vp]
    lib.en_context_bytes.argtypes = [vp, vp]
    lib.en_context_bytes.restype = C.c_size_t
    lib.en_workspace_bytes.argtypes = [vp, vp]
    lib.en_workspace_bytes.restype = C.c_size_t
    lib.gather_rope.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.segmented_prefill_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.gather_rope_queries.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.segmented_prefill_attention_prepared.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.segment_attention_mass.argtypes = [vp, vp, vp, C.c_int32, vp, vp]
    lib.segment_cluster_assign.argtypes = [vp, vp, vp, C.c_int32, i32p, C.c_int32, C.c_int32, C.c_float,
                                           C.c_float, vp, vp, vp]
    lib.segment_cluster_assign_rows.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, C.c_int32, i32p, C.c_int32,
                                                C.c_int32, C.c_float, C.c_float, vp, vp, vp]
    lib.en_decode_workspace_bytes.argtypes = [vp, vp, C.c_int32]
    lib.en_decode_workspace_bytes.restype = C.c_size_t
    lib.segmented_decode_step.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp,
                                          C.c_size_t, vp]
    lib.segmented_decode_step_static.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.en_timing_enable.argtypes = [vp, C.c_int32]
    lib.en_timing_collect.argtypes = [vp, f32p, C.c_int32, i32p]
    lib.en_last_error.restype = C.c_char_p
    lib.en_ceiling_mfma_bf16.argtypes = [vp, C.c_size_t, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_double), vp]
    lib.en_ceiling_read_stream.argtypes = [vp, C.c_size_t, vp, C.c_size_t, C.c_int32, vp]
    lib.kv_tier_slot_bytes.argtypes = [C.POINTER(PoolDesc)]
    lib.kv_tier_slot_bytes.restype = C.c_int64
    lib.kv_tier_create.argtypes = [C.POINTER(PoolDesc), C.c_int32, vp, vp, C.POINTER(vp)]
    lib.kv_tier_pool.argtypes = [vp]
    lib.kv_tier_pool.restype = vp
    lib.kv_tier_put.argtypes = [vp, C.c_int32, vp, vp, C.c_int32]
    lib.kv_tier_append.argtypes = [vp, C.c_int32, vp, vp, C.c_int32, vp]
    lib.kv_tier_select_scored.argtypes = [vp, f32p, C.c_float, C.c_int64, i32p, i32p]
    lib.kv_tier_fetch.argtypes = [vp, i32p, C.c_int32, i32p, vp]
    lib.kv_tier_fence.argtypes = [vp, vp]
    lib.kv_tier_prefetch.argtypes = [vp, i32p, C.c_int32, i32p]
    lib.kv_tier_get_stats.argtypes = [vp, C.POINTER(TierStats)]
    lib.kv_tier_residency.argtypes = [vp, i32p]
    lib.kv_tier_destroy.argtypes = [vp]
    lib.en_tree_workspace_bytes.argtypes = [vp, vp, C.c_int32]
    lib.en_tree_workspace_bytes.restype = C.c_size_t
    lib.segmented_tree_attention.argtypes = [vp, vp, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.token_rules_apply.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, C.c_int64, vp, C.c_int64, vp]
    lib.en_tree_accept_workspace_bytes.argtypes = [vp, C.c_int32, C.c_int32]
    lib.en_tree_accept_workspace_bytes.restype = C.c_size_t
    lib.token_tree_accept.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, C.c_int64, vp, vp, vp, vp, vp, vp,
                                      C.c_size_t, vp]
    lib.segmented_tree_commit.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp]
    for name in EXPORTS:
        if name not in ("en_context_bytes", "en_workspace_bytes", "en_decode_workspace_bytes", "en_last_error",
                        "kv_tier_slot_bytes", "kv_tier_pool", "en_tree_workspace_bytes", "en_tree_accept_workspace_bytes"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(rc: int):
    if rc != 0:
        raise EnError(rc, load().en_last_error().decode())


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _ip(a: np.ndarray) -> int:
    """Address of a contiguous array, which the caller keeps alive over the call."""
    return a.ctypes.data


_current_stream = None


def _find_current_stream():
    """The function that returns the handle of torch's current stream. torch.cuda.current_stream() makes a
    stream object on the way, 2.9 us of every call into the library; the handle alone takes 0.1 us."""
    import torch
    torch.cuda.current_stream()          # sets the device up if nothing has yet
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> int:
    global _current_stream
    if stream is not None:
        return int(stream)
    if _current_stream is None:
        _current_stream = _find_current_stream()
    return _current_stream()


class Pool:
    """Handle of a KV pool. Keeps the K/V tensors alive."""

    def __init__(self, handle, k, v, desc: PoolDesc, owned: bool = True):
        self.handle, self.k, self.v, self.desc = handle, k, v, desc
        self._owned = owned                  # False: the handle belongs to a tier, which destroys it
        self._plans = weakref.WeakSet()      # a pool must outlive its plans: it closes them first

    def close(self):
        if self.handle:
            for p in list(self._plans):
                p.close()
            if self._owned:
                load().kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone: the process frees everything
        if sys is None or sys.is_finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


class Plan:
    def __init__(self, handle, pool: Pool, n_agents: int = 1):
        self.handle, self.pool, self.n_agents, self._context_bytes = handle, pool, n_agents, None
        pool._plans.add(self)

    @property
    def context_bytes(self) -> int:
        """Bytes of a context buffer; fixed when the plan is made."""
        if self._context_bytes is None:
            self._context_bytes = context_bytes(self.pool, self)
        return self._context_bytes

    @property
    def info(self) -> PlanInfo:
        inf = PlanInfo()
        _check(load().en_plan_get_info(self.handle, C.byref(inf)))
        return inf

    def offsets(self, agent: int) -> np.ndarray:
        n = C.c_int32()
        _check(load().en_plan_query(self.handle, agent, None, C.byref(n)))
        off = np.zeros(n.value + 1, dtype=np.int32)
        _check(load().en_plan_query(self.handle, agent, _ip(off), None))
        return off

    def set_splits(self, n: int):
        _check(load().en_plan_set_splits(self.handle, int(n)))

    def values_from_pool(self, on: bool):
        _check(load().en_plan_values_from_pool(self.handle, 1 if on else 0))

    def close(self):
        if self.handle:
            load().en_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone: the process frees everything
        if sys is None or sys.is_finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


def kv_pool_create(k_pool, v_pool, lens, n_q_heads: int, rope_base: float, max_ctx: int,
                   dtype: Optional[int] = None, k_ptr: Optional[int] = None,
                   v_ptr: Optional[int] = None, shape: Optional[Sequence[int]] = None) -> Pool:
    """k_pool, v_pool: torch tensors [G,Hkv,C,D] on the GPU (float32 or bfloat16).
    For host-only planner use, pass k_pool=v_pool=None with ``shape``, ``dtype``
    and opaque non-null ``k_ptr``/``v_ptr`` values that are never dereferenced."""
    if k_pool is not None:
        import torch
        assert k_pool.is_contiguous() and v_pool.is_contiguous() and k_pool.shape == v_pool.shape
        shape = tuple(k_pool.shape)
        dtype = EN_BF16 if k_pool.dtype == torch.bfloat16 else EN_I8 if k_pool.dtype == torch.int8 else EN_F32
        k_ptr, v_ptr = k_pool.data_ptr(), v_pool.data_ptr()
    G, Hkv, Cap, D = shape
    desc = PoolDesc(G, Cap, Hkv, n_q_heads, D, dtype, max_ctx, 0, rope_base)
    lens = _i32(lens)
    h = C.c_void_p()
    _check(load().kv_pool_create(C.byref(desc), C.c_void_p(k_ptr), C.c_void_p(v_ptr), _ip(lens),
                                 C.byref(h)))
    return Pool(h, k_pool, v_pool, desc)


def kv_pool_set_scales(pool: Pool, k_scale, v_scale):
    """k_scale, v_scale: float32 tensors [G, Hkv, C] on the GPU (kept alive by the pool), or integers as
    opaque pointers for host-only tests."""
    if hasattr(k_scale, "data_ptr"):
        assert k_scale.is_contiguous() and v_scale.is_contiguous()
        pool.k_scale, pool.v_scale = k_scale, v_scale
        kp, vp_ = k_scale.data_ptr(), v_scale.data_ptr()
    else:
        kp, vp_ = k_scale, v_scale
    _check(load().kv_pool_set_scales(pool.handle, C.c_void_p(kp), C.c_void_p(vp_)))


def kv_pool_set_len(pool: Pool, group: int, length: int):
    _check(load().kv_pool_set_len(pool.handle, group, length))


def kv_pool_append(pool: Pool, group: int, k_rows, v_rows, n_tokens: Optional[int] = None, stream=None):
    """k_rows, v_rows: torch tensors [n, Hkv, D] (contiguous, pool dtype, keys unrotated) on the GPU;
    for host-only tests pass integers as opaque pointers together with n_tokens."""
    if hasattr(k_rows, "data_ptr"):
        assert k_rows.is_contiguous() and v_rows.is_contiguous() and k_rows.shape == v_rows.shape
        n_tokens = int(k_rows.shape[0]) if n_tokens is None else int(n_tokens)
        kp, vp_ = k_rows.data_ptr(), v_rows.data_ptr()
        stream = _stream(stream)
    else:
        kp, vp_ = k_rows, v_rows
        stream = C.c_void_p(0)
    _check(load().kv_pool_append(pool.handle, int(group), C.c_void_p(kp), C.c_void_p(vp_), int(n_tokens), stream))


def segment_select(pool: Pool, sel, sel_ptr, n_new: int) -> Plan:
    sel, sel_ptr = _i32(sel), _i32(sel_ptr)
    h = C.c_void_p()
    _check(load().segment_select(pool.handle, len(sel_ptr) - 1, _ip(sel), _ip(sel_ptr), n_new,
                                 C.byref(h)))
    return Plan(h, pool, len(sel_ptr) - 1)


def segment_select_scored(pool: Pool, p, threshold: float, budget_tokens: int, n_new: int,
                          want_plan: bool = True) -> Tuple[np.ndarray, Optional[Plan]]:
    p = np.ascontiguousarray(p, dtype=np.float32)
    out = np.zeros(pool.desc.n_groups, dtype=np.int32)
    n = C.c_int32()
    h = C.c_void_p()
    _check(load().segment_select_scored(pool.handle, _ip(p),
                                        C.c_float(threshold), C.c_int64(int(budget_tokens)), n_new,
                                        _ip(out), C.byref(n), C.byref(h) if want_plan else None))
    return out[:n.value].copy(), (Plan(h, pool) if want_plan else None)


def context_bytes(pool: Pool, plan: Plan) -> int:
    return int(load().en_context_bytes(pool.handle, plan.handle))


def workspace_bytes(pool: Pool, plan: Plan) -> int:
    return int(load().en_workspace_bytes(pool.handle, plan.handle))


def alloc_context(pool: Pool, plan: Plan):
    """Uninitialised context buffers (kc, vt) as flat byte tensors."""
    import torch
    n = context_bytes(pool, plan)
    dev = pool.k.device
    return (torch.empty(n, dtype=torch.uint8, device=dev), torch.empty(n, dtype=torch.uint8, device=dev))


def alloc_workspace(pool: Pool, plan: Plan):
    import torch
    return torch.empty(max(workspace_bytes(pool, plan), 256), dtype=torch.uint8, device=pool.k.device)


def gather_rope(pool: Pool, plan: Plan, k_new, v_new, kc, vt, stream=None):
    _check(load().gather_rope(pool.handle, plan.handle, k_new.data_ptr(), v_new.data_ptr(),
                              kc.data_ptr(), vt.data_ptr(), _stream(stream)))
    return kc, vt


def segmented_prefill_attention(pool: Pool, plan: Plan, q, kc, vt, out, ws=None, stream=None):
    _check(load().segmented_prefill_attention(
        pool.handle, plan.handle, q.data_ptr(), kc.data_ptr(), vt.data_ptr(), out.data_ptr(),
        ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0,
        _stream(stream)))
    return out


def gather_rope_queries(pool: Pool, plan: Plan, k_new, v_new, q, kc, vt, q_prep, stream=None):
    _check(load().gather_rope_queries(pool.handle, plan.handle, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                                      kc.data_ptr(), vt.data_ptr(), q_prep.data_ptr(), _stream(stream)))
    return kc, vt, q_prep


def segmented_prefill_attention_prepared(pool: Pool, plan: Plan, q_prep, kc, vt, out, ws=None, mass_red_out=None,
                                         stream=None):
    _check(load().segmented_prefill_attention_prepared(
        pool.handle, plan.handle, q_prep.data_ptr(), kc.data_ptr(), vt.data_ptr(), out.data_ptr(),
        mass_red_out.data_ptr() if mass_red_out is not None else None,
        ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0,
        _stream(stream)))
    return out


def segment_attention_mass(pool: Pool, plan: Plan, ws, reduce: int, mass_out, stream=None):
    _check(load().segment_attention_mass(pool.handle, plan.handle, ws.data_ptr(), int(reduce),
                                         mass_out.data_ptr(), _stream(stream)))
    return mass_out


def segment_cluster_assign(pool: Pool, plan: Plan, ws, spans, score, assign=None, per_key: bool = False,
                           accumulate: bool = False, scale: float = 1.0, threshold: float = 0.0, stream=None):
    """spans: host int32 [n_obj+1]; score: float32 tensor [B, n_obj, Smax+1]; assign: int32 tensor
    [B, n_obj] or None. For host-only tests ws/score may be integers (opaque pointers)."""
    spans = _i32(spans)
    ptr = lambda t: C.c_void_p(t.data_ptr() if hasattr(t, "data_ptr") else t)
    _check(load().segment_cluster_assign(
        pool.handle, plan.handle, ptr(ws), len(spans) - 1, _ip(spans), int(per_key), int(accumulate),
        C.c_float(scale), C.c_float(threshold), ptr(score), ptr(assign) if assign is not None else None,
        _stream(stream) if hasattr(ws, "data_ptr") else C.c_void_p(0)))
    return score, assign


def segment_cluster_assign_rows(pool: Pool, plan: Plan, q_first: int, n_rows: int, ws, spans, score, assign=None,
                                per_key: bool = False, accumulate: bool = False, scale: float = 1.0,
                                threshold: float = 0.0, stream=None):
    """As segment_cluster_assign, from the scratch that segmented_decode_step(q_first, n_rows) left."""
    spans = _i32(spans)
    ptr = lambda t: C.c_void_p(t.data_ptr() if hasattr(t, "data_ptr") else t)
    _check(load().segment_cluster_assign_rows(
        pool.handle, plan.handle, int(q_first), int(n_rows), ptr(ws), len(spans) - 1, _ip(spans), int(per_key),
        int(accumulate), C.c_float(scale), C.c_float(threshold), ptr(score),
        ptr(assign) if assign is not None else None, _stream(stream) if hasattr(ws, "data_ptr") else C.c_void_p(0)))
    return score, assign


def decode_workspace_bytes(pool: Pool, plan: Plan, n_rows: int) -> int:
    return int(load().en_decode_workspace_bytes(pool.handle, plan.handle, int(n_rows)))


def segmented_decode_step(pool: Pool, plan: Plan, q_first: int, q, k_rows, v_rows, kc, vt, out, ws,
                          mass_out=None, stream=None):
    """q [B,n,Hq,D], k_rows/v_rows [B,n,Hkv,D], out [B,n,Hq,D]: contiguous torch tensors of the step."""
    n = int(q.shape[1])
    _check(load().segmented_decode_step(
        pool.handle, plan.handle, int(q_first), n, q.data_ptr(), k_rows.data_ptr(), v_rows.data_ptr(),
        kc.data_ptr(), vt.data_ptr(), out.data_ptr(), mass_out.data_ptr() if mass_out is not None else None,
        ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0,
        _stream(stream)))
    return out


def segmented_decode_step_static(pool: Pool, plan: Plan, q_first: int, q, k_rows, v_rows, kc, vt, out,
                                 mass_out=None, stream=None):
    """segmented_decode_step on the library's static device scratch: the call allocates nothing."""
    n = int(q.shape[1])
    _check(load().segmented_decode_step_static(
        pool.handle, plan.handle, int(q_first), n, q.data_ptr(), k_rows.data_ptr(), v_rows.data_ptr(),
        kc.data_ptr(), vt.data_ptr(), out.data_ptr(), mass_out.data_ptr() if mass_out is not None else None,
        _stream(stream)))
    return out


def _unfit(name: str, t, want: str) -> ValueError:
    return ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}; "
                      f"{want} on the current device is wanted")


_get_device = None


def _device() -> int:
    """Launches go to the current device: a tensor elsewhere would be read there by address."""
    global _get_device
    if _get_device is None:
        import torch
        if not torch.cuda.is_available():
            raise ValueError("drafted tokens are tensors on a GPU, and there is none")
        torch.cuda.current_device()          # sets the device up if nothing has yet
        _get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _get_device()


def _at(name: str, t, shape, dtype, dev: int) -> int:
    """Address of a contiguous tensor of that shape and type on the device."""
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != dev:
        raise _unfit(name, t, f"a contiguous {tuple(shape)} of {dtype}")
    return t.data_ptr()


def _buffer(name: str, t, nbytes: int, dev: int) -> int:
    """Address of a buffer of at least `nbytes` on the device."""
    if t.nbytes < nbytes or not t.is_contiguous() or t.get_device() != dev:
        raise _unfit(name, t, f"a contiguous buffer of {nbytes} bytes")
    return t.data_ptr()


def _other_numbers(x, dtype) -> bool:
    """Numbers of another type than `dtype`, not bare bytes."""
    return x is not dtype and (x.is_floating_point or x.is_complex)


def _context(name: str, t, nbytes: int, dtype, dev: int) -> int:
    """Address of a context buffer, numbers of that type or bare bytes (as alloc_context makes them)."""
    if _other_numbers(t.dtype, dtype):
        raise _unfit(name, t, f"a context of {dtype}")
    return _buffer(name, t, nbytes, dev)


def _layers_rows(name: str, ts, shape: tuple, dtype, dev: int) -> array.array:
    """Addresses of the layers' rows, contiguous tensors of that shape and type on the device."""
    t_ = _torch().Tensor
    if not (list(map(t_.shape.__get__, ts)).count(shape) == len(ts) and set(map(t_.dtype.__get__, ts)) == {dtype} and
            all(map(t_.is_contiguous, ts)) and set(map(t_.get_device, ts)) == {dev}):
        raise ValueError(f"{name}: a contiguous {shape} of {dtype} on the current device is wanted for every layer")
    return array.array("Q", list(map(t_.data_ptr, ts)))


def _layers_contexts(name: str, ts, nbytes: int, dtype, dev: int) -> array.array:
    """Addresses of the layers' contexts (see _context)."""
    t_ = _torch().Tensor
    types = set(map(t_.dtype.__get__, ts))
    if (min(map(t_.nbytes.__get__, ts)) < nbytes or types != {dtype} and any(_other_numbers(x, dtype) for x in types) or
            not all(map(t_.is_contiguous, ts)) or set(map(t_.get_device, ts)) != {dev}):
        raise ValueError(f"{name}: a contiguous context of at least {nbytes} bytes, {dtype} or bytes, on the current device is wanted "
                         "for every layer")
    return array.array("Q", list(map(t_.data_ptr, ts)))


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _row_type(desc: PoolDesc):
    return _torch().float32 if desc.dtype == EN_F32 else _torch().bfloat16


def tree_workspace_bytes(pool: Pool, plan: Plan, n_nodes: int) -> int:
    return int(load().en_tree_workspace_bytes(pool.handle, plan.handle, int(n_nodes)))


def segmented_tree_attention(pool: Pool, plan: Plan, done, parent, q, k_rows, v_rows, kc, vt, out, ws=None, stream=None):
    """done int32 [B], parent int32 [B, n]; q, out [B, n, Hq, D], k_rows/v_rows [B, n, Hkv, D] in the contexts' type; kc, vt
    context buffers, of that type or of bytes."""
    lib, i32, t, dev, d = load(), _torch().int32, _row_type(pool.desc), _device(), pool.desc
    b, n = parent.shape
    if b != plan.n_agents:
        raise ValueError(f"parent: {b} agents, the plan has {plan.n_agents}")
    rows, mine, ctx = (b, n, d.n_q_heads, d.head_dim), (b, n, d.n_kv_heads, d.head_dim), plan.context_bytes
    _check(lib.segmented_tree_attention(
        pool.handle, plan.handle, n, _at("done", done, (b,), i32, dev), _at("parent", parent, (b, n), i32, dev),
        _at("q", q, rows, t, dev), _at("k_rows", k_rows, mine, t, dev), _at("v_rows", v_rows, mine, t, dev),
        _context("kc", kc, ctx, t, dev), _context("vt", vt, ctx, t, dev), _at("out", out, rows, t, dev),
        _buffer("ws", ws, 0, dev) if ws is not None else None, ws.nbytes if ws is not None else 0, _stream(stream)))
    return out


class TokenRules:
    """Rules on logits; keeps their tensors alive. See token_rules."""

    def __init__(self, struct: _TokenRules, tensors: list):
        self.struct, self.tensors = struct, tensors
        self.address = C.addressof(struct)

    def check(self, n_agents: int, n_nodes: int, vocab: int, dev: int):
        """The rules fit logits [n_agents, n_nodes, vocab] on that device."""
        for name, x in self.tensors:
            if x.get_device() != dev or x.shape[0] != n_agents and not (name == "bias" and x.dim() == 1):
                raise _unfit(name, x, f"one for {n_agents} agents")
            if name == "bias" and x.shape[-1] < vocab:
                raise _unfit(name, x, f"one for {vocab} tokens")
            if name == "mask" and (x.shape[1] not in (1, n_nodes) or 32 * x.shape[2] < vocab):
                raise _unfit(name, x, f"one for {n_nodes} nodes and {vocab} tokens")


def token_rules(penalties=None, history=None, history_len=None, bias=None, mask=None) -> TokenRules:
    """penalties float32 [B, 3] (repetition, frequency, presence); history int32 [B, H] with history_len int32 [B]; bias
    float32 [vocab] or [B, vocab]; mask int32 [B, 1 or n, words], bit v % 32 of word v / 32. Each may be None."""
    import torch
    want = {"penalties": (penalties, torch.float32, (2,)), "history": (history, torch.int32, (2,)),
            "history_len": (history_len, torch.int32, (1,)), "bias": (bias, torch.float32, (1, 2)), "mask": (mask, torch.int32, (3,))}
    for name, (x, dtype, dims) in want.items():
        if x is not None and (x.dtype != dtype or x.dim() not in dims or not x.is_contiguous()):
            raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype}; a contiguous {dtype} of {dims} axes is wanted")
    if penalties is not None and penalties.shape[1] != 3:
        raise ValueError(f"penalties: {tuple(penalties.shape)}, not [B, 3]")
    if (history is None) != (history_len is None):
        raise ValueError("history and history_len go together")
    at = lambda x: None if x is None else x.data_ptr()
    s = _TokenRules(at(penalties), at(history), at(history_len), at(bias), at(mask),
                    bias.shape[1] if bias is not None and bias.dim() == 2 else 0,
                    mask.shape[1] * mask.shape[2] if mask is not None else 0,
                    mask.shape[2] if mask is not None and mask.shape[1] > 1 else 0,
                    history.shape[1] if history is not None else 0, 0)
    return TokenRules(s, [(name, x) for name, (x, _, _) in want.items() if x is not None])


def _logit_rows(name: str, t, dev: int):
    """Address, distance of the rows in elements and type of logits [B, n, vocab]."""
    if t.dtype is _torch().bfloat16:
        dtype = EN_BF16
    elif t.dtype is _torch().float32:
        dtype = EN_F32
    else:
        raise _unfit(name, t, "float32 or bfloat16")
    if t.dim() != 3 or t.get_device() != dev:
        raise _unfit(name, t, "[B, n, vocab]")
    b, n, vocab = t.shape
    of_agent, stride, of_token = t.stride()
    if n == 1:
        stride = of_agent if b > 1 else vocab
    if of_token != 1 and vocab > 1 or b > 1 and of_agent != n * stride:
        raise _unfit(name, t, "[B, n, vocab] with tokens side by side and all rows equally far apart")
    return t.data_ptr(), stride, dtype


def token_rules_apply(rules: TokenRules, logits, out, parent=None, tokens=None, stream=None):
    """logits, out: [B, n, vocab] float32 or bfloat16 (out may be logits); parent, tokens int32 [B, n] or both None."""
    lib, i32, dev = load(), _torch().int32, _device()
    at, stride, dtype = _logit_rows("logits", logits, dev)
    to, out_stride, _ = _logit_rows("out", out, dev)
    if out.shape != logits.shape or out.dtype is not logits.dtype:
        raise _unfit("out", out, f"{tuple(logits.shape)} of {logits.dtype}")
    b, n, vocab = logits.shape
    rules.check(b, n, vocab, dev)
    _check(lib.token_rules_apply(
        rules.address, b, n, vocab, dtype, None if parent is None else _at("parent", parent, (b, n), i32, dev),
        None if tokens is None else _at("tokens", tokens, (b, n), i32, dev), at, stride, to, out_stride, _stream(stream)))
    return out


def tree_accept_workspace_bytes(plan: Plan, n_nodes: int, vocab: int) -> int:
    return int(load().en_tree_accept_workspace_bytes(plan.handle, int(n_nodes), int(vocab)))


def token_tree_accept(plan: Plan, done, parent, tokens, logits, choice, path, n_accepted, next_token, done_out, ws=None,
                      rules: Optional[TokenRules] = None, stream=None):
    """done, n_accepted, next_token, done_out int32 [B]; parent, tokens, choice, path int32 [B, n]; logits [B, n, vocab]
    float32 or bfloat16, or None: choice holds the choices. choice may be None with logits, done_out may be done."""
    lib, i32, dev = load(), _torch().int32, _device()
    b, n = tree = parent.shape
    if b != plan.n_agents:
        raise ValueError(f"parent: {b} agents, the plan has {plan.n_agents}")
    at, stride, dtype, vocab, agents = None, 0, EN_F32, 0, (b,)
    if logits is not None:
        at, stride, dtype = _logit_rows("logits", logits, dev)
        vocab = logits.shape[2]
        if logits.shape[:2] != tree:
            raise _unfit("logits", logits, f"[{b}, {n}, vocab]")
        if rules is not None:
            rules.check(b, n, vocab, dev)
    _check(lib.token_tree_accept(
        plan.handle, rules.address if rules is not None else None, n, vocab, dtype, _at("done", done, agents, i32, dev),
        _at("parent", parent, tree, i32, dev), _at("tokens", tokens, tree, i32, dev), at, stride,
        None if choice is None else _at("choice", choice, tree, i32, dev), _at("path", path, tree, i32, dev),
        _at("n_accepted", n_accepted, agents, i32, dev), _at("next_token", next_token, agents, i32, dev),
        _at("done_out", done_out, agents, i32, dev), _buffer("ws", ws, 0, dev) if ws is not None else None,
        ws.nbytes if ws is not None else 0, _stream(stream)))
    return path, n_accepted, next_token


def segmented_tree_commit(pool: Pool, plan: Plan, done, n_accepted, path, k_rows, v_rows, kc, vt, stream=None):
    """done (after the acceptance), n_accepted int32 [B], path int32 [B, n]; k_rows, v_rows: a tensor [B, n, Hkv, D] per
    layer, kc, vt: a context buffer per layer, in the type of the rows or of bytes."""
    lib, i32, dev, d, t = load(), _torch().int32, _device(), pool.desc, _row_type(pool.desc)
    b, n = path.shape
    if b != plan.n_agents:
        raise ValueError(f"path: {b} agents, the plan has {plan.n_agents}")
    layers = len(k_rows)
    if not layers == len(v_rows) == len(kc) == len(vt):
        raise ValueError(f"{layers}, {len(v_rows)}, {len(kc)}, {len(vt)} layers")
    if layers == 0:
        return
    mine, ctx = (b, n, d.n_kv_heads, d.head_dim), plan.context_bytes
    ptrs = [_layers_rows("k_rows", k_rows, mine, t, dev), _layers_rows("v_rows", v_rows, mine, t, dev),
            _layers_contexts("kc", kc, ctx, t, dev), _layers_contexts("vt", vt, ctx, t, dev)]
    _check(lib.segmented_tree_commit(
        pool.handle, plan.handle, n, layers, _at("done", done, (b,), i32, dev), _at("n_accepted", n_accepted, (b,), i32, dev),
        _at("path", path, (b, n), i32, dev), *(p.buffer_info()[0] for p in ptrs), _stream(stream)))


class Tier:
    """Handle of a residency tier. ``pool`` is the pool over the device slots (None for a tier that only
    keeps the books)."""

    def __init__(self, handle, pool: Optional[Pool], n_groups_total: int, desc: PoolDesc):
        self.handle, self.pool, self.n_groups_total, self.desc = handle, pool, n_groups_total, desc

    @property
    def stats(self) -> TierStats:
        st = TierStats()
        _check(load().kv_tier_get_stats(self.handle, C.byref(st)))
        return st

    def residency(self) -> np.ndarray:
        out = np.zeros(self.n_groups_total, dtype=np.int32)
        _check(load().kv_tier_residency(self.handle, _ip(out)))
        return out

    def close(self):
        if self.handle:
            if self.pool is not None:
                self.pool.close()
            load().kv_tier_destroy(self.handle)
            self.handle = None

    def __del__(self):
        if sys is None or sys.is_finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


def kv_tier_slot_bytes(shape: Sequence[int], dtype: int) -> int:
    """Bytes of one device slot (K and V) for blocks [Hkv, C, D]."""
    Hkv, Cap, D = shape
    desc = PoolDesc(1, Cap, Hkv, Hkv, D, dtype, 1, 0, 1.0)
    return int(load().kv_tier_slot_bytes(C.byref(desc)))


def kv_tier_create(k_slots, v_slots, n_groups_total: int, n_q_heads: int, rope_base: float, max_ctx: int,
                   dtype: Optional[int] = None, shape: Optional[Sequence[int]] = None) -> Tier:
    """k_slots, v_slots: torch tensors [slots, Hkv, C, D] on the GPU, or None with ``shape`` and
    ``dtype`` for a tier that only keeps the books."""
    kp = vp_ = None
    if k_slots is not None:
        import torch
        assert k_slots.is_contiguous() and v_slots.is_contiguous() and k_slots.shape == v_slots.shape
        shape = tuple(k_slots.shape)
        dtype = EN_BF16 if k_slots.dtype == torch.bfloat16 else EN_F32
        kp, vp_ = k_slots.data_ptr(), v_slots.data_ptr()
    n_slots, Hkv, Cap, D = shape
    desc = PoolDesc(n_slots, Cap, Hkv, n_q_heads, D, dtype, max_ctx, 0, rope_base)
    h = C.c_void_p()
    _check(load().kv_tier_create(C.byref(desc), int(n_groups_total), C.c_void_p(kp), C.c_void_p(vp_), C.byref(h)))
    ph = load().kv_tier_pool(h)
    pool = Pool(C.c_void_p(ph), k_slots, v_slots, desc, owned=False) if ph else None
    return Tier(h, pool, int(n_groups_total), desc)


def kv_tier_put(tier: Tier, group: int, k_rows, v_rows, length: Optional[int] = None):
    """k_rows, v_rows: host arrays or CPU tensors [Hkv, len, D] in the tier's dtype (contiguous); for a
    tier that only keeps the books pass None and ``length``."""
    if k_rows is None:
        _check(load().kv_tier_put(tier.handle, int(group), None, None, int(length)))
        return
    assert k_rows.is_contiguous() and v_rows.is_contiguous() and k_rows.shape == v_rows.shape
    assert k_rows.device.type == "cpu" and v_rows.device.type == "cpu"
    length = int(k_rows.shape[1]) if length is None else int(length)
    _check(load().kv_tier_put(tier.handle, int(group), C.c_void_p(k_rows.data_ptr()),
                              C.c_void_p(v_rows.data_ptr()), length))


def kv_tier_append(tier: Tier, group: int, k_rows, v_rows, n_tokens: Optional[int] = None, stream=None):
    """k_rows, v_rows: torch tensors [n, Hkv, D] on the GPU (contiguous, tier dtype, keys unrotated); for a
    tier that only keeps the books pass None and n_tokens."""
    if k_rows is None:
        _check(load().kv_tier_append(tier.handle, int(group), None, None, int(n_tokens), C.c_void_p(0)))
        return
    assert k_rows.is_contiguous() and v_rows.is_contiguous() and k_rows.shape == v_rows.shape
    n_tokens = int(k_rows.shape[0]) if n_tokens is None else int(n_tokens)
    _check(load().kv_tier_append(tier.handle, int(group), C.c_void_p(k_rows.data_ptr()),
                                 C.c_void_p(v_rows.data_ptr()), n_tokens, _stream(stream)))


def kv_tier_select_scored(tier: Tier, p, threshold: float, budget_tokens: int) -> np.ndarray:
    p = np.ascontiguousarray(p, dtype=np.float32)
    assert p.shape == (tier.n_groups_total,)
    out = np.zeros(tier.n_groups_total, dtype=np.int32)
    n = C.c_int32()
    _check(load().kv_tier_select_scored(tier.handle, _ip(p), C.c_float(threshold),
                                        C.c_int64(int(budget_tokens)), _ip(out), C.byref(n)))
    return out[:n.value].copy()


def kv_tier_fetch(tier: Tier, groups, stream=None) -> np.ndarray:
    """Make the groups resident; returns the slot of each (ids for segment_select on ``tier.pool``)."""
    groups = _i32(groups)
    slots = np.zeros(len(groups), dtype=np.int32)
    st = C.c_void_p(0) if tier.pool is None else _stream(stream)
    _check(load().kv_tier_fetch(tier.handle, _ip(groups), len(groups), _ip(slots), st))
    return slots


def kv_tier_fence(tier: Tier, stream=None):
    st = C.c_void_p(0) if tier.pool is None else _stream(stream)
    _check(load().kv_tier_fence(tier.handle, st))


def kv_tier_prefetch(tier: Tier, groups) -> int:
    groups = _i32(groups)
    n = C.c_int32()
    _check(load().kv_tier_prefetch(tier.handle, _ip(groups), len(groups), C.byref(n)))
    return n.value


def timing_enable(pool: Pool, n: int):
    _check(load().en_timing_enable(pool.handle, int(n)))


def timing_collect(pool: Pool, cap: int) -> np.ndarray:
    """Durations (ms) of the attention kernel launches on this pool recorded since
    the last collect."""
    ms = np.zeros(cap, dtype=np.float32)
    n = C.c_int32()
    _check(load().en_timing_collect(pool.handle, _ip(ms), cap, C.byref(n)))
    return ms[:n.value].copy()


def ceiling_mfma_bf16(sink, n_workgroups: int, iters: int, constant_operands: bool, stream=None) -> float:
    """Enqueue the matrix-instruction-only loop; returns the operations of the launch."""
    flops = C.c_double()
    _check(load().en_ceiling_mfma_bf16(sink.data_ptr(), sink.numel() * sink.element_size(), int(n_workgroups),
                                       int(iters), int(bool(constant_operands)), C.byref(flops), _stream(stream)))
    return flops.value


def ceiling_read_stream(src, sink, n_workgroups: int, stream=None) -> int:
    """Enqueue the read-only stream over `src`; returns the bytes one launch reads."""
    nbytes = src.numel() * src.element_size()
    _check(load().en_ceiling_read_stream(src.data_ptr(), nbytes, sink.data_ptr(), sink.numel() * sink.element_size(),
                                         int(n_workgroups), _stream(stream)))
    return nbytes
