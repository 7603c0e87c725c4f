"""Thin ctypes binding over the C-ABI of ``liboilbird.so`` (see ``include/oilbird.h``).

Argument marshalling only: every step of the retrieval path (normalise, score, top-k,
firing rule, depth, continuation gather) runs in the CUDA library.  torch is used for
device memory and streams.  There is no fallback: if the library cannot be loaded the
import of :func:`lib` raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, field

# The library chains the kernels of a step with programmatic launches only when the process
# loads CUDA modules eagerly (under lazy loading, the CUDA default, it launches plainly: the
# combination of lazy loading and chained launches was seen to dead-lock the first steps of a
# process now and then).  Asking for eager loading here buys those ~6 us per step on small
# pools; it takes effect if CUDA has not been initialised yet (importing torch does not do
# that), and the library is safe either way.
os.environ.setdefault("CUDA_MODULE_LOADING", "EAGER")

import numpy as np  # noqa: E402
import torch  # noqa: E402

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liboilbird.so")

OK, EINVAL, ECAPACITY, ENOMEM, ECUDA, ESTALL, EGUARD = 0, -1, -2, -3, -4, -5, -6
NEW_TRACE = 1
EVICT_TO_FIT = 2
EVICT_TO_FIT = 2
KEYS_E4M3 = 1          # pool flag: 8-bit keys
DEBUG_GUARDS = 2       # pool flag: sentinel bytes behind every array (see Pool.check_guards)
DEPTH_FIXED, DEPTH_TIERED, DEPTH_RANKED = 0, 1, 2
PATH_AUTO, PATH_GEMV, PATH_TENSOR, PATH_MMA = 0, 1, 2, 3
MAX_NQ, MAX_K, MAX_CONT_LEN, MAX_TIERS = 256, 128, 128, 4
HOST_SLOTS = 2


class PoolConfig(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("capacity_rows", ctypes.c_int64),
                ("max_traces", ctypes.c_int32), ("max_nq", ctypes.c_int32),
                ("max_k", ctypes.c_int32), ("max_append", ctypes.c_int32),
                ("device", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("arena", ctypes.c_void_p), ("arena_bytes", ctypes.c_size_t)]


class CQueryParams(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("theta", ctypes.c_float), ("offset", ctypes.c_int32),
                ("depth_mode", ctypes.c_int32), ("cont_len", ctypes.c_int32),
                ("n_tiers", ctypes.c_int32), ("tier_thr", ctypes.c_float * MAX_TIERS),
                ("tier_depth", ctypes.c_int32 * MAX_TIERS), ("exclude_tag", ctypes.c_void_p),
                ("path", ctypes.c_int32)]


class CQueryOut(ctypes.Structure):
    _fields_ = [("idx", ctypes.c_void_p), ("score", ctypes.c_void_p), ("fired", ctypes.c_void_p),
                ("cont_len", ctypes.c_void_p), ("cont_tok", ctypes.c_void_p)]


class StaticPool(ctypes.Structure):
    _fields_ = [("keys", ctypes.c_void_p), ("tokens", ctypes.c_void_p),
                ("trace_id", ctypes.c_void_p), ("trace_end", ctypes.c_void_p),
                ("n_rows", ctypes.c_int64), ("d", ctypes.c_int32), ("device", ctypes.c_int32)]


class RingConfig(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("capacity", ctypes.c_int64),
                ("max_rollout", ctypes.c_int32), ("device", ctypes.c_int32)]


class CRingOut(ctypes.Structure):
    _fields_ = [("slot", ctypes.c_void_p), ("score", ctypes.c_void_p), ("count", ctypes.c_void_p),
                ("rollout", ctypes.c_void_p), ("rollout_len", ctypes.c_void_p)]


class MergeParams(ctypes.Structure):
    _fields_ = [("budget", ctypes.c_int32), ("max_nodes", ctypes.c_int32),
                ("min_len", ctypes.c_int32), ("root_attached", ctypes.c_int32)]


class CKVCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("n_pos", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("n_pages", ctypes.c_int64),
                ("n_seq", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("device", ctypes.c_int32)]


class CKVRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class PoolStats(ctypes.Structure):
    _fields_ = [("degenerate_rows", ctypes.c_int64), ("nonfinite_queries", ctypes.c_int64),
                ("stalled", ctypes.c_int32), ("reserved", ctypes.c_int32)]


# name -> (restype, argtypes): every symbol include/oilbird.h declares
_vp, _i32, _i64, _u64, _u32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                               ctypes.c_uint32)
SYMBOLS = {
    "oilbird_query_params_default": (None, [ctypes.POINTER(CQueryParams)]),
    "oilbird_pool_arena_bytes": (ctypes.c_size_t, [ctypes.POINTER(PoolConfig)]),
    "oilbird_pool_create": (ctypes.c_int, [ctypes.POINTER(_vp), ctypes.POINTER(PoolConfig)]),
    "oilbird_pool_reset": (ctypes.c_int, [_vp, _vp]),
    "oilbird_pool_destroy": (ctypes.c_int, [_vp]),
    "oilbird_pool_append": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _vp]),
    "oilbird_pool_query": (ctypes.c_int, [_vp, _vp, _i32, ctypes.POINTER(CQueryParams),
                                          ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_pool_gather": (ctypes.c_int, [_vp, _vp, _vp, _i32, ctypes.POINTER(CQueryParams),
                                           ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_pool_evict_oldest": (ctypes.c_int, [_vp, _i32, ctypes.POINTER(_i64), _vp]),
    "oilbird_pool_step": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _vp, _i32,
                                         ctypes.POINTER(CQueryParams),
                                         ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_pool_append_host": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _vp]),
    "oilbird_pool_query_host": (ctypes.c_int, [_vp, _vp, _i32, ctypes.POINTER(CQueryParams),
                                               ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_pool_step_host": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _vp, _i32,
                                              ctypes.POINTER(CQueryParams),
                                              ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_pool_step_host_begin": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _vp, _i32,
                                                    ctypes.POINTER(CQueryParams), _i32, _vp]),
    "oilbird_pool_step_host_end": (ctypes.c_int, [_vp, _i32, ctypes.POINTER(CQueryOut)]),
    "oilbird_pool_size": (_i64, [_vp]),
    "oilbird_pool_num_traces": (_i32, [_vp]),
    "oilbird_pool_status": (ctypes.c_int, [_vp, ctypes.POINTER(PoolStats), _vp]),
    "oilbird_pool_set_wait_limit": (ctypes.c_int, [_vp, _u64, _vp]),
    "oilbird_pool_stall_selftest": (ctypes.c_int, [_vp, _vp]),
    "oilbird_pool_check_guards": (ctypes.c_int, [_vp, _vp]),
    "oilbird_pool_read_rows": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "oilbird_pool_read_codes": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp]),
    "oilbird_pool_read_traces": (_i32, [_vp, _vp, _vp, _vp, _i32]),
    "oilbird_pool_profile": (ctypes.c_int, [_vp, _i32]),
    "oilbird_pool_profile_read": (_i32, [_vp, _vp, _i32]),
    "oilbird_pool_launch_count": (_i64, [_vp]),
    "oilbird_ring_create": (ctypes.c_int, [ctypes.POINTER(_vp), ctypes.POINTER(RingConfig)]),
    "oilbird_ring_destroy": (ctypes.c_int, [_vp]),
    "oilbird_ring_reset": (ctypes.c_int, [_vp, _vp]),
    "oilbird_ring_size": (_i64, [_vp]),
    "oilbird_ring_total": (_i64, [_vp]),
    "oilbird_ring_append": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _vp]),
    "oilbird_ring_query": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i32, ctypes.c_float,
                                          ctypes.POINTER(CRingOut), _vp]),
    "oilbird_ring_step": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _i32, _i32,
                                         ctypes.c_float, ctypes.POINTER(CRingOut), _vp]),
    "oilbird_ring_read": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "oilbird_ring_last_error": (ctypes.c_char_p, []),
    "oilbird_pool_append_global": (ctypes.c_int, [_vp, _vp, _vp, _i64, _u64, _u32, _i64, _vp]),
    "oilbird_pool_to_global": (ctypes.c_int, [_vp, _vp, _vp, _i64, _vp]),
    "oilbird_merge_shards": (ctypes.c_int, [_i32, _i32, _i32, _i32, ctypes.c_float, _vp,
                                            ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t,
                                            ctypes.c_size_t, ctypes.c_size_t, _vp, _vp, _vp, _vp,
                                            _vp, _i32, _vp]),
    "oilbird_merge_params_default": (None, [ctypes.POINTER(MergeParams)]),
    "oilbird_merge_chains": (ctypes.c_int, [_i32, _vp, _vp, _i32, _i32, _vp, _vp, _i32, _i32, _vp,
                                            _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                            ctypes.POINTER(MergeParams), _i32, _vp]),
    "oilbird_index_create": (ctypes.c_int, [ctypes.POINTER(_vp), _vp, _vp, _i32, _vp]),
    "oilbird_index_refresh": (ctypes.c_int, [_vp, _vp]),
    "oilbird_index_reset": (ctypes.c_int, [_vp, _vp]),
    "oilbird_index_train": (ctypes.c_int, [_vp, _i32, _vp]),
    "oilbird_index_read_centroids": (ctypes.c_int, [_vp, _vp]),
    "oilbird_index_query": (ctypes.c_int, [_vp, _vp, _i32, _i32, ctypes.POINTER(CQueryParams),
                                           ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_index_destroy": (ctypes.c_int, [_vp]),
    "oilbird_index_rows": (_i64, [_vp]),
    "oilbird_index_read": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "oilbird_index_last_error": (ctypes.c_char_p, []),
    "oilbird_kv_block_bytes": (_i64, [_i32, _i32]),
    "oilbird_kv_workspace_bytes": (ctypes.c_size_t, [_i32]),
    "oilbird_kv_append": (ctypes.c_int, [ctypes.POINTER(CKVCache), _vp, _vp, _i32, _i32, _vp, _vp,
                                         _vp, _vp]),
    "oilbird_kv_append_packed": (ctypes.c_int, [ctypes.POINTER(CKVCache), _vp, _vp, _i32, _vp, _vp, _vp]),
    "oilbird_kv_read": (ctypes.c_int, [ctypes.POINTER(CKVCache), _i32, _vp, _vp, _vp, _vp]),
    "oilbird_kv_attend": (ctypes.c_int, [ctypes.POINTER(CKVCache), _i32, _i32, _vp, _vp, _vp, _vp,
                                         _i64, _vp, ctypes.c_float, _vp, _vp, _vp, _vp]),
    "oilbird_kv_weigh": (ctypes.c_int, [ctypes.POINTER(CKVCache), _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                        _i64, _vp, _vp, ctypes.c_float, _vp, _vp]),
    "oilbird_kv_evict": (ctypes.c_int, [ctypes.POINTER(CKVCache), _i32, _i32, _i32, _vp]),
    "oilbird_kv_status": (ctypes.c_int, [ctypes.POINTER(CKVCache), ctypes.POINTER(_i64), _vp]),
    "oilbird_kv_last_error": (ctypes.c_char_p, []),
    "oilbird_prompt_attend": (ctypes.c_int, [_vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp]),
    "oilbird_prompt_weigh": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp]),
    "oilbird_prompt_status": (ctypes.c_int, [_i32, _vp]),
    "oilbird_prompt_set_wait_limit": (ctypes.c_int, [_i32, _u64, _vp]),
    "oilbird_prompt_last_error": (ctypes.c_char_p, []),
    "oilbird_token_scores": (ctypes.c_int, [_vp, _i64, _i32, _i32, _i32, _vp, _i32, _i32, _vp, _i32, _vp]),
    "oilbird_token_scores_error": (ctypes.c_char_p, []),
    "oilbird_query_static": (ctypes.c_int, [ctypes.POINTER(StaticPool), _vp, _i32,
                                            ctypes.POINTER(CQueryParams),
                                            ctypes.POINTER(CQueryOut), _vp]),
    "oilbird_query_static_error": (ctypes.c_char_p, []),
    "oilbird_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "oilbird_last_cuda_error": (ctypes.c_char_p, []),
}

_lib = None
# Pools made without an explicit debug_guards argument take this (the GPU tests switch it on).
DEFAULT_DEBUG_GUARDS = False
GUARD_FAILURES: list = []      # pools whose guard check failed inside __del__


def _torch_empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


# Every result tensor this module creates comes from ALLOC(shape, dtype, device); the GPU
# tests replace it with an allocator that surrounds each tensor with sentinel bytes.
ALLOC = _torch_empty


def _results(stream, make):
    """make(): the results of a call on `stream` (None: the current one).  Their memory is that stream's, as it is under
    torch.cuda.stream(stream) - the current stream may still be at work on what lay there -, and once they are
    dropped it waits for the current stream too."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        got = make()
    for t in (got,) if isinstance(got, torch.Tensor) else vars(got).values() if isinstance(got, TokenScores) else got:
        if t is not None:
            t.record_stream(torch.cuda.current_stream(t.device))
    return got


def lib() -> ctypes.CDLL:
    """Load liboilbird.so (built by ``paper_2608_03839_b200.build``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2608_03839_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(L, name)          # AttributeError if a declared symbol is missing
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


class OilbirdError(RuntimeError):
    def __init__(self, code: int, where: str):
        L = lib()
        msg = L.oilbird_strerror(code).decode()
        if code in (ECUDA, ENOMEM, EGUARD) or (code == EINVAL and any(
                w in L.oilbird_last_cuda_error().decode() for w in ("aligned", "in flight"))):
            msg += " (" + L.oilbird_last_cuda_error().decode() + ")"
        super().__init__(f"{where}: {msg} [{code}]")
        self.code = code


def _flags(new_trace: bool, evict_to_fit: bool) -> int:
    return (NEW_TRACE if new_trace else 0) | (EVICT_TO_FIT if evict_to_fit else 0)


def _check(code: int, where: str) -> None:
    if code != OK:
        raise OilbirdError(code, where)


@dataclass
class QueryParams:
    """Defaults are the deployed values of the paper (k=8, theta=0.8, offset 2, D(s))."""
    k: int = 8
    theta: float = 0.8
    offset: int = 2
    depth_mode: int = DEPTH_TIERED
    cont_len: int = 48
    tier_thr: tuple = (0.90, 0.82)
    tier_depth: tuple = (48, 8)
    exclude_tag: torch.Tensor | np.ndarray | None = None   # [nq] uint64 (device: int64 tensor)
    path: int = PATH_AUTO

    def to_c(self, exclude_ptr=None) -> CQueryParams:
        key = (self.k, self.theta, self.offset, self.depth_mode, self.cont_len,
               tuple(self.tier_thr), tuple(self.tier_depth), self.path)
        c = _PARAM_CACHE.get(key)
        if c is None:
            c = CQueryParams()
            c.k, c.theta, c.offset = int(self.k), float(self.theta), int(self.offset)
            c.depth_mode, c.cont_len = int(self.depth_mode), int(self.cont_len)
            if len(self.tier_thr) != len(self.tier_depth) or len(self.tier_thr) > MAX_TIERS:
                raise ValueError("tier_thr / tier_depth: same length, at most 4")
            c.n_tiers = len(self.tier_thr)
            for i, (t, dd) in enumerate(zip(self.tier_thr, self.tier_depth)):
                c.tier_thr[i], c.tier_depth[i] = float(t), int(dd)
            c.path = int(self.path)
            if len(_PARAM_CACHE) < 256:
                _PARAM_CACHE[key] = c
        c.exclude_tag = exclude_ptr
        return c


_PARAM_CACHE: dict = {}


@dataclass
class QueryOut:
    idx: torch.Tensor        # [nq,k] int32
    score: torch.Tensor      # [nq,k] float32
    fired: torch.Tensor      # [nq] int32
    cont_len: torch.Tensor   # [nq,k] int32
    cont_tok: torch.Tensor   # [nq,k,L] int32
    _c: CQueryOut = field(default=None, repr=False)

    @staticmethod
    def empty(nq: int, k: int, L: int, device, stream=None) -> "QueryOut":
        o = QueryOut(*_results(stream, lambda: (ALLOC((nq, k), torch.int32, device),
                                                ALLOC((nq, k), torch.float32, device),
                                                ALLOC((nq,), torch.int32, device),
                                                ALLOC((nq, k), torch.int32, device),
                                                ALLOC((nq, k, L), torch.int32, device))))
        o._c = CQueryOut(o.idx.data_ptr(), o.score.data_ptr(), o.fired.data_ptr(),
                         o.cont_len.data_ptr(), o.cont_tok.data_ptr())
        return o

    def cpu(self) -> "QueryOut":
        return QueryOut(self.idx.cpu(), self.score.cpu(), self.fired.cpu(), self.cont_len.cpu(),
                        self.cont_tok.cpu())


def query_static(keys: torch.Tensor, tokens: torch.Tensor, trace_id: torch.Tensor,
                 trace_end: torch.Tensor, q: torch.Tensor, params: QueryParams,
                 out: QueryOut | None = None, stream=None) -> QueryOut:
    """oilbird_query_static: query caller-held pool arrays without any allocation.

    For hosts that own all device memory themselves and cannot let the library allocate;
    the library's only scratch is a fixed 1 MiB array in its image, so nq <= 2, k <= 128,
    no exclusion tags.  keys: CUDA bf16 [n,d], already L2-normalised (as append stores
    them); tokens / trace_id: CUDA int32 [n]; trace_end: CUDA int32 [n_traces].  Pass
    `out` to keep this wrapper itself from allocating result tensors.
    """
    for t, dt in ((keys, torch.bfloat16), (tokens, torch.int32), (trace_id, torch.int32),
                  (trace_end, torch.int32), (q, torch.bfloat16)):
        assert t.is_cuda and t.dtype == dt and t.is_contiguous()
    n, d = keys.shape
    q = q.reshape(-1, d)
    nq = q.shape[0]
    if out is None:
        out = QueryOut.empty(nq, params.k, params.cont_len, keys.device, stream)
    sp = StaticPool(keys.data_ptr(), tokens.data_ptr(), trace_id.data_ptr(), trace_end.data_ptr(),
                    n, d, keys.device.index or 0)
    cp = params.to_c(None)
    if params.exclude_tag is not None:
        cp.exclude_tag = params.exclude_tag.data_ptr()
    L = lib()
    rc = L.oilbird_query_static(ctypes.byref(sp), q.data_ptr(), nq, ctypes.byref(cp),
                                ctypes.byref(out._c), _stream_ptr(stream))
    if rc != OK:
        err = OilbirdError(rc, "oilbird_query_static")
        err.args = (err.args[0] + ": " + L.oilbird_query_static_error().decode(),)
        raise err
    return out


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


class Pool:
    """A semantic draft pool on one GPU (one per tenant)."""

    def __init__(self, d: int, capacity_rows: int, *, max_traces: int = 0, max_nq: int = 0,
                 max_k: int = 0, max_append: int = 0, device: int = 0, use_torch_arena=False,
                 key_format: str = "bf16", debug_guards: bool | None = None):
        """key_format: "bf16" (the paper's store) or "e4m3" (8-bit keys, one scale per row).
        debug_guards: sentinel bytes behind every array of the pool (check_guards() verifies
        them); None takes the module default DEFAULT_DEBUG_GUARDS."""
        self._L = lib()
        if key_format not in ("bf16", "e4m3"):
            raise ValueError("key_format must be 'bf16' or 'e4m3'")
        self.key_format = key_format
        self.debug_guards = DEFAULT_DEBUG_GUARDS if debug_guards is None else bool(debug_guards)
        if not torch.cuda.is_available():
            raise RuntimeError("oilbird pool needs a CUDA device; there is no CPU fallback")
        self.d, self.device = int(d), int(device)
        cfg = PoolConfig(d=d, capacity_rows=capacity_rows, max_traces=max_traces, max_nq=max_nq,
                         max_k=max_k, max_append=max_append, device=device,
                         flags=(KEYS_E4M3 if key_format == "e4m3" else 0) |
                               (DEBUG_GUARDS if self.debug_guards else 0),
                         arena=None, arena_bytes=0)
        self._arena = None
        if use_torch_arena:
            nbytes = self._L.oilbird_pool_arena_bytes(ctypes.byref(cfg))
            if nbytes == 0:
                raise OilbirdError(EINVAL, "oilbird_pool_arena_bytes")
            self._arena = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{device}")
            cfg.arena, cfg.arena_bytes = self._arena.data_ptr(), nbytes
        h = ctypes.c_void_p()
        _check(self._L.oilbird_pool_create(ctypes.byref(h), ctypes.byref(cfg)),
               "oilbird_pool_create")
        self._h = h
        self._dev = torch.device(f"cuda:{device}")

    def close(self) -> None:
        h, self._h = getattr(self, "_h", None), None
        if h:
            rc = OK
            if self.debug_guards:
                rc = self._L.oilbird_pool_check_guards(h, _stream_ptr(None))
            self._L.oilbird_pool_destroy(h)
            _check(rc, "oilbird_pool_check_guards (at close)")

    def __del__(self):
        try:
            self.close()
        except Exception as e:           # (module globals may be gone at interpreter exit)
            if type(e).__name__ == "OilbirdError":
                import traceback
                traceback.print_exc()
                GUARD_FAILURES.append(self)

    def check_guards(self, stream=None) -> None:
        """Raises OilbirdError(EGUARD) if a kernel wrote behind one of the pool's arrays."""
        _check(self._L.oilbird_pool_check_guards(self._h, _stream_ptr(stream)),
               "oilbird_pool_check_guards")

    def set_wait_limit(self, limit_ns: int, stream=None) -> None:
        _check(self._L.oilbird_pool_set_wait_limit(self._h, int(limit_ns), _stream_ptr(stream)),
               "oilbird_pool_set_wait_limit")

    def stall_selftest(self, stream=None) -> None:
        _check(self._L.oilbird_pool_stall_selftest(self._h, _stream_ptr(stream)),
               "oilbird_pool_stall_selftest")

    def status(self, stream=None) -> int:
        """The code of oilbird_pool_status: OK, or ESTALL after a device-side wait gave up."""
        return int(self._L.oilbird_pool_status(self._h, None, _stream_ptr(stream)))

    def __len__(self) -> int:
        return int(self._L.oilbird_pool_size(self._h))

    @property
    def num_traces(self) -> int:
        return int(self._L.oilbird_pool_num_traces(self._h))

    @property
    def launch_count(self) -> int:
        return int(self._L.oilbird_pool_launch_count(self._h))

    def reset(self, stream=None) -> None:
        _check(self._L.oilbird_pool_reset(self._h, _stream_ptr(stream)), "oilbird_pool_reset")

    # ---- device-buffer entry points -------------------------------------------------
    def append(self, states: torch.Tensor, tokens: torch.Tensor, tag: int = 0,
               new_trace: bool = True, evict_to_fit: bool = False, stream=None) -> None:
        n = int(tokens.shape[0])
        if n:
            assert states.is_cuda and tokens.is_cuda and states.dtype == torch.bfloat16
            assert tokens.dtype == torch.int32 and states.is_contiguous() and tokens.is_contiguous()
            assert states.shape == (n, self.d)
        _check(self._L.oilbird_pool_append(self._h, states.data_ptr() if n else None,
                                           tokens.data_ptr() if n else None, n, int(tag),
                                           _flags(new_trace, evict_to_fit), _stream_ptr(stream)),
               "oilbird_pool_append")

    def append_global(self, states: torch.Tensor, tokens: torch.Tensor, global_row: int,
                      tag: int = 0, new_trace: bool = True, evict_to_fit: bool = False, stream=None) -> None:
        """append() for a pool that is one shard of a larger one: global_row is the position
        of the first appended row in the logical pool."""
        n = int(tokens.shape[0])
        assert states.is_cuda and tokens.is_cuda and states.dtype == torch.bfloat16
        assert tokens.dtype == torch.int32 and states.is_contiguous() and tokens.is_contiguous()
        _check(self._L.oilbird_pool_append_global(
            self._h, states.data_ptr(), tokens.data_ptr(), n, int(tag),
            _flags(new_trace, evict_to_fit), int(global_row), _stream_ptr(stream)),
            "oilbird_pool_append_global")

    def to_global(self, idx: torch.Tensor, out: torch.Tensor | None = None, stream=None
                  ) -> torch.Tensor:
        """Local rows (int32) -> global positions (int64); -1 stays -1."""
        assert idx.is_cuda and idx.dtype == torch.int32 and idx.is_contiguous()
        if out is None:
            out, = _results(stream, lambda: (ALLOC(tuple(idx.shape), torch.int64, idx.device),))
        _check(self._L.oilbird_pool_to_global(self._h, idx.data_ptr(), out.data_ptr(),
                                              idx.numel(), _stream_ptr(stream)),
               "oilbird_pool_to_global")
        return out

    def query(self, q: torch.Tensor, params: QueryParams | None = None,
              out: QueryOut | None = None, stream=None) -> QueryOut:
        pr = params or QueryParams()
        assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        q = q.reshape(-1, self.d)
        nq = q.shape[0]
        ex_ptr = None
        if pr.exclude_tag is not None:
            ex = pr.exclude_tag
            assert ex.is_cuda and ex.dtype in (torch.int64, torch.uint64) and ex.numel() == nq
            ex_ptr = ex.data_ptr()
        if out is None:
            out = QueryOut.empty(nq, pr.k, pr.cont_len, self._dev, stream)
        cp = pr.to_c(ex_ptr)
        _check(self._L.oilbird_pool_query(self._h, q.data_ptr(), nq, ctypes.byref(cp),
                                          ctypes.byref(out._c), _stream_ptr(stream)),
               "oilbird_pool_query")
        return out

    def evict_oldest(self, n_traces: int, stream=None) -> int:
        """Drop the n_traces oldest traces and compact; rows and traces are renumbered.
        Returns the number of rows dropped."""
        dropped = ctypes.c_int64(0)
        _check(self._L.oilbird_pool_evict_oldest(self._h, int(n_traces), ctypes.byref(dropped),
                                                 _stream_ptr(stream)), "oilbird_pool_evict_oldest")
        return int(dropped.value)

    def step(self, states: torch.Tensor, tokens: torch.Tensor, q: torch.Tensor,
             params: QueryParams | None = None, out: QueryOut | None = None, tag: int = 0,
             new_trace: bool = True, evict_to_fit: bool = False, stream=None) -> QueryOut:
        """One serving step on device tensors: append(states, tokens) then query(q), in one
        call (same results as the two calls; the single-request scan overlaps the append)."""
        pr = params or QueryParams()
        assert states.is_cuda and states.dtype == torch.bfloat16 and states.is_contiguous()
        assert tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()
        assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        n = int(tokens.shape[0])
        assert states.numel() == n * self.d
        q = q.reshape(-1, self.d)
        nq = q.shape[0]
        ex_ptr = None
        if pr.exclude_tag is not None:
            ex = pr.exclude_tag
            assert ex.is_cuda and ex.dtype in (torch.int64, torch.uint64) and ex.numel() == nq
            ex_ptr = ex.data_ptr()
        if out is None:
            out = QueryOut.empty(nq, pr.k, pr.cont_len, self._dev, stream)
        cp = pr.to_c(ex_ptr)
        _check(self._L.oilbird_pool_step(
            self._h, states.data_ptr(), tokens.data_ptr(), n, int(tag),
            _flags(new_trace, evict_to_fit), q.data_ptr(), nq, ctypes.byref(cp),
            ctypes.byref(out._c), _stream_ptr(stream)), "oilbird_pool_step")
        return out

    def gather(self, idx: torch.Tensor, score: torch.Tensor, params: QueryParams,
               stream=None) -> QueryOut:
        assert idx.is_cuda and idx.dtype == torch.int32 and score.dtype == torch.float32
        nq = idx.shape[0]
        out = QueryOut.empty(nq, params.k, params.cont_len, self._dev, stream)
        out.idx, out.score = idx, score
        cp = params.to_c(None)
        co = CQueryOut(None, None, out.fired.data_ptr(), out.cont_len.data_ptr(),
                       out.cont_tok.data_ptr())
        _check(self._L.oilbird_pool_gather(self._h, idx.data_ptr(), score.data_ptr(), nq,
                                           ctypes.byref(cp), ctypes.byref(co),
                                           _stream_ptr(stream)), "oilbird_pool_gather")
        return out

    # ---- host-buffer entry points ---------------------------------------------------
    def append_host(self, states: torch.Tensor, tokens: torch.Tensor, tag: int = 0,
                    new_trace: bool = True, evict_to_fit: bool = False, stream=None) -> None:
        """states: CPU bf16 tensor [n,d] (ideally pinned); tokens: CPU int32 [n]."""
        n = int(tokens.shape[0])
        assert not states.is_cuda and not tokens.is_cuda and states.is_contiguous()
        _check(self._L.oilbird_pool_append_host(self._h, states.data_ptr(), tokens.data_ptr(), n,
                                                int(tag), _flags(new_trace, evict_to_fit),
                                                _stream_ptr(stream)), "oilbird_pool_append_host")

    def query_host(self, q: torch.Tensor, params: QueryParams | None = None,
                   out: QueryOut | None = None, stream=None) -> QueryOut:
        """q: CPU bf16 tensor [nq,d]; results land in CPU tensors."""
        pr = params or QueryParams()
        assert not q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        q = q.reshape(-1, self.d)
        nq = q.shape[0]
        ex_ptr = None
        if pr.exclude_tag is not None:
            ex = pr.exclude_tag
            assert not ex.is_cuda and ex.numel() == nq
            ex_ptr = ex.data_ptr()
        if out is None:
            out = QueryOut.empty(nq, pr.k, pr.cont_len, "cpu")
        cp = pr.to_c(ex_ptr)
        _check(self._L.oilbird_pool_query_host(self._h, q.data_ptr(), nq, ctypes.byref(cp),
                                               ctypes.byref(out._c), _stream_ptr(stream)),
               "oilbird_pool_query_host")
        return out

    def step_host(self, states: torch.Tensor, tokens: torch.Tensor, q: torch.Tensor,
                  params: QueryParams, out: QueryOut, tag: int = 0, new_trace: bool = True, evict_to_fit: bool = False,
                  stream=None) -> QueryOut:
        """One serving step from host memory: append the committed rows, then query.
        All tensors are CPU tensors; `out` must have been made with QueryOut.empty(..., "cpu")."""
        cp = params.to_c(None)
        _check(self._L.oilbird_pool_step_host(
            self._h, states.data_ptr(), tokens.data_ptr(), int(tokens.shape[0]), int(tag),
            _flags(new_trace, evict_to_fit), q.data_ptr(), int(q.shape[0]), ctypes.byref(cp),
            ctypes.byref(out._c), _stream_ptr(stream)), "oilbird_pool_step_host")
        return out

    def step_host_begin(self, states: torch.Tensor, tokens: torch.Tensor, q: torch.Tensor,
                        params: QueryParams, slot: int, tag: int = 0, new_trace: bool = True, evict_to_fit: bool = False,
                        stream=None) -> None:
        """First half of step_host: returns once the step is enqueued (slot 0 or 1)."""
        ex_ptr = params.exclude_tag.data_ptr() if params.exclude_tag is not None else None
        cp = params.to_c(ex_ptr)
        _check(self._L.oilbird_pool_step_host_begin(
            self._h, states.data_ptr(), tokens.data_ptr(), int(tokens.shape[0]), int(tag),
            _flags(new_trace, evict_to_fit), q.data_ptr(), int(q.shape[0]), ctypes.byref(cp),
            int(slot), _stream_ptr(stream)), "oilbird_pool_step_host_begin")

    def step_host_end(self, slot: int, out: QueryOut) -> QueryOut:
        """Second half: waits for that slot's step, fills the CPU tensors of `out`."""
        _check(self._L.oilbird_pool_step_host_end(self._h, int(slot), ctypes.byref(out._c)),
               "oilbird_pool_step_host_end")
        return out

    # ---- introspection --------------------------------------------------------------
    def stats(self, stream=None) -> dict:
        s = PoolStats()
        rc = self._L.oilbird_pool_status(self._h, ctypes.byref(s), _stream_ptr(stream))
        if rc not in (OK, ESTALL):
            _check(rc, "oilbird_pool_status")
        return dict(degenerate_rows=int(s.degenerate_rows),
                    nonfinite_queries=int(s.nonfinite_queries), stalled=int(s.stalled))

    def read_rows(self, row0: int = 0, n: int | None = None):
        """(keys uint16 [n,d], tokens int32 [n], trace_ids int32 [n]) as numpy arrays."""
        n = len(self) - row0 if n is None else n
        keys = np.empty((n, self.d), dtype=np.uint16) if self.key_format == "bf16" else None
        tok = np.empty(n, dtype=np.int32)
        tid = np.empty(n, dtype=np.int32)
        _check(self._L.oilbird_pool_read_rows(self._h, row0, n,
                                              keys.ctypes.data if keys is not None else None,
                                              tok.ctypes.data, tid.ctypes.data),
               "oilbird_pool_read_rows")
        return keys, tok, tid

    def read_codes(self, row0: int = 0, n: int | None = None):
        """8-bit pools: (codes uint8 [n,d], scales float32 [n]) as numpy arrays."""
        n = len(self) - row0 if n is None else n
        codes = np.empty((n, self.d), dtype=np.uint8)
        scales = np.empty(n, dtype=np.float32)
        _check(self._L.oilbird_pool_read_codes(self._h, row0, n, codes.ctypes.data,
                                               scales.ctypes.data), "oilbird_pool_read_codes")
        return codes, scales

    def traces(self):
        """(start int64 [T], end int64 [T], tag uint64 [T]) as the host tracks them."""
        T = self.num_traces
        st, en, tg = (np.empty(T, np.int64), np.empty(T, np.int64), np.empty(T, np.uint64))
        self._L.oilbird_pool_read_traces(self._h, st.ctypes.data, en.ctypes.data, tg.ctypes.data, T)
        return st, en, tg

    def profile(self, enable: bool) -> None:
        _check(self._L.oilbird_pool_profile(self._h, int(enable)), "oilbird_pool_profile")

    def profile_read(self, max_n: int = 4096) -> np.ndarray:
        buf = np.empty(max_n, dtype=np.float32)
        n = self._L.oilbird_pool_profile_read(self._h, buf.ctypes.data, max_n)
        return buf[:n].copy()


# ------------------------------------------------------------------ coarse index ----
class Index:
    """Inverted-file index over a Pool (oilbird_index_* of the C-ABI): centroids the caller
    supplies, rows assigned by the library's own k = 1 lookup, queries answered from the
    n_probe best lists plus the rows appended since the last refresh."""

    def __init__(self, pool: Pool, centroids: torch.Tensor, stream=None):
        assert centroids.is_cuda and centroids.dtype == torch.bfloat16 and centroids.is_contiguous()
        assert centroids.dim() == 2 and centroids.shape[1] == pool.d
        self._L, self.pool, self.n_lists = lib(), pool, int(centroids.shape[0])
        h = ctypes.c_void_p()
        _check(self._L.oilbird_index_create(ctypes.byref(h), pool._h, centroids.data_ptr(),
                                            self.n_lists, _stream_ptr(stream)), "oilbird_index_create")
        self._h = h

    def close(self) -> None:
        h, self._h = getattr(self, "_h", None), None
        if h:
            self._L.oilbird_index_destroy(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __len__(self) -> int:
        return int(self._L.oilbird_index_rows(self._h))

    def refresh(self, stream=None) -> None:
        _check(self._L.oilbird_index_refresh(self._h, _stream_ptr(stream)), "oilbird_index_refresh")

    def reset(self, stream=None) -> None:
        _check(self._L.oilbird_index_reset(self._h, _stream_ptr(stream)), "oilbird_index_reset")

    def train(self, iterations: int, stream=None) -> None:
        """Lloyd's iterations on the pool's rows; the lists are rebuilt afterwards."""
        _check(self._L.oilbird_index_train(self._h, int(iterations), _stream_ptr(stream)),
               "oilbird_index_train")

    def centroids(self) -> np.ndarray:
        """The raw centroid states, [n_lists, d] bf16 bit patterns (uint16)."""
        out = np.empty((self.n_lists, self.pool.d), dtype=np.uint16)
        _check(self._L.oilbird_index_read_centroids(self._h, out.ctypes.data),
               "oilbird_index_read_centroids")
        return out

    def query(self, q: torch.Tensor, n_probe: int, params: QueryParams | None = None,
              out: QueryOut | None = None, stream=None) -> QueryOut:
        pr = params or QueryParams()
        assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        q = q.reshape(-1, self.pool.d)
        nq = q.shape[0]
        ex_ptr = None
        if pr.exclude_tag is not None:
            ex = pr.exclude_tag
            assert ex.is_cuda and ex.dtype in (torch.int64, torch.uint64) and ex.numel() == nq
            ex_ptr = ex.data_ptr()
        if out is None:
            out = QueryOut.empty(nq, pr.k, pr.cont_len, self.pool._dev, stream)
        cp = pr.to_c(ex_ptr)
        _check(self._L.oilbird_index_query(self._h, q.data_ptr(), nq, int(n_probe), ctypes.byref(cp),
                                           ctypes.byref(out._c), _stream_ptr(stream)),
               "oilbird_index_query")
        return out

    def read(self):
        """(assign int32 [rows], list_off int32 [n_lists+1], list_rows int32 [rows])."""
        n = len(self)
        a, o, r = np.empty(n, np.int32), np.empty(self.n_lists + 1, np.int32), np.empty(n, np.int32)
        _check(self._L.oilbird_index_read(self._h, a.ctypes.data, o.ctypes.data, r.ctypes.data),
               "oilbird_index_read")
        return a, o, r


# ------------------------------------------------------------------ recycled pool ----
RING_MAX_M, RING_MAX_ROLLOUT, RING_MAX_NQ = 32, 16, 64


@dataclass
class RingOut:
    slot: torch.Tensor         # [nq,m] int32, -1 padded
    score: torch.Tensor        # [nq,m] float32, -inf padded
    count: torch.Tensor        # [nq] int32
    rollout: torch.Tensor      # [nq,m,R] int32, -1 padded
    rollout_len: torch.Tensor  # [nq,m] int32

    def cpu(self) -> "RingOut":
        return RingOut(self.slot.cpu(), self.score.cpu(), self.count.cpu(), self.rollout.cpu(),
                       self.rollout_len.cpu())


class Ring:
    """Rejected-branch ring buffer on one GPU (oilbird_ring_* of the C-ABI)."""

    def __init__(self, d: int, capacity: int, max_rollout: int = 6, device: int = 0):
        self._L = lib()
        if not torch.cuda.is_available():
            raise RuntimeError("oilbird ring needs a CUDA device; there is no CPU fallback")
        self.d, self.capacity, self.max_rollout = int(d), int(capacity), int(max_rollout)
        cfg = RingConfig(d=d, capacity=capacity, max_rollout=max_rollout, device=device)
        h = ctypes.c_void_p()
        _check(self._L.oilbird_ring_create(ctypes.byref(h), ctypes.byref(cfg)),
               "oilbird_ring_create")
        self._h = h
        self._dev = torch.device(f"cuda:{device}")

    def close(self) -> None:
        h, self._h = getattr(self, "_h", None), None
        if h:
            self._L.oilbird_ring_destroy(h)

    __del__ = close

    def __len__(self) -> int:
        return int(self._L.oilbird_ring_size(self._h))

    @property
    def total(self) -> int:
        return int(self._L.oilbird_ring_total(self._h))

    def reset(self, stream=None) -> None:
        _check(self._L.oilbird_ring_reset(self._h, _stream_ptr(stream)), "oilbird_ring_reset")

    def append(self, states: torch.Tensor, anchors: torch.Tensor, rollouts: torch.Tensor,
               stream=None) -> None:
        n = int(anchors.shape[0])
        assert states.is_cuda and states.dtype == torch.bfloat16 and states.is_contiguous()
        assert anchors.is_cuda and anchors.dtype == torch.int32 and anchors.is_contiguous()
        assert rollouts.is_cuda and rollouts.dtype == torch.int32 and rollouts.is_contiguous()
        assert states.shape == (n, self.d) and rollouts.shape == (n, self.max_rollout)
        _check(self._L.oilbird_ring_append(self._h, states.data_ptr(), anchors.data_ptr(),
                                           rollouts.data_ptr(), n, _stream_ptr(stream)),
               "oilbird_ring_append")

    def _out(self, nq: int, m: int, stream) -> RingOut:
        return RingOut(*_results(stream, lambda: (ALLOC((nq, m), torch.int32, self._dev),
                                                  ALLOC((nq, m), torch.float32, self._dev),
                                                  ALLOC((nq,), torch.int32, self._dev),
                                                  ALLOC((nq, m, self.max_rollout), torch.int32, self._dev),
                                                  ALLOC((nq, m), torch.int32, self._dev))))

    def query(self, q: torch.Tensor, anchors: torch.Tensor, m: int = 4, floor: float = 0.8,
              out: RingOut | None = None, stream=None) -> RingOut:
        assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        q = q.reshape(-1, self.d)
        nq = q.shape[0]
        assert anchors.is_cuda and anchors.dtype == torch.int32 and anchors.numel() == nq
        if out is None:
            out = self._out(nq, m, stream)
        co = CRingOut(out.slot.data_ptr(), out.score.data_ptr(), out.count.data_ptr(),
                      out.rollout.data_ptr(), out.rollout_len.data_ptr())
        _check(self._L.oilbird_ring_query(self._h, q.data_ptr(), anchors.data_ptr(), nq, int(m),
                                          float(floor), ctypes.byref(co), _stream_ptr(stream)),
               "oilbird_ring_query")
        return out

    def step(self, states: torch.Tensor, anchors: torch.Tensor, rollouts: torch.Tensor,
             q: torch.Tensor, q_anchors: torch.Tensor, m: int = 4, floor: float = 0.8,
             out: RingOut | None = None, stream=None) -> RingOut:
        """One verification pass: append the records, then look up, in one call."""
        n = int(anchors.shape[0])
        assert states.is_cuda and states.dtype == torch.bfloat16 and states.is_contiguous()
        assert anchors.is_cuda and anchors.dtype == torch.int32 and anchors.is_contiguous()
        assert rollouts.is_cuda and rollouts.dtype == torch.int32 and rollouts.is_contiguous()
        assert states.shape == (n, self.d) and rollouts.shape == (n, self.max_rollout)
        assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous()
        q = q.reshape(-1, self.d)
        nq = q.shape[0]
        assert q_anchors.is_cuda and q_anchors.dtype == torch.int32 and q_anchors.numel() == nq
        if out is None:
            out = self._out(nq, m, stream)
        co = CRingOut(out.slot.data_ptr(), out.score.data_ptr(), out.count.data_ptr(),
                      out.rollout.data_ptr(), out.rollout_len.data_ptr())
        _check(self._L.oilbird_ring_step(self._h, states.data_ptr(), anchors.data_ptr(),
                                         rollouts.data_ptr(), n, q.data_ptr(), q_anchors.data_ptr(),
                                         nq, int(m), float(floor), ctypes.byref(co),
                                         _stream_ptr(stream)), "oilbird_ring_step")
        return out

    def read(self):
        """(keys uint16 [cap,d], anchors int32 [cap], rollouts int32 [cap,R]) as numpy arrays."""
        keys = np.empty((self.capacity, self.d), np.uint16)
        anc = np.empty(self.capacity, np.int32)
        roll = np.empty((self.capacity, self.max_rollout), np.int32)
        _check(self._L.oilbird_ring_read(self._h, keys.ctypes.data, anc.ctypes.data,
                                         roll.ctypes.data), "oilbird_ring_read")
        return keys, anc, roll


# ------------------------------------------------------------------ tree merge ----
TREE_MAX_NODES = 64
CHAIN_SHORT, CHAIN_DUPLICATE, CHAIN_MERGED, CHAIN_CUT, CHAIN_NOT_REACHED = range(5)


@dataclass
class MergeOut:
    tree_tok: torch.Tensor      # [nq,max_nodes] int32 (updated in place)
    tree_parent: torch.Tensor   # [nq,max_nodes] int32
    n_nodes: torch.Tensor       # [nq] int32
    depth: torch.Tensor         # [nq,max_nodes] int32
    mask: torch.Tensor          # [nq,max_nodes] int64 (bit j: node j is self or an ancestor)
    status: torch.Tensor        # [nq,k+ne] int32
    bought: torch.Tensor        # [nq,k+ne] int32
    walked: torch.Tensor        # [nq,k+ne] int32


def merge_chains(tree_tok: torch.Tensor, tree_parent: torch.Tensor, n_nodes: torch.Tensor,
                 sem_tok: torch.Tensor | None, sem_len: torch.Tensor | None,
                 extra_tok: torch.Tensor | None = None, extra_len: torch.Tensor | None = None,
                 budget: int = 16, min_len: int = 2, root_attached: bool = False,
                 stream=None, out: "MergeOut | None" = None) -> MergeOut:
    """oilbird_merge_chains: post-filter the chains and merge them into each request's tree.

    tree_tok / tree_parent: CUDA int32 [nq,max_nodes] (updated in place), n_nodes: [nq].
    sem_tok [nq,k,L] / sem_len [nq,k]: a query's cont_tok / cont_len.  extra_*: further chains.
    """
    nq, max_nodes = tree_tok.shape
    dev = tree_tok.device
    k, L = (sem_tok.shape[1], sem_tok.shape[2]) if sem_tok is not None else (0, 1)
    ne, Le = (extra_tok.shape[1], extra_tok.shape[2]) if extra_tok is not None else (0, 1)
    for t in (tree_tok, tree_parent, n_nodes, sem_tok, sem_len, extra_tok, extra_len):
        assert t is None or (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous())
    if out is not None:                      # result arrays of an earlier call, written again
        depth, mask, status, bought, walked = out.depth, out.mask, out.status, out.bought, out.walked
        assert depth.shape == (nq, max_nodes) and status.shape == (nq, k + ne)
    else:
        depth, mask, status, bought, walked = _results(stream, lambda: (
            ALLOC((nq, max_nodes), torch.int32, dev), ALLOC((nq, max_nodes), torch.int64, dev),
            *(ALLOC((nq, k + ne), torch.int32, dev) for _ in range(3))))
    mp = MergeParams(budget, max_nodes, min_len, int(bool(root_attached)))
    ptr = lambda t: None if t is None else t.data_ptr()
    _check(lib().oilbird_merge_chains(nq, ptr(sem_tok), ptr(sem_len), k, L, ptr(extra_tok),
                                      ptr(extra_len), ne, Le, tree_tok.data_ptr(),
                                      tree_parent.data_ptr(), n_nodes.data_ptr(), depth.data_ptr(),
                                      mask.data_ptr(), status.data_ptr(), bought.data_ptr(),
                                      walked.data_ptr(), ctypes.byref(mp), dev.index or 0,
                                      _stream_ptr(stream)), "oilbird_merge_chains")
    return MergeOut(tree_tok, tree_parent, n_nodes, depth, mask, status, bought, walked)


# ------------------------------------------------- the verifier's 4-bit key/value cache ----
KV_BF16, KV_F16 = 0, 1
KV_MAX_SEQ, KV_MAX_GROUP, KV_MAX_EVICT_SLOTS = 1024, 64, 851968
_KV_DTYPES = {torch.bfloat16: KV_BF16, torch.float16: KV_F16}
_KV_MASKS = (torch.int64, torch.uint64)
_KV_ROWS = ctypes.c_int64 * 4          # the layout of CKVRows
_KV_STRIDES = ctypes.c_int64 * 3


def _raw_stream(index: int) -> int:
    """Handle of the device's current stream."""
    return torch.cuda.current_stream(index).cuda_stream


# the same without the Stream object (six microseconds), where torch offers it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _kv_check(rc: int, where: str) -> None:
    if rc != OK:
        err = OilbirdError(rc, where)
        err.args = (err.args[0] + ": " + lib().oilbird_kv_last_error().decode(),)
        raise err


def _no_backward(who: str) -> None:
    """For a tensor that wants a gradient: results come without one."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{who} no backward pass: detach the tensor, or call under torch.no_grad()")


class KVCache:
    """Keys and values of n_seq requests (one layer) in 4 bits, in pages, with the attention
    weight each slot has received (oilbird_kv_* of the C-ABI; see include/oilbird.h for the
    format and the semantics of every call).

    KVCache(...) allocates everything, max_len slots for each sequence.  KVCache.over(...) works
    on tensors the caller holds: pages (uint8, the blocks of all pages), weight (fp32) and pos
    (int32) [n_pages, n_kv_heads, page_size], page_table (int32 [n_seq, max_pages]), seq_len and
    n_pos (int32 [n_seq]).  workspace (22 MB for heads of 64, 43 MB for 128; None: one of its own) may
    be shared by caches that are used on one stream, as a model's layers are: pass another's .workspace.
    There is no backward pass: tensors that want a gradient are refused where one would be recorded.
    """

    def __init__(self, n_seq: int, n_kv_heads: int, head_dim: int, max_len: int, *,
                 page_size: int = 64, dtype=torch.bfloat16, device: int = 0,
                 workspace: torch.Tensor | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("the key/value cache needs a CUDA device; there is no CPU fallback")
        dev = torch.device(f"cuda:{device}")
        block = lib().oilbird_kv_block_bytes(int(head_dim), int(page_size))
        if block == 0:
            raise ValueError("head_dim: 64 or 128; page_size: 16, 32 or 64")
        per = max(1, -(-int(max_len) // page_size))
        n_pages = n_seq * per
        self._setup(torch.zeros(n_pages * n_kv_heads * block, dtype=torch.uint8, device=dev),
                    torch.zeros(n_pages, n_kv_heads, page_size, device=dev),
                    torch.zeros(n_pages, n_kv_heads, page_size, dtype=torch.int32, device=dev),
                    torch.arange(n_pages, dtype=torch.int32, device=dev).view(n_seq, per),
                    torch.zeros(n_seq, dtype=torch.int32, device=dev),
                    torch.zeros(n_seq, dtype=torch.int32, device=dev), dtype, head_dim, workspace)

    @classmethod
    def over(cls, pages: torch.Tensor, weight: torch.Tensor, pos: torch.Tensor,
             page_table: torch.Tensor, seq_len: torch.Tensor, n_pos: torch.Tensor, *,
             dtype=torch.bfloat16, workspace: torch.Tensor | None = None) -> "KVCache":
        self = cls.__new__(cls)
        L = lib()
        page_size = int(weight.shape[2])
        cells = max(1, weight.shape[0] * weight.shape[1])
        head_dim = [d for d in (64, 128) if L.oilbird_kv_block_bytes(d, page_size) * cells == pages.numel()]
        if not head_dim:
            raise ValueError("pages: n_pages * n_kv_heads blocks of oilbird_kv_block_bytes() bytes")
        self._setup(pages, weight, pos, page_table, seq_len, n_pos, dtype, head_dim[0], workspace)
        return self

    def _setup(self, pages, weight, pos, page_table, seq_len, n_pos, dtype, head_dim, workspace):
        self._L = lib()
        dev = pages.device
        if dtype not in _KV_DTYPES:
            raise ValueError("dtype: torch.bfloat16 or torch.float16")
        n_seq, max_pages = page_table.shape
        for t, dt, shape in ((pages, torch.uint8, None), (weight, torch.float32, None),
                             (pos, torch.int32, weight.shape), (page_table, torch.int32, None),
                             (seq_len, torch.int32, (n_seq,)), (n_pos, torch.int32, (n_seq,))):
            if not t.is_cuda or t.device != dev or t.dtype != dt or not t.is_contiguous() or \
                    (shape is not None and tuple(t.shape) != tuple(shape)):
                raise ValueError("the cache's tensors: contiguous, on one CUDA device, of the documented "
                                 "types and shapes")
        need = self._L.oilbird_kv_workspace_bytes(int(head_dim))
        if workspace is None:
            workspace = torch.zeros(need, dtype=torch.uint8, device=dev)
        elif workspace.device != dev or workspace.dtype != torch.uint8 or not workspace.is_contiguous() or \
                workspace.numel() < need or workspace.data_ptr() % 16:
            raise ValueError(f"workspace: {need} bytes at least (uint8, contiguous, 16-byte aligned, zeroed once), "
                             "on the cache's device")
        self.pages, self.weight, self.pos, self.page_table = pages, weight, pos, page_table
        self.seq_len, self.n_pos, self.workspace = seq_len, n_pos, workspace
        self.dtype, self.head_dim, self.n_kv_heads = dtype, int(head_dim), int(weight.shape[1])
        self.n_seq, self.page_size = int(n_seq), int(weight.shape[2])
        self._dev, self._index = dev, dev.index or 0
        self._seqs, self._scale = (self.n_seq,), self.head_dim ** -0.5
        self._c = CKVCache(pages.data_ptr(), weight.data_ptr(), pos.data_ptr(),
                           page_table.data_ptr(), seq_len.data_ptr(), n_pos.data_ptr(),
                           workspace.data_ptr(), workspace.numel(), weight.shape[0], n_seq,
                           max_pages, self.page_size, self.n_kv_heads, self.head_dim,
                           _KV_DTYPES[dtype], dev.index or 0)
        self._ref = ctypes.byref(self._c)

    # (These run for every argument of every call, on the path that bounds small calls: one
    # comparison for each property, and four integers in place of the struct of the same layout.)
    def _rows(self, t: torch.Tensor, heads: int, m: int):
        """The C view of a [n_seq, m, heads, head_dim] tensor (any strides but the last)."""
        if t.dtype is self.dtype and t.shape == (self.n_seq, m, heads, self.head_dim) and t.get_device() == self._index:
            if t.requires_grad:
                _no_backward("the key/value cache has")
            s0, s1, s2, s3 = t.stride()
            if s3 == 1:
                return _KV_ROWS(t.data_ptr(), s0, s1, s2)
        raise AssertionError(f"a {self.dtype} tensor [{self.n_seq}, {m}, {heads}, {self.head_dim}] on {self._dev} "
                             "with contiguous channels")

    def _packed_rows(self, t: torch.Tensor, m: int):
        """The C view of a [m, n_kv_heads, head_dim] tensor (any strides but the last)."""
        if t.shape != (m, self.n_kv_heads, self.head_dim):
            raise AssertionError(f"a tensor [{m}, {self.n_kv_heads}, {self.head_dim}]")
        return self._rows(t.expand(self.n_seq, -1, -1, -1), self.n_kv_heads, m)

    def _vec(self, t, dtype, shape):
        """Pointer of an optional contiguous tensor of that type and shape."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index or not t.is_contiguous():
            raise AssertionError(f"a contiguous {dtype} tensor {list(shape)} on {self._dev}")
        if t.requires_grad:
            _no_backward("the key/value cache has")
        return t.data_ptr()

    def _lse(self, t, m, heads):
        """Pointer and strides of a [n_seq, m, heads] fp32 tensor."""
        if t.dtype is not torch.float32 or t.shape != (self.n_seq, m, heads) or t.get_device() != self._index:
            raise AssertionError(f"an fp32 tensor [{self.n_seq}, {m}, {heads}] on {self._dev}")
        if t.requires_grad:
            _no_backward("the key/value cache has")
        return t.data_ptr(), None if t.is_contiguous() else _KV_STRIDES(*t.stride())

    def _mask(self, mask, m):
        if mask is None:
            return None, 0
        shape = mask.shape
        if mask.dtype not in _KV_MASKS or len(shape) != 2 or shape[0] != self.n_seq or shape[1] < m or \
                mask.get_device() != self._index or (mask.stride(1) != 1 and shape[1] > 1):
            raise AssertionError(f"an int64 tensor [{self.n_seq}, {m} or more] on {self._dev}")
        return mask.data_ptr(), mask.stride(0)

    def _new(self, like: torch.Tensor, shape, stream) -> torch.Tensor:
        if stream is not None:
            return _results(stream, lambda: (self._new(like, shape, None),))[0]
        # (new_empty takes half the time of torch.empty with a type and a device)
        return like.new_empty(shape) if ALLOC is _torch_empty else ALLOC(shape, like.dtype, self._dev)

    def _stream(self, stream) -> int:
        if stream is not None:
            return stream.cuda_stream
        return _raw_stream(self._index)

    def append(self, k: torch.Tensor, v: torch.Tensor, n_new: torch.Tensor | None = None,
               select: torch.Tensor | None = None, weight: torch.Tensor | None = None,
               stream=None, first: torch.Tensor | None = None) -> None:
        """Store rows of k and v [n_seq, m, n_kv_heads, head_dim]: rows select[s, :n_new[s]]
        (int32 [n_seq, rows]; None: the first n_new[s], None: all).  weight: fp32
        [n_seq, n_kv_heads, m], the rows' first weights (None: 0).  With first (int32 [n_seq + 1]) k and v are packed
        [m, n_kv_heads, head_dim]: rows first[s] .. first[s + 1] - 1 join sequence s; weight [n_kv_heads, m]."""
        if first is not None:
            if n_new is not None or select is not None:
                raise AssertionError("packed rows (first) take neither n_new nor select")
            m = k.shape[0]
            if m > 0:
                _kv_check(self._L.oilbird_kv_append_packed(
                    self._ref, self._packed_rows(k, m), self._packed_rows(v, m), m,
                    self._vec(first, torch.int32, (self.n_seq + 1,)),
                    self._vec(weight, torch.float32, (self.n_kv_heads, m)), self._stream(stream)), "oilbird_kv_append_packed")
            return
        m = k.shape[1]
        if m == 0:
            return
        rows = m if select is None else select.shape[1]
        _kv_check(self._L.oilbird_kv_append(
            self._ref, self._rows(k, self.n_kv_heads, m), self._rows(v, self.n_kv_heads, m), m, rows,
            self._vec(n_new, torch.int32, self._seqs),
            self._vec(select, torch.int32, (self.n_seq, rows)),
            self._vec(weight, torch.float32, (self.n_seq, self.n_kv_heads, m)),
            self._stream(stream)), "oilbird_kv_append")

    def read(self, n: int, start: torch.Tensor | None = None, stream=None):
        """Slots start[s] .. start[s] + n - 1 (int32 [n_seq]; None: from 0) in 16 bits: (k, v), each
        [n_seq, n, n_kv_heads, head_dim]; zeros where a sequence has no slot."""
        shape = (self.n_seq, n, self.n_kv_heads, self.head_dim)
        k, v = _results(stream, lambda: (ALLOC(shape, self.dtype, self._dev), ALLOC(shape, self.dtype, self._dev)))
        _kv_check(self._L.oilbird_kv_read(self._ref, n, self._vec(start, torch.int32, self._seqs),
                                          k.data_ptr(), v.data_ptr(), self._stream(stream)),
                  "oilbird_kv_read")
        return k, v

    def attend(self, q: torch.Tensor, k_new: torch.Tensor | None = None,
               v_new: torch.Tensor | None = None, mask: torch.Tensor | None = None,
               n_new: torch.Tensor | None = None, scale: float | None = None,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None, stream=None):
        """Attention of q [n_seq, m, n_q_heads, head_dim] over the cached slots and, with k_new and
        v_new [n_seq, m, n_kv_heads, head_dim], over the nodes that mask (int64 [n_seq, >= m], bit j:
        sees node j; None: nodes 0..i) names.  n_new: int32 [n_seq] nodes of each sequence (None: m).
        Returns (out, lse): out like q, lse fp32 [n_seq, m, n_q_heads] (natural logarithm)."""
        _, m, heads, _ = q.shape
        if out is None:
            out = self._new(q, (self.n_seq, m, heads, self.head_dim), stream)
        if lse is None:
            lse = self._new(self.weight, (self.n_seq, m, heads), stream)
        mp, ms = self._mask(mask, m)
        _kv_check(self._L.oilbird_kv_attend(
            self._ref, heads, m, self._rows(q, heads, m),
            None if k_new is None else self._rows(k_new, self.n_kv_heads, m),
            None if v_new is None else self._rows(v_new, self.n_kv_heads, m), mp, ms,
            self._vec(n_new, torch.int32, self._seqs),
            self._scale if scale is None else scale, self._rows(out, heads, m),
            *self._lse(lse, m, heads), self._stream(stream)), "oilbird_kv_attend")
        return out, lse

    def weigh(self, q: torch.Tensor, lse: torch.Tensor, k_new: torch.Tensor | None = None,
              mask: torch.Tensor | None = None, n_new: torch.Tensor | None = None,
              row_weight: torch.Tensor | None = None, scale: float | None = None, stream=None):
        """Add to every slot's weight what the nodes with row_weight (fp32 [n_seq, m]; None: 1) gave
        it in attend (same arguments, and its lse).  Returns the same sums for the new nodes,
        fp32 [n_seq, n_kv_heads, m] (None without k_new): append()'s weight."""
        _, m, heads, _ = q.shape
        nodes = None
        if k_new is not None:
            nodes = self._new(self.weight, (self.n_seq, self.n_kv_heads, m), stream)
        mp, ms = self._mask(mask, m)
        _kv_check(self._L.oilbird_kv_weigh(
            self._ref, heads, m, self._rows(q, heads, m),
            *self._lse(lse, m, heads),
            None if k_new is None else self._rows(k_new, self.n_kv_heads, m), mp, ms,
            self._vec(n_new, torch.int32, self._seqs),
            self._vec(row_weight, torch.float32, (self.n_seq, m)),
            self._scale if scale is None else scale,
            None if nodes is None else nodes.data_ptr(), self._stream(stream)), "oilbird_kv_weigh")
        return nodes

    def evict(self, budget: int, sink: int = 4, recent: int | None = None, stream=None) -> None:
        """Cut every sequence to `budget` slots per head: positions below sink and the newest
        `recent` (None: half the budget, as far as sink leaves room) stay, then the slots of
        greatest weight."""
        # (the C call takes 32 bits, and a number beyond them would come out as another)
        budget, sink = (max(-1, min(int(x), 2 ** 31 - 1)) for x in (budget, sink))
        recent = max(0, min(budget // 2, budget - sink)) if recent is None else max(-1, min(int(recent), 2 ** 31 - 1))
        _kv_check(self._L.oilbird_kv_evict(self._ref, budget, sink, recent, self._stream(stream)), "oilbird_kv_evict")

    def dropped(self, stream=None) -> int:
        """Rows append() could not store so far (synchronises)."""
        n = ctypes.c_int64()
        _kv_check(self._L.oilbird_kv_status(self._ref, ctypes.byref(n), self._stream(stream)),
                  "oilbird_kv_status")
        return int(n.value)


# ------------------------------------------------------------------ whole prompts ----
def _stream_of(stream, t: torch.Tensor):
    if stream.device != t.device:
        raise AssertionError(f"a stream of {t.device}")
    return stream


_PROMPT = ctypes.c_int64 * 9         # oilbird_prompt: two sides of three words, six 32-bit numbers


def _prompt_check(rc: int, where: str) -> None:
    if rc != OK:
        err = OilbirdError(rc, where)
        err.args = (err.args[0] + ": " + lib().oilbird_prompt_last_error().decode(),)
        raise err


class _Prompt:
    """Checked arguments of a prompt call: the C view of both sides, and of every tensor given."""

    def __init__(self, q, k, first, n_new, first_k, n_k):
        self.packed, self.packed_k = q.dim() == 3, k.dim() == 3
        if (not self.packed and q.dim() != 4) or (not self.packed_k and k.dim() != 4):
            raise AssertionError("q and k: [rows, heads, head_dim] packed, [n_seq, rows, heads, head_dim] padded")
        if q.dtype not in _KV_DTYPES or not q.is_cuda:
            raise AssertionError("q: a bf16 or f16 tensor on a CUDA device; there is no CPU fallback")
        self.dtype, self.dev, self.index = q.dtype, q.device, q.get_device()
        if self.packed and first is None or not self.packed and first is not None:
            raise AssertionError("first goes with packed q [rows, heads, head_dim], and only with it")
        if first_k is None and self.packed_k:
            first_k = first
        if self.packed_k != (first_k is not None):
            raise AssertionError("first_k (or first) goes with packed k, and only with it")
        if self.packed and n_new is not None or self.packed_k and n_k is not None:
            raise AssertionError("n_new and n_k count the rows of padded sequences")
        self.q_shape, self.k_shape = q.shape, k.shape
        *lead, self.rows, self.heads, self.d = self.q_shape
        *lead_k, self.rows_k, self.kv_heads, d = self.k_shape
        self.n_seq = first.shape[0] - 1 if self.packed else lead[0]
        if d != self.d or (lead_k and lead_k[0] != self.n_seq):
            raise AssertionError(f"k: {'' if self.packed_k else f'{self.n_seq} sequences, '}head_dim {self.d}")
        if n_k is None and not self.packed and not self.packed_k and self.rows_k == self.rows:
            n_k = n_new                  # a prompt over itself
        offsets, counts = (self.n_seq + 1,), (self.n_seq,)
        self.c = _PROMPT(self.vec(first, torch.int32, offsets) or 0, self.vec(n_new, torch.int32, counts) or 0, self.rows,
                         self.vec(first_k, torch.int32, offsets) or 0, self.vec(n_k, torch.int32, counts) or 0, self.rows_k,
                         self.n_seq | self.heads << 32, self.kv_heads | self.d << 32,
                         _KV_DTYPES[self.dtype] | self.index << 32)

    def vec(self, t, dtype, shape):
        """Pointer of an optional contiguous tensor of that type and shape."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.index or not t.is_contiguous():
            raise AssertionError(f"a contiguous {dtype} tensor {list(shape)} on {self.dev}")
        if t.requires_grad:
            _no_backward("prompt calls have")
        return t.data_ptr()

    # (what runs for every argument of every call bounds the smallest calls: see KVCache._rows)
    def view(self, t, shape):
        """The C view of a tensor of that shape (any strides but the last)."""
        if t.dtype is self.dtype and t.shape == shape and t.get_device() == self.index:
            if t.requires_grad:
                _no_backward("prompt calls have")
            stride = t.stride()
            if stride[-1] == 1:
                return _KV_ROWS(t.data_ptr(), *stride[:3]) if len(stride) == 4 else _KV_ROWS(t.data_ptr(), 0, *stride[:2])
        raise AssertionError(f"a {self.dtype} tensor {list(shape)} on {self.dev} with contiguous channels")

    def new(self, q):
        """A fresh result like q, and its C view."""
        t = q.new_empty(self.q_shape) if ALLOC is _torch_empty else ALLOC(self.q_shape, self.dtype, self.dev)
        row = self.heads * self.d
        return t, _KV_ROWS(t.data_ptr(), 0 if self.packed else self.rows * row, row, self.d)

    def lse(self, t):
        """Pointer and strides of an fp32 tensor [.., n_q_heads]."""
        if t.dtype is not torch.float32 or t.shape != self.q_shape[:-1] or t.get_device() != self.index:
            raise AssertionError(f"an fp32 tensor {list(self.q_shape[:-1])} on {self.dev}")
        if t.requires_grad:
            _no_backward("prompt calls have")
        if t.is_contiguous():
            return t.data_ptr(), None
        return t.data_ptr(), _KV_STRIDES(0 if self.packed else t.stride(0), *t.stride()[-2:])


def prompt_attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor | None = None,
                  n_new: torch.Tensor | None = None, first_k: torch.Tensor | None = None,
                  n_k: torch.Tensor | None = None, scale: float | None = None, out: torch.Tensor | None = None,
                  lse: torch.Tensor | None = None, stream=None):
    """Causal attention over whole prompts (oilbird_prompt_attend).  Packed: q [rows, n_q_heads, head_dim], k and v
    [rows_k, n_kv_heads, head_dim], first and first_k (int32 [n_seq + 1]; first_k None: first) say where
    each sequence begins.  Padded: q [n_seq, rows, n_q_heads, head_dim], k and v likewise, n_new and n_k
    (int32 [n_seq]; None: all rows, n_k: n_new where both have as many rows) count each sequence's rows.
    The query rows are the last of their sequence's keys.  scale: None for 1 / sqrt(head_dim).
    Returns (out, lse): out like q, lse fp32 [..., n_q_heads] (natural logarithm).  Packed rows of no sequence
    are not written."""
    if stream is not None:
        return _results(_stream_of(stream, q), lambda: prompt_attend(q, k, v, first, n_new, first_k, n_k, scale, out, lse))
    p = _Prompt(q, k, first, n_new, first_k, n_k)
    out, out_view = p.new(q) if out is None else (out, p.view(out, p.q_shape))
    if lse is None:
        lse = (q.new_empty(p.q_shape[:-1], dtype=torch.float32) if ALLOC is _torch_empty else
               ALLOC(p.q_shape[:-1], torch.float32, p.dev))
    _prompt_check(lib().oilbird_prompt_attend(
        p.c, p.view(q, p.q_shape), p.view(k, p.k_shape), p.view(v, p.k_shape), p.d ** -0.5 if scale is None else scale, out_view,
        *p.lse(lse), _raw_stream(p.index)), "oilbird_prompt_attend")
    return out, lse


def prompt_weigh(q: torch.Tensor, lse: torch.Tensor, k: torch.Tensor, first: torch.Tensor | None = None,
                 n_new: torch.Tensor | None = None, first_k: torch.Tensor | None = None,
                 n_k: torch.Tensor | None = None, row_weight: torch.Tensor | None = None,
                 scale: float | None = None, weight: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The attention weight that the rows with row_weight (fp32 [n_seq, rows] or [rows]; None: 1) gave each key in
    prompt_attend (same arguments, and its lse; oilbird_prompt_weigh): fp32 [n_seq, n_kv_heads, rows_k], which
    KVCache.append takes, packed [n_kv_heads, rows_k]."""
    if stream is not None:
        return _results(_stream_of(stream, q),
                        lambda: prompt_weigh(q, lse, k, first, n_new, first_k, n_k, row_weight, scale, weight))
    p = _Prompt(q, k, first, n_new, first_k, n_k)
    shape = (p.kv_heads, p.rows_k) if p.packed_k else (p.n_seq, p.kv_heads, p.rows_k)
    if weight is None:
        weight = ALLOC(shape, torch.float32, p.dev)
    _prompt_check(lib().oilbird_prompt_weigh(
        p.c, p.view(q, p.q_shape), *p.lse(lse), p.view(k, p.k_shape), p.vec(row_weight, torch.float32, p.q_shape[:-2]),
        p.d ** -0.5 if scale is None else scale, p.vec(weight, torch.float32, shape), _raw_stream(p.index)), "oilbird_prompt_weigh")
    return weight


def prompt_status(device: int = 0, stream=None) -> int:
    """OK, or ESTALL if a bounded wait of a prompt call gave up since the last status (synchronises)."""
    rc = lib().oilbird_prompt_status(device, _raw_stream(device) if stream is None else stream.cuda_stream)
    if rc != ESTALL:
        _prompt_check(rc, "oilbird_prompt_status")
    return rc


def prompt_set_wait_limit(limit_ns: int, device: int = 0, stream=None) -> None:
    """How long the device-side waits of prompt calls may take (0: two seconds)."""
    _prompt_check(lib().oilbird_prompt_set_wait_limit(device, limit_ns, _raw_stream(device) if stream is None
                                                      else stream.cuda_stream), "oilbird_prompt_set_wait_limit")


# ------------------------------------------------------------------ token scores ----
LOGITS_BF16, LOGITS_F16, LOGITS_F32 = 0, 1, 2
SCORES_MAX_VOCAB, SCORES_MAX_TOP = 16777216, 64
_LOGITS_DTYPES = {torch.bfloat16: LOGITS_BF16, torch.float16: LOGITS_F16, torch.float32: LOGITS_F32}
_SCORES_OUT = ctypes.c_int64 * 5     # oilbird_scores_out


@dataclass
class TokenScores:
    logp: torch.Tensor | None   # [rows, n_tokens] fp32 (None without tokens)
    lse: torch.Tensor           # [rows] fp32
    entropy: torch.Tensor       # [rows] fp32
    top_id: torch.Tensor        # [rows, top] int32
    top_logp: torch.Tensor      # [rows, top] fp32


def token_scores(logits: torch.Tensor, tokens: torch.Tensor | None = None, top: int = 0, stream=None) -> TokenScores:
    """Log probabilities of the given tokens (int32 [rows, n_tokens]), entropy and the `top` best tokens of each row
    of logits [rows, vocab] (bf16, f16 or fp32; rows of any stride), in one reading (oilbird_token_scores)."""
    if logits.dtype not in _LOGITS_DTYPES or logits.dim() != 2 or not logits.is_cuda or \
            (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise AssertionError("logits: a bf16, f16 or fp32 tensor [rows, vocab] on a CUDA device, with contiguous rows; "
                             "there is no CPU fallback")
    if logits.requires_grad:
        _no_backward("token scores have")
    if stream is not None:
        return _results(_stream_of(stream, logits), lambda: token_scores(logits, tokens, top))
    rows, vocab = logits.shape
    index, dev = logits.get_device(), logits.device
    n = 0
    if tokens is not None:
        if tokens.dtype is not torch.int32 or tokens.dim() != 2 or tokens.shape[0] != rows or \
                tokens.get_device() != index or not tokens.is_contiguous():
            raise AssertionError(f"tokens: a contiguous int32 tensor [{rows}, n] on {dev}")
        n = tokens.shape[1]
    top = max(-1, min(int(top), 2 ** 31 - 1))
    k = max(0, min(top, SCORES_MAX_TOP))
    if ALLOC is _torch_empty:            # one allocation for all results: five take longer than the call
        buf = logits.new_empty(rows * (2 + n + 2 * k), dtype=torch.float32)
        lse, entropy, logp, best, top_logp = buf.split_with_sizes((rows, rows, rows * n, rows * k, rows * k))
        got = TokenScores(None if tokens is None else logp.view(rows, n), lse, entropy, best.view(torch.int32).view(rows, k),
                          top_logp.view(rows, k))
    else:
        got = TokenScores(None if tokens is None else ALLOC((rows, n), torch.float32, dev), ALLOC((rows,), torch.float32, dev),
                          ALLOC((rows,), torch.float32, dev), ALLOC((rows, k), torch.int32, dev), ALLOC((rows, k), torch.float32, dev))
    out = _SCORES_OUT(got.logp.data_ptr() if n else 0, got.lse.data_ptr(), got.entropy.data_ptr(), got.top_id.data_ptr(),
                      got.top_logp.data_ptr())
    rc = lib().oilbird_token_scores(logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, rows, vocab,
                                    _LOGITS_DTYPES[logits.dtype], tokens.data_ptr() if n else None, n, top, out, index,
                                    _raw_stream(index))
    if rc != OK:
        err = OilbirdError(rc, "oilbird_token_scores")
        err.args = (err.args[0] + ": " + lib().oilbird_token_scores_error().decode(),)
        raise err
    return got
