"""ctypes binding of libkvmem_b200.so: argument marshalling only.

Every step of the recall path (index build, scoring, selection, view assembly, attention)
runs in the library's CUDA kernels; PyTorch supplies device memory and streams.  There is no
CPU fallback: if the shared library is missing or a call fails, an exception is raised.
Names mirror the C ABI declared in ``include/kvmem.h``.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import _build

OK = 0
E_INVALID, E_CAPACITY, E_STATE, E_CUDA, E_TIMEOUT, E_UNSUPPORTED, E_DEVICE_RANGE = -1, -2, -3, -4, -5, -6, -7


class KvmemError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"kvmem status {status}: {message}")
        self.status = status


class PoolConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "block_tokens",
                                          "max_sessions", "max_blocks", "max_blocks_per_session", "device",
                                          "rope_max_positions")] + [("rope_theta", C.c_float),
                                                                   ("rope_in_block_keys", C.c_int32), ("fp8_pages", C.c_int32),
                                                                   ("fp8_k_scale", C.c_float), ("fp8_v_scale", C.c_float)]


class TailStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("cap_tokens", C.c_int32), ("n_tokens", C.c_void_p)]


class RopeStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("layout", "rotary_dim", "scaling")] + \
               [(n, C.c_float) for n in ("factor", "original_positions", "turns_fast", "turns_slow")]


class SelectParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("budget_blocks", "max_view_tokens", "mandatory_tokens",
                                          "n_sink_blocks", "n_recent_blocks")]


_lib = None
_BF16, _I32 = torch.bfloat16, torch.int32


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Load (building first if sources are newer) the CUDA library.  Raises if that is impossible."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    if path is None:
        path = _build.LIB_PATH
        if not os.path.exists(path) or os.environ.get("KVMEM_REBUILD"):
            _build.build()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with paper_2609_04852_b200._build.build()")
    L = C.CDLL(path)
    vp, i32, sz, f32 = C.c_void_p, C.c_int32, C.c_size_t, C.c_float
    cfgp, prmp, tailp = C.POINTER(PoolConfig), C.POINTER(SelectParams), C.POINTER(TailStruct)
    ropep, i64 = C.POINTER(RopeStruct), C.c_int64
    sig = {
        "kvmem_pool_bytes": (sz, [cfgp]),
        "kvmem_budget_blocks": (i32, [prmp, i32, i32]),
        "kvmem_select_workspace_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_attend_workspace_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_last_error": (C.c_char_p, []),
        "kvmem_pool_create": (C.c_int, [cfgp, vp, sz, C.POINTER(vp)]),
        "kvmem_pool_destroy": (C.c_int, [vp]),
        "kvmem_session_reset": (C.c_int, [vp, i32, vp]),
        "kvmem_session_blocks": (i32, [vp, i32]),
        "kvmem_append_blocks": (C.c_int, [vp, i32, vp, vp, i32, C.POINTER(i32), vp]),
        "kvmem_score": (C.c_int, [vp, i32, i32, vp, i32, vp, f32, vp, sz, vp]),
        "kvmem_topk": (C.c_int, [vp, i32, i32, vp, i32, prmp, vp, i32, vp, vp]),
        "kvmem_score_host_workspace_bytes": (sz, [vp, i32, i32, i32]),
        "kvmem_score_host_staging_bytes": (sz, [vp, i32]),
        "kvmem_score_host_index": (C.c_int, [vp, vp, i32, i32, vp, i32, i32, vp, vp, sz, vp, sz, vp]),
        "kvmem_select": (C.c_int, [vp, i32, i32, vp, i32, prmp, vp, i32, vp, vp, vp, sz, vp]),
        "kvmem_materialize": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, i32, vp]),
        "kvmem_materialize_delta": (C.c_int, [vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp]),
        "kvmem_view_attend": (C.c_int, [vp, i32, vp, i32, vp, vp, i32, vp, f32, vp, vp, vp, sz, vp]),
        "kvmem_get_index": (C.c_int, [vp, i32, C.POINTER(vp), C.POINTER(i32)]),
        "kvmem_get_block_table": (C.c_int, [vp, i32, C.POINTER(vp), C.POINTER(i32)]),
        "kvmem_device_status": (C.c_int, [vp, C.POINTER(i32), vp]),
        "kvmem_set_option": (C.c_int, [C.c_char_p, i32]),
        "kvmem_materialize_attend": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_append_blocks_rope": (C.c_int, [vp, i32, vp, vp, i32, C.POINTER(i32), C.POINTER(i32), vp]),
        "kvmem_rope_rotate": (C.c_int, [vp, vp, vp, C.c_int64, i32, vp, i32, vp]),
        "kvmem_materialize_rope": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, i32, i32, vp]),
        "kvmem_working_set_delta": (C.c_int, [vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]),
        "kvmem_view_cache_bytes": (sz, [vp, i32]),
        "kvmem_view_cache_layout": (C.c_int, [vp, i32, C.POINTER(sz)]),
        "kvmem_view_cache_reset": (C.c_int, [vp, vp, sz, i32, vp]),
        "kvmem_view_cache_update": (C.c_int, [vp, i32, vp, vp, vp, sz, i32, i32, i32, vp, vp]),
        "kvmem_view_cache_attend": (C.c_int, [vp, vp, i32, vp, sz, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_paged_attend": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, f32, vp, vp, vp, sz, vp]),
        "kvmem_paged_attend_rope": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_materialize_attend_rope": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, i32, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_materialize_fp8": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, i32, f32, f32, vp]),
        "kvmem_materialize_fp8_rope": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, i32, i32, f32, f32, vp]),
        "kvmem_paged_attend_fp8": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, f32, vp, vp, vp, sz, vp]),
        "kvmem_paged_attend_fp8_rope": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_materialize_attend_fp8": (C.c_int, [vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp]),
        "kvmem_view_attend_fp8": (C.c_int, [vp, i32, vp, i32, vp, vp, i32, vp, f32, f32, f32, vp, vp, vp, sz, vp]),
        "kvmem_view_attend_static": (C.c_int, [vp, i32, vp, i32, vp, vp, i32, vp, f32, vp, vp, vp]),
        "kvmem_selftest_wait_timeout": (C.c_int, [vp, C.c_uint32, vp, vp]),
        "kvmem_selftest_joint_wait_timeout": (C.c_int, [vp, i32, C.c_uint32, vp, vp]),
        "kvmem_tree_workspace_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_mass_workspace_bytes": (sz, [cfgp, i32, i32, i32]),
        "kvmem_evict_workspace_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_view_tree_attend": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, vp, i32, vp, tailp, f32, vp, vp, vp, sz, vp]),
        "kvmem_paged_tree_attend": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, i32, vp, tailp, f32, vp, vp, vp, sz, vp]),
        "kvmem_view_attend_mass": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, i32, vp, tailp, f32, vp, f32, vp, vp, vp, sz, vp]),
        "kvmem_view_evict": (C.c_int, [vp, i32, vp, vp, i32, vp, vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, sz, vp]),
        "kvmem_rope_frequencies": (C.c_int, [cfgp, ropep, C.POINTER(C.c_double)]),
        "kvmem_set_rope": (C.c_int, [vp, ropep, vp]),
        "kvmem_rope_apply": (C.c_int, [vp, vp, i64, i64, i32, vp, i64, i64, i32, i64, i32, vp, i32, f32, vp]),
        "kvmem_rope_apply_call": (C.c_int, [vp]),
        "kvmem_reserve_blocks": (C.c_int, [vp, i32, i32, C.POINTER(i32), vp]),
        "kvmem_session_reserved": (i32, [vp, i32]),
        "kvmem_append_tokens": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, i32, vp]),
        "kvmem_append_tokens_call": (C.c_int, [vp]),
        "kvmem_commit_blocks": (C.c_int, [vp, i32, i32, C.POINTER(i32), tailp, vp]),
        "kvmem_prefill_workspace_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_view_prefill_attend": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, i32, vp, tailp, f32, vp, vp, vp, sz, vp]),
        "kvmem_get_pages": (C.c_int, [vp, C.POINTER(vp)]),
        "kvmem_step_staging_bytes": (sz, [cfgp, i32, i32]),
        "kvmem_recall_step_host": (C.c_int, [vp, i32, i32, vp, i32, prmp, vp, i32, vp, vp, vp, i32, f32, vp, vp,
                                             vp, sz, vp, sz, vp, sz, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    if path == _build.LIB_PATH:
        _lib = L
    return L


EXPORTED = ("kvmem_pool_bytes", "kvmem_budget_blocks", "kvmem_select_workspace_bytes",
            "kvmem_attend_workspace_bytes", "kvmem_last_error", "kvmem_pool_create", "kvmem_pool_destroy",
            "kvmem_session_reset", "kvmem_session_blocks", "kvmem_append_blocks", "kvmem_select",
            "kvmem_materialize", "kvmem_view_attend", "kvmem_get_index", "kvmem_get_block_table",
            "kvmem_device_status", "kvmem_set_option", "kvmem_step_staging_bytes", "kvmem_recall_step_host",
            "kvmem_view_attend_static", "kvmem_materialize_attend",
            "kvmem_paged_attend", "kvmem_append_blocks_rope", "kvmem_rope_rotate", "kvmem_materialize_rope",
            "kvmem_working_set_delta", "kvmem_score", "kvmem_view_cache_bytes", "kvmem_view_cache_layout",
            "kvmem_view_cache_reset", "kvmem_view_cache_update", "kvmem_view_cache_attend", "kvmem_paged_attend_rope", "kvmem_topk", "kvmem_score_host_workspace_bytes",
            "kvmem_score_host_staging_bytes", "kvmem_score_host_index", "kvmem_materialize_fp8", "kvmem_view_attend_fp8",
            "kvmem_materialize_attend_rope", "kvmem_paged_attend_fp8", "kvmem_materialize_attend_fp8",
            "kvmem_paged_attend_fp8_rope", "kvmem_selftest_wait_timeout", "kvmem_selftest_joint_wait_timeout", "kvmem_materialize_delta",
            "kvmem_materialize_fp8_rope", "kvmem_tree_workspace_bytes", "kvmem_view_tree_attend", "kvmem_paged_tree_attend",
            "kvmem_mass_workspace_bytes", "kvmem_view_attend_mass", "kvmem_evict_workspace_bytes", "kvmem_view_evict",
            "kvmem_rope_frequencies", "kvmem_set_rope", "kvmem_rope_apply", "kvmem_rope_apply_call", "kvmem_reserve_blocks", "kvmem_session_reserved",
            "kvmem_append_tokens", "kvmem_append_tokens_call", "kvmem_commit_blocks", "kvmem_prefill_workspace_bytes", "kvmem_view_prefill_attend", "kvmem_get_pages")


def _check(status: int) -> None:
    if status != OK:
        raise KvmemError(status, load_library().kvmem_last_error().decode())


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None)      # torch.cuda.is_current_stream_capturing; a build without CUDA has none


def _dev(t: torch.Tensor, dtype=None) -> int:
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _place(name: str, t: torch.Tensor, dtype, shape: tuple, device: int) -> int:
    """Pointer of a contiguous tensor of this dtype and shape on this device; ValueError for any other."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on cuda:{device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ' (strided)'}")
    return t.data_ptr()


# kvmem_append_call_t and kvmem_rope_call_t, packed into buffers that the pool keeps (building ctypes structures, or converting sixteen
# arguments, takes as long as the launch)
_APPEND, _ROPE = struct.Struct("PP" + 3 * "P4q" + "PP" + "PPiP" + "PP" + "5if"), struct.Struct("5P5q4if")
_NO_ROWS = (0, 0, 0, 0, 0)


def _rows(name: str, t: torch.Tensor, shape: tuple, device: int) -> tuple:
    """Pointer and strides of rows [n_sessions][n_tokens][L][heads][d] of any strides but the last: a slice of a packed projection, read
    where it lies."""
    st = t.stride()
    if t.dtype is not _BF16 or t.shape != shape or t.get_device() != device or st[4] != 1:
        raise ValueError(f"{name}: expected a bf16 tensor {tuple(shape)} on cuda:{device} with contiguous heads, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device} with strides {st}")
    return (t.data_ptr(), *st[:4])


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}
ORDERS = {"model": 0, "pool": 1}


def _one_of(name: str, value: str, choices: Dict[str, int]) -> int:
    if value not in choices:
        raise ValueError(f"{name}: expected one of {', '.join(choices)}, got {value!r}")
    return choices[value]


class HostStep:
    """kvmem_recall_step_host with its arguments checked and marshalled once; see Pool.host_step."""

    def __init__(self, pool, q_shape, params, sel_ids, n_sel, view, out_host, lse_host, scale, session_first):
        ns, M = q_shape[0], q_shape[1]
        for t, dt in ((out_host, torch.float32), (lse_host, torch.float32)):
            if t.is_cuda or not t.is_contiguous() or t.dtype != dt:
                raise ValueError("expected contiguous CPU tensors (fp32 outputs)")
        need = pool.lib.kvmem_step_staging_bytes(C.byref(pool.cfg), ns, M)
        if pool._staging is None or pool._staging.numel() < need:
            pool._staging = torch.empty(need, dtype=torch.uint8, device=pool.device)
        sws, aws = pool.select_workspace(ns, M), pool.attend_workspace(ns, M)
        self._keep = (pool, params, sel_ids, n_sel, view, out_host, lse_host, pool._staging, sws, aws)   # the buffers stay alive
        self._q_shape, self._fn = q_shape, pool.lib.kvmem_recall_step_host
        self._head = (pool.handle, session_first, ns)
        self._tail = (M, C.byref(params), _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                      _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16), view.cap_tokens, scale, out_host.data_ptr(),
                      lse_host.data_ptr(), pool._staging.data_ptr(), pool._staging.numel(), sws.data_ptr(), sws.numel(),
                      aws.data_ptr(), aws.numel())

    def __call__(self, q_host: torch.Tensor) -> None:
        if q_host.is_cuda or q_host.dtype != torch.bfloat16 or tuple(q_host.shape) != self._q_shape or not q_host.is_contiguous():
            raise ValueError("expected a contiguous CPU bf16 query of the planned shape")
        _check(self._fn(*self._head, q_host.data_ptr(), *self._tail, _stream()))


def budget_blocks(params: SelectParams, block_tokens: int, n_blocks: int) -> int:
    return int(load_library().kvmem_budget_blocks(C.byref(params), block_tokens, n_blocks))


def set_option(name: str, value: int) -> None:
    _check(load_library().kvmem_set_option(name.encode(), value))


@dataclass
class Rope:
    """Rotary form of a model (kvmem_rope_t): layout "half" or "interleaved", the dims that rotate (0: all), and how the
    frequencies are scaled for long contexts: "none", "linear", "base", "ramp" or "bands"."""
    layout: str = "half"
    rotary_dim: int = 0
    scaling: str = "none"
    factor: float = 1.0
    original_positions: float = 0.0
    turns_fast: float = 0.0
    turns_slow: float = 0.0

    def struct(self) -> RopeStruct:
        return RopeStruct(_one_of("layout", self.layout, ROPE_LAYOUTS), self.rotary_dim, _one_of("scaling", self.scaling, ROPE_SCALINGS),
                          self.factor, self.original_positions, self.turns_fast, self.turns_slow)


@dataclass
class Tail:
    """Tokens behind a view that fill no block yet: k, v bf16 [n_sessions][cap_tokens][L][G][d]; n_tokens int32
    [n_sessions] committed ones on the device, with the drafted tokens in the rows behind them."""
    k: torch.Tensor
    v: torch.Tensor
    n_tokens: torch.Tensor


@dataclass
class View:
    """Execution view buffers: bf16 [n_sessions][L][G][cap_tokens][d] each."""
    k: torch.Tensor
    v: torch.Tensor
    cap_tokens: int


class Pool:
    """A paged KV repository with its Mean-K index, living in one torch uint8 tensor."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, block_tokens: int,
                 max_sessions: int, max_blocks: int, max_blocks_per_session: int, device: int = 0,
                 rope_max_positions: int = 0, rope_theta: float = 0.0, rope_in_block_keys: bool = False,
                 fp8_pages: bool = False, fp8_k_scale: float = 1.0, fp8_v_scale: float = 1.0):
        self.lib = load_library()
        self.cfg = PoolConfig(n_layers, n_q_heads, n_kv_heads, head_dim, block_tokens, max_sessions, max_blocks,
                              max_blocks_per_session, device, rope_max_positions, rope_theta, int(rope_in_block_keys),
                              int(fp8_pages), fp8_k_scale, fp8_v_scale)
        nbytes = self.lib.kvmem_pool_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise KvmemError(E_INVALID, self.lib.kvmem_last_error().decode())
        self.device = torch.device("cuda", device)
        self.storage = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.handle = C.c_void_p()
        _check(self.lib.kvmem_pool_create(C.byref(self.cfg), self.storage.data_ptr(), nbytes, C.byref(self.handle)))
        self._select_ws: Optional[torch.Tensor] = None
        self._attend_ws: Optional[torch.Tensor] = None
        self._host_ws: Optional[torch.Tensor] = None
        self._host_staging: Optional[torch.Tensor] = None
        self._staging: Optional[torch.Tensor] = None
        self._index = device
        self._dims = (n_layers, n_q_heads, n_kv_heads, head_dim)
        self._decode_ws: Optional[torch.Tensor] = None
        self._decode_at: Tuple[int, int] = (0, 0)                      # its pointer and bytes
        self._decode_stream = 0                                        # the stream it was made on
        self._decode_pinned = False                                    # a captured graph or another stream may still write it
        self._decode_kept: List[torch.Tensor] = []                     # smaller ones of which that holds
        self._decode_need: Dict[tuple, int] = {}
        self._append_buf, self._rope_buf = C.create_string_buffer(_APPEND.size), C.create_string_buffer(_ROPE.size)
        self._append_at, self._rope_at = C.addressof(self._append_buf), C.addressof(self._rope_buf)

    # ---- lifetime
    def close(self) -> None:
        """The work of this pool must be over, and no captured graph of it is replayed any more: its workspaces are given back."""
        if self.handle:
            self.lib.kvmem_pool_destroy(self.handle)
            self.handle = C.c_void_p()
            self._decode_ws, self._decode_at, self._decode_pinned = None, (0, 0), False
            self._decode_kept.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- repository
    def session_reset(self, session: int) -> None:
        _check(self.lib.kvmem_session_reset(self.handle, session, _stream()))

    def session_blocks(self, session: int) -> int:
        n = self.lib.kvmem_session_blocks(self.handle, session)
        if n < 0:
            _check(n)
        return n

    def append_blocks(self, session: int, k: torch.Tensor, v: torch.Tensor,
                      phys_ids: Optional[Sequence[int]] = None) -> None:
        c = self.cfg
        per_block = c.block_tokens * c.n_layers * c.n_kv_heads * c.head_dim
        if k.numel() % per_block or k.shape != v.shape:
            raise KvmemError(E_INVALID, "k and v must hold whole blocks of identical shape")
        n = k.numel() // per_block
        ids = None
        if phys_ids is not None:
            if len(phys_ids) != n:
                raise KvmemError(E_INVALID, "one page id per block")
            ids = (C.c_int32 * n)(*[int(x) for x in phys_ids])
        _check(self.lib.kvmem_append_blocks(self.handle, session, _dev(k, torch.bfloat16), _dev(v, torch.bfloat16),
                                            n, ids, _stream()))

    # ---- working-set delta
    def working_set_delta(self, prev_ids: torch.Tensor, n_prev: torch.Tensor, next_ids: torch.Tensor,
                          n_next: torch.Tensor):
        """Retained / incoming / outgoing blocks between two selections (ascending int32 id lists of equal stride).
        Returns (retained [ns][stride][3], incoming [ns][stride][2], outgoing [ns][stride], counts [ns][3])."""
        ns, stride = prev_ids.shape
        if next_ids.shape != prev_ids.shape:
            raise ValueError("both id lists must have the same [n_sessions][stride] shape")
        dev = prev_ids.device
        ret = torch.zeros(ns, stride, 3, dtype=torch.int32, device=dev)
        inc = torch.zeros(ns, stride, 2, dtype=torch.int32, device=dev)
        out = torch.zeros(ns, stride, dtype=torch.int32, device=dev)
        cnt = torch.zeros(ns, 3, dtype=torch.int32, device=dev)
        _check(self.lib.kvmem_working_set_delta(self.handle, ns, _dev(prev_ids, torch.int32), _dev(n_prev, torch.int32),
                                                _dev(next_ids, torch.int32), _dev(n_next, torch.int32), stride,
                                                ret.data_ptr(), inc.data_ptr(), out.data_ptr(), cnt.data_ptr(), _stream()))
        return ret, inc, out, cnt

    # ---- execution cache: working-set reuse with bounded delta re-RoPE
    def new_view_cache(self, cap_blocks: int, max_delta_ropes: int, first_position: int = 0) -> "ViewCache":
        return ViewCache(self, cap_blocks, max_delta_ropes, first_position)

    # ---- position-consistent keys
    def append_blocks_rope(self, session: int, k_roped: torch.Tensor, v: torch.Tensor, block_pos0: Sequence[int],
                           phys_ids: Optional[Sequence[int]] = None) -> None:
        """append_blocks for keys that carry RoPE: token t of block i was encoded at block_pos0[i] + t."""
        c = self.cfg
        per_block = c.block_tokens * c.n_layers * c.n_kv_heads * c.head_dim
        if k_roped.numel() % per_block or k_roped.shape != v.shape:
            raise KvmemError(E_INVALID, "k and v must hold whole blocks of identical shape")
        n = k_roped.numel() // per_block
        if len(block_pos0) != n or (phys_ids is not None and len(phys_ids) != n):
            raise KvmemError(E_INVALID, "one position (and page id) per block")
        ids = None if phys_ids is None else (C.c_int32 * n)(*[int(x) for x in phys_ids])
        pos = (C.c_int32 * n)(*[int(x) for x in block_pos0])
        _check(self.lib.kvmem_append_blocks_rope(self.handle, session, _dev(k_roped, torch.bfloat16),
                                                 _dev(v, torch.bfloat16), n, ids, pos, _stream()))

    def rope_rotate(self, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None,
                    inverse: bool = False) -> torch.Tensor:
        """x bf16 [n_rows][n_vec][head_dim], positions int32 [n_rows] -> rotated copy (inverse: encoding removed)."""
        if out is None:
            out = torch.empty_like(x)
        n_rows, n_vec = x.shape[0], x.numel() // (x.shape[0] * self.cfg.head_dim)
        _check(self.lib.kvmem_rope_rotate(self.handle, _dev(x, torch.bfloat16), _dev(out, torch.bfloat16), n_rows, n_vec,
                                          _dev(positions, torch.int32), int(inverse), _stream()))
        return out

    def materialize_rope(self, sel_ids: torch.Tensor, n_sel: torch.Tensor, view: View, first_position: int = 0,
                         session_first: int = 0) -> None:
        """materialize with keys rotated to their compact positions first_position + j*B + t; values copied."""
        ns = n_sel.shape[0]
        _check(self.lib.kvmem_materialize_rope(self.handle, session_first, ns, _dev(sel_ids, torch.int32),
                                               sel_ids.shape[-1], _dev(n_sel, torch.int32), _dev(view.k, torch.bfloat16),
                                               _dev(view.v, torch.bfloat16), view.cap_tokens, first_position, _stream()))

    # ---- the recall step
    def select_workspace(self, n_sessions: int, n_q_tokens: int) -> torch.Tensor:
        need = self.lib.kvmem_select_workspace_bytes(C.byref(self.cfg), n_sessions, n_q_tokens)
        if need == 0:
            raise KvmemError(E_INVALID, self.lib.kvmem_last_error().decode())
        if self._select_ws is None or self._select_ws.numel() < need:
            self._select_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._select_ws

    def attend_workspace(self, n_sessions: int, n_q_tokens: int) -> torch.Tensor:
        need = self.lib.kvmem_attend_workspace_bytes(C.byref(self.cfg), n_sessions, n_q_tokens)
        if need == 0:
            raise KvmemError(E_INVALID, self.lib.kvmem_last_error().decode())
        if self._attend_ws is None or self._attend_ws.numel() < need:
            self._attend_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._attend_ws

    def score(self, q: torch.Tensor, scores: torch.Tensor, session_first: int = 0, score_scale: float = 1.0) -> None:
        """Block relevance only: q bf16 [n_sessions][M][L][H][d] -> scores fp32 [n_sessions][max_blocks_per_session]
        (times score_scale: a rank holding 1/N of a session's heads passes 1/N, so that the ranks' outputs sum to R)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.select_workspace(ns, M)
        _check(self.lib.kvmem_score(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                    _dev(scores, torch.float32), score_scale, ws.data_ptr(), ws.numel(), _stream()))

    def topk(self, scores: torch.Tensor, params: SelectParams, sel_ids: torch.Tensor, n_sel: torch.Tensor,
             session_first: int = 0) -> None:
        """Selection from scores the caller already has: scores fp32 [n_sessions][stride] on the device."""
        ns = scores.shape[0]
        _check(self.lib.kvmem_topk(self.handle, session_first, ns, _dev(scores, torch.float32), scores.shape[1],
                                   C.byref(params), _dev(sel_ids, torch.int32), sel_ids.shape[-1],
                                   _dev(n_sel, torch.int32), _stream()))

    def score_host_index(self, index_host: torch.Tensor, n_blocks: int, q: torch.Tensor, scores: torch.Tensor,
                         tile_blocks: int = 4096) -> None:
        """Block relevance against an index in HOST memory (bf16 [L][G][stride][d], ideally pinned), streamed to the
        GPU in tiles of tile_blocks blocks; q bf16 [M][L][H][d] and scores fp32 [n_blocks] on the device."""
        if index_host.is_cuda or index_host.dtype != torch.bfloat16 or not index_host.is_contiguous():
            raise ValueError("index_host must be a contiguous CPU bf16 tensor")
        M = q.shape[0]
        need_ws = self.lib.kvmem_score_host_workspace_bytes(self.handle, n_blocks, M, tile_blocks)
        need_st = self.lib.kvmem_score_host_staging_bytes(self.handle, tile_blocks)
        if need_ws == 0 or need_st == 0:
            raise KvmemError(E_INVALID, self.lib.kvmem_last_error().decode())
        if self._host_ws is None or self._host_ws.numel() < need_ws:
            self._host_ws = torch.empty(need_ws, dtype=torch.uint8, device=self.device)
        if self._host_staging is None or self._host_staging.numel() < need_st:
            self._host_staging = torch.empty(need_st, dtype=torch.uint8, device=self.device)
        _check(self.lib.kvmem_score_host_index(self.handle, index_host.data_ptr(), n_blocks, index_host.shape[2],
                                               _dev(q, torch.bfloat16), M, tile_blocks, _dev(scores, torch.float32),
                                               self._host_staging.data_ptr(), self._host_staging.numel(),
                                               self._host_ws.data_ptr(), self._host_ws.numel(), _stream()))

    def select(self, q: torch.Tensor, params: SelectParams, sel_ids: torch.Tensor, n_sel: torch.Tensor,
               scores: Optional[torch.Tensor] = None, session_first: int = 0) -> None:
        """q bf16 [n_sessions][M][L][H][d]; sel_ids int32 [n_sessions][stride]; n_sel int32 [n_sessions]."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.select_workspace(ns, M)
        _check(self.lib.kvmem_select(self.handle, session_first, ns, _dev(q, torch.bfloat16), M, C.byref(params),
                                     _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                     None if scores is None else _dev(scores, torch.float32),
                                     ws.data_ptr(), ws.numel(), _stream()))

    def materialize(self, sel_ids: torch.Tensor, n_sel: torch.Tensor, view: View, session_first: int = 0) -> None:
        ns = n_sel.shape[0]
        _check(self.lib.kvmem_materialize(self.handle, session_first, ns, _dev(sel_ids, torch.int32),
                                          sel_ids.shape[-1], _dev(n_sel, torch.int32), _dev(view.k, torch.bfloat16),
                                          _dev(view.v, torch.bfloat16), view.cap_tokens, _stream()))

    def materialize_delta(self, prev_ids: torch.Tensor, n_prev: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor,
                          view: View, stats: Optional[torch.Tensor] = None, session_first: int = 0) -> None:
        """Move a view built from prev_ids to sel_ids: slots whose block stays are not touched, the others are fetched.
        stats int32 [n_sessions][3] (optional) receives (unchanged, retained and moved, incoming) per session."""
        ns = n_sel.shape[0]
        if prev_ids.shape != sel_ids.shape:
            raise ValueError("both id lists must have the same [n_sessions][stride] shape")
        _check(self.lib.kvmem_materialize_delta(self.handle, session_first, ns, _dev(prev_ids, torch.int32), _dev(n_prev, torch.int32),
                                                _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16), view.cap_tokens,
                                                None if stats is None else _dev(stats, torch.int32), _stream()))

    def view_attend(self, q: torch.Tensor, view: View, n_sel: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                    scale: float = 0.0) -> None:
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_view_attend(self.handle, ns, _dev(q, torch.bfloat16), M, _dev(view.k, torch.bfloat16),
                                          _dev(view.v, torch.bfloat16), view.cap_tokens, _dev(n_sel, torch.int32),
                                          scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                          ws.data_ptr(), ws.numel(), _stream()))

    # ---- decode over a view: drafted tokens, accumulated weights, eviction
    # These calls run once per decoded token, on views that may take a few microseconds: their checks are kept short.
    def _decode_workspace(self, workspace: Optional[torch.Tensor], stream: int, *key) -> Tuple[Optional[int], int]:
        """The caller's tensor, or the pool's own of kvmem_<key[0]>_workspace_bytes(cfg, *key[1:]) bytes.  A size that has none goes to
        the call without a workspace: it is refused there, with its own status."""
        if workspace is not None:
            return _place("workspace", workspace, torch.uint8, (workspace.numel(),), self._index), workspace.numel()
        need = self._decode_need.get(key)
        if need is None:
            need = getattr(self.lib, f"kvmem_{key[0]}_workspace_bytes")(C.byref(self.cfg), *key[1:])
            if need == 0:
                return None, 0
            self._decode_need[key] = need
        if self._decode_at[1] < need:
            self._grow_decode_workspace(need, stream)
        # (the default stream, 0, cannot be captured: calls on it need not ask)
        if not self._decode_pinned and (stream != self._decode_stream or (stream != 0 and _capturing())):
            self._decode_pinned = True
        return self._decode_at

    def _grow_decode_workspace(self, need: int, stream: int) -> None:
        # One that only calls of its own stream used goes back to the allocator, which hands it out in that stream's order.  One that a
        # captured graph replays on or another stream used is kept; small ones then at least double, so that what is kept stays little.
        size = need
        if self._decode_pinned:
            self._decode_kept.append(self._decode_ws)
            if 2 * self._decode_at[1] <= 64 << 20:
                size = max(need, 2 * self._decode_at[1])
        self._decode_ws, self._decode_at, self._decode_pinned = None, (0, 0), False
        ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        self._decode_ws, self._decode_at, self._decode_stream = ws, (ws.data_ptr(), size), stream

    def _decode_common(self, q, n_sel, tail, out, lse, n_q):
        L, H, G, d = self._dims
        dev, bf16, i32 = self._index, torch.bfloat16, torch.int32
        if q.dim() != 5:
            raise ValueError("q: expected [n_sessions][n_q_tokens][L][H][d]")
        ns, M, _, _, _ = q.shape
        shape, per_session = (ns, M, L, H, d), (ns,)
        qp = _place("q", q, bf16, shape, dev)
        np_ = _place("n_sel", n_sel, i32, per_session, dev)
        op, lp = _place("out", out, bf16, shape, dev), _place("lse", lse, torch.float32, (ns, M, L, H), dev)
        nq = None if n_q is None else _place("n_q", n_q, i32, per_session, dev)
        tp = None
        if tail is not None:
            tk = tail.k
            cap = tk.shape[1] if tk.dim() == 5 else -1
            ts = (ns, cap, L, G, d)
            tp = TailStruct(_place("tail.k", tk, bf16, ts, dev), _place("tail.v", tail.v, bf16, ts, dev), cap,
                            _place("tail.n_tokens", tail.n_tokens, i32, per_session, dev))
        return ns, M, qp, np_, tp, op, lp, nq

    def _view_of(self, name: str, view: View, ns: int) -> Tuple[int, int, int]:
        L, _, G, d = self._dims
        cap = view.cap_tokens
        shape = (ns, L, G, cap, d)
        return _place(name, view.k, torch.bfloat16, shape, self._index), _place(name, view.v, torch.bfloat16, shape, self._index), cap

    def _raw_stream(self) -> int:
        return torch._C._cuda_getCurrentRawStream(self._index)

    def view_tree_attend(self, q: torch.Tensor, view: View, n_sel: torch.Tensor, tail: Optional[Tail], out: torch.Tensor,
                         lse: torch.Tensor, mask: Optional[torch.Tensor] = None, n_q: Optional[torch.Tensor] = None,
                         scale: float = 0.0, workspace: Optional[torch.Tensor] = None) -> None:
        """Attention of up to 64 drafted tokens per session over view and tail: q bf16 [n_sessions][M][L][H][d], mask
        int64 [n_sessions][M] (bit j of word i: token i sees drafted token j; None: a chain), n_q int32 [n_sessions]
        drafted tokens in use, out bf16 like q, lse fp32 [n_sessions][M][L][H].  Calls that may overlap on the GPU (other
        streams, other captured graphs) need a workspace each (kvmem_tree_workspace_bytes); None: the pool's own."""
        ns, M, qp, np_, tp, op, lp, nq = self._decode_common(q, n_sel, tail, out, lse, n_q)
        vk, vv, cap = self._view_of("view", view, ns)
        mp = None if mask is None else _place("mask", mask, torch.int64, (ns, M), self._index)
        st = self._raw_stream()
        wp, wn = self._decode_workspace(workspace, st, "tree", ns, M)
        _check(self.lib.kvmem_view_tree_attend(self.handle, ns, qp, M, nq, mp, vk, vv, cap, np_, tp, scale, op, lp, wp, wn, st))

    def paged_tree_attend(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, tail: Optional[Tail],
                          out: torch.Tensor, lse: torch.Tensor, mask: Optional[torch.Tensor] = None,
                          n_q: Optional[torch.Tensor] = None, scale: float = 0.0, session_first: int = 0,
                          workspace: Optional[torch.Tensor] = None) -> None:
        """view_tree_attend straight over the selected blocks' pages: sel_ids int32 [n_sessions][stride].  Stored keys as they lie: where
        keys carry positions, materialize_rope and view_tree_attend (a pool with rope_in_block_keys is refused)."""
        ns, M, qp, np_, tp, op, lp, nq = self._decode_common(q, n_sel, tail, out, lse, n_q)
        sp = _place("sel_ids", sel_ids, torch.int32, (ns, sel_ids.shape[-1]), self._index)
        mp = None if mask is None else _place("mask", mask, torch.int64, (ns, M), self._index)
        st = self._raw_stream()
        wp, wn = self._decode_workspace(workspace, st, "tree", ns, M)
        _check(self.lib.kvmem_paged_tree_attend(self.handle, session_first, ns, qp, M, nq, mp, sp, sel_ids.shape[-1], np_, tp,
                                                scale, op, lp, wp, wn, st))

    def view_attend_mass(self, q: torch.Tensor, view: View, n_sel: torch.Tensor, mass: torch.Tensor, out: torch.Tensor,
                         lse: torch.Tensor, tail: Optional[Tail] = None, n_q: Optional[torch.Tensor] = None, decay: float = 1.0,
                         scale: float = 0.0, workspace: Optional[torch.Tensor] = None) -> None:
        """view_tree_attend for a chain that also sets mass fp32 [n_sessions][L][G][cap_tokens] to decay * mass + the
        attention weight of each view token, summed over the query rows of its KV head (n_q_tokens * H/G <= 64)."""
        L, _, G, _ = self._dims
        ns, M, qp, np_, tp, op, lp, nq = self._decode_common(q, n_sel, tail, out, lse, n_q)
        vk, vv, cap = self._view_of("view", view, ns)
        ap = _place("mass", mass, torch.float32, (ns, L, G, cap), self._index)
        st = self._raw_stream()
        wp, wn = self._decode_workspace(workspace, st, "mass", ns, M, cap)
        _check(self.lib.kvmem_view_attend_mass(self.handle, ns, qp, M, nq, vk, vv, cap, np_, tp, scale, ap, decay, op, lp, wp, wn,
                                               st))

    def view_evict(self, view: View, n_sel: torch.Tensor, mass: torch.Tensor, dst: View, n_sel_out: torch.Tensor,
                   dst_mass: torch.Tensor, kept: Optional[torch.Tensor] = None, keep_blocks: Optional[int] = None,
                   n_sink_tokens: int = 0, n_recent_tokens: int = 0, workspace: Optional[torch.Tensor] = None) -> None:
        """Keep the keep_blocks (default: dst's capacity) * block_tokens tokens of each KV head with the largest mass,
        the first n_sink_tokens and last n_recent_tokens among them, and move them in order to dst; n_sel_out int32
        [n_sessions] receives dst's lengths in blocks, kept int32 [n_sessions][L][G][keep_blocks * B] the tokens' places."""
        L, _, G, _ = self._dims
        B = self.cfg.block_tokens
        ns = n_sel.shape[0]
        keep = dst.cap_tokens // B if keep_blocks is None else keep_blocks
        vk, vv, cap = self._view_of("view", view, ns)
        dk, dv, dcap = self._view_of("dst", dst, ns)
        heads = (ns, L, G)
        ap, dp = _place("mass", mass, torch.float32, (*heads, cap), self._index), _place("dst_mass", dst_mass, torch.float32, (*heads, dcap), self._index)
        kp = None if kept is None else _place("kept", kept, torch.int32, (*heads, keep * B), self._index)
        np_, no = _place("n_sel", n_sel, torch.int32, (ns,), self._index), _place("n_sel_out", n_sel_out, torch.int32, (ns,), self._index)
        st = self._raw_stream()
        wp, wn = self._decode_workspace(workspace, st, "evict", ns, keep)
        _check(self.lib.kvmem_view_evict(self.handle, ns, vk, vv, cap, np_, ap, keep, n_sink_tokens, n_recent_tokens, dk, dv, dcap,
                                         dp, kp, no, wp, wn, st))

    # ---- new tokens: rotary forms, tail and pages, prompt chunks
    def rope_frequencies(self, rope: Optional[Rope] = None) -> List[float]:
        """Radians per position of the pairs (i, i + d/2) in the pool's order; 0 where dims pass."""
        f = (C.c_double * (self.cfg.head_dim // 2))()
        _check(self.lib.kvmem_rope_frequencies(C.byref(self.cfg), None if rope is None else C.byref(rope.struct()), f))
        return list(f)

    def set_rope(self, rope: Optional[Rope] = None) -> None:
        """Make this the pool of a model with this rotary form (None: the pool's own), before any block comes in."""
        _check(self.lib.kvmem_set_rope(self.handle, None if rope is None else C.byref(rope.struct()), self._raw_stream()))

    def rope_apply(self, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None, inverse: bool = False,
                   amplitude: float = 1.0, x_order: str = "model", out_order: str = "pool") -> torch.Tensor:
        """x bf16 [n_rows][n_vec][head_dim] (rows and vectors strided as they lie), positions int32 [n_rows] -> rotated vectors,
        "model" or "pool" order of the dims on either side; out may be x if the orders are the same."""
        d, dev = self._dims[3], self._index
        shape = x.shape
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=x.device)
        xs, ys = x.stride(), out.stride()
        if (len(shape) != 3 or shape[2] != d or out.shape != shape or x.dtype is not _BF16 or out.dtype is not _BF16 or x.get_device() != dev or
                out.get_device() != dev or xs[2] != 1 or ys[2] != 1):
            raise ValueError(f"x, out: expected bf16 tensors [n_rows][n_vec][{d}] on cuda:{dev} with contiguous vectors, got {x.dtype} "
                             f"{tuple(shape)} on {x.device} with strides {xs}, {out.dtype} {tuple(out.shape)} on {out.device} with strides {ys}")
        n_rows, n_vec, _ = shape
        pp = _place("positions", positions, _I32, (n_rows,), dev)
        xo, yo = _one_of("x_order", x_order, ORDERS), _one_of("out_order", out_order, ORDERS)
        if n_rows and n_vec:
            _ROPE.pack_into(self._rope_buf, 0, self.handle.value or 0, x.data_ptr(), out.data_ptr(), pp, self._raw_stream(), n_rows, xs[0], xs[1],
                            ys[0], ys[1], n_vec, xo, yo, bool(inverse), amplitude)
            rc = self.lib.kvmem_rope_apply_call(self._rope_at)
            if rc:
                _check(rc)
        return out

    def reserve_blocks(self, session: int, n_blocks: int, phys_ids: Optional[Sequence[int]] = None) -> None:
        """Pages for n_blocks blocks behind the session's last, to be filled by append_tokens(pages=True)."""
        if phys_ids is not None and len(phys_ids) != n_blocks:
            raise KvmemError(E_INVALID, "one page id per block")
        ids = None if phys_ids is None else (C.c_int32 * n_blocks)(*[int(x) for x in phys_ids])
        _check(self.lib.kvmem_reserve_blocks(self.handle, session, n_blocks, ids, self._raw_stream()))

    def session_reserved(self, session: int) -> int:
        n = self.lib.kvmem_session_reserved(self.handle, session)
        if n < 0:
            _check(n)
        return n

    def _tail_struct(self, tail: Tail, ns: int) -> TailStruct:
        L, _, G, d = self._dims
        tk, dev = tail.k, self._index
        cap = tk.shape[1] if tk.dim() == 5 else -1
        shape = (ns, cap, L, G, d)
        return TailStruct(_place("tail.k", tk, _BF16, shape, dev), _place("tail.v", tail.v, _BF16, shape, dev), cap,
                          _place("tail.n_tokens", tail.n_tokens, _I32, (ns,), dev))

    def append_tokens(self, k: torch.Tensor, v: torch.Tensor, tail: Tail, q: Optional[torch.Tensor] = None,
                      q_out: Optional[torch.Tensor] = None, n_new: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                      n_sel: Optional[torch.Tensor] = None, first_position: int = 0, q_amplitude: float = 1.0, pages: bool = False,
                      session_first: int = 0) -> None:
        """New tokens behind the tail's committed ones: q bf16 [n_sessions][M][L][H][d] (optional, with q_out of that shape), k, v
        [n_sessions][M][L][G][d], strided as they lie.  Rotated queries go to q_out, rotated keys and values to the tail, with pages
        raw keys and values to the reserved pages as well.  Positions are positions int32 [n_sessions][M], or first_position +
        n_sel * block_tokens + the tail's row; what the tail holds already stays where it is (see commit_blocks)."""
        L, H, G, d = self._dims
        dev = self._index
        shape = k.shape
        if len(shape) != 5:
            raise ValueError("k: expected [n_sessions][n_new_tokens][L][G][d]")
        ns, M, _, _, _ = shape
        kv, qs, per_session = (ns, M, L, G, d), (ns, M, L, H, d), (ns,)
        tk = tail.k
        cap = tk.shape[1] if tk.dim() == 5 else -1
        ts = (ns, cap, L, G, d)
        _APPEND.pack_into(
            self._append_buf, 0, self.handle.value or 0, 0 if n_new is None else _place("n_new", n_new, _I32, per_session, dev),
            *(_NO_ROWS if q is None else _rows("q", q, qs, dev)), *_rows("k", k, kv, dev), *_rows("v", v, kv, dev),
            0 if positions is None else _place("positions", positions, _I32, (ns, M), dev),
            0 if n_sel is None else _place("n_sel", n_sel, _I32, per_session, dev),
            _place("tail.k", tk, _BF16, ts, dev), _place("tail.v", tail.v, _BF16, ts, dev), cap,
            _place("tail.n_tokens", tail.n_tokens, _I32, per_session, dev), 0 if q_out is None else _place("q_out", q_out, _BF16, qs, dev),
            self._raw_stream(), session_first, ns, M, first_position, bool(pages), q_amplitude)
        rc = self.lib.kvmem_append_tokens_call(self._append_at)
        if rc:
            _check(rc)

    def commit_blocks(self, n_blocks: Sequence[int], tail: Optional[Tail] = None, session_first: int = 0) -> None:
        """The first n_blocks[s] reserved blocks of each session become part of it, with their index rows; the tail's rows behind
        them move to its front, their keys at the positions that they had.  Before the next append or attention: a view that has grown by
        these blocks, or a first_position that has grown by their tokens, or keys brought to their new positions by rope_apply in the
        "pool" order or by appending them again (kvmem_commit_blocks in the header)."""
        ns = len(n_blocks)
        ts = None if tail is None else self._tail_struct(tail, ns)
        _check(self.lib.kvmem_commit_blocks(self.handle, session_first, ns, (C.c_int32 * max(ns, 1))(*[int(x) for x in n_blocks]), ts,
                                            self._raw_stream()))

    def view_prefill_attend(self, q: torch.Tensor, view: View, n_sel: torch.Tensor, tail: Optional[Tail], out: torch.Tensor,
                            lse: torch.Tensor, n_q: Optional[torch.Tensor] = None, scale: float = 0.0,
                            workspace: Optional[torch.Tensor] = None) -> None:
        """view_tree_attend for a prompt chunk of any length: token i sees the view, the committed tail and the chunk's tokens 0 .. i.
        Calls that may overlap on the GPU need a workspace each (kvmem_prefill_workspace_bytes); None: the pool's own."""
        ns, M, qp, np_, tp, op, lp, nq = self._decode_common(q, n_sel, tail, out, lse, n_q)
        vk, vv, cap = self._view_of("view", view, ns)
        st = self._raw_stream()
        wp, wn = self._decode_workspace(workspace, st, "prefill", ns, M)
        _check(self.lib.kvmem_view_prefill_attend(self.handle, ns, qp, M, nq, vk, vv, cap, np_, tp, scale, op, lp, wp, wn, st))

    def materialize_attend(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, view: View,
                           out: torch.Tensor, lse: torch.Tensor, scale: float = 0.0, session_first: int = 0) -> None:
        """materialize + view_attend in one pass over the selected blocks (same results, a third less HBM traffic)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_materialize_attend(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                                 _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                 _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16),
                                                 view.cap_tokens, scale, _dev(out, torch.float32),
                                                 _dev(lse, torch.float32), ws.data_ptr(), ws.numel(), _stream()))

    def paged_attend(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, out: torch.Tensor,
                     lse: torch.Tensor, scale: float = 0.0, session_first: int = 0) -> None:
        """Copy-free execution view: attention straight over the selected blocks' pages (no view written)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_paged_attend(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                           _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                           scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                           ws.data_ptr(), ws.numel(), _stream()))

    def paged_attend_rope(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, out: torch.Tensor,
                          lse: torch.Tensor, first_position: int = 0, scale: float = 0.0, session_first: int = 0) -> None:
        """Copy-free view with position-consistent keys: raw key tiles are RoPE'd in shared memory on their way
        to the tensor cores (same results as materialize_rope + view_attend, no view written)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_paged_attend_rope(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                                _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                first_position, scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                                ws.data_ptr(), ws.numel(), _stream()))

    def materialize_attend_rope(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, view: View,
                                out: torch.Tensor, lse: torch.Tensor, first_position: int = 0, scale: float = 0.0,
                                session_first: int = 0) -> None:
        """materialize_rope + view_attend in one call (one pass on a pool with the in-block key layout)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_materialize_attend_rope(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                                      _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                      _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16),
                                                      view.cap_tokens, first_position, scale, _dev(out, torch.float32),
                                                      _dev(lse, torch.float32), ws.data_ptr(), ws.numel(), _stream()))

    # ---- FP8 (E4M3) execution view
    def new_view_fp8(self, n_sessions: int, cap_tokens: int) -> Tuple[torch.Tensor, torch.Tensor]:
        """(keys uint8 [ns][L][G][cap][d], values uint8 [ns][L][G][cap/64][d][64]) for materialize_fp8."""
        c = self.cfg
        k8 = torch.zeros(n_sessions, c.n_layers, c.n_kv_heads, cap_tokens, c.head_dim, dtype=torch.uint8, device=self.device)
        v8t = torch.zeros(n_sessions, c.n_layers, c.n_kv_heads, cap_tokens // 64, c.head_dim, 64, dtype=torch.uint8,
                          device=self.device)
        return k8, v8t

    def materialize_fp8(self, sel_ids: torch.Tensor, n_sel: torch.Tensor, k8: torch.Tensor, v8t: torch.Tensor,
                        k_scale: float = 1.0, v_scale: float = 1.0, session_first: int = 0) -> None:
        ns = sel_ids.shape[0]
        _check(self.lib.kvmem_materialize_fp8(self.handle, session_first, ns, _dev(sel_ids, torch.int32), sel_ids.shape[-1],
                                              _dev(n_sel, torch.int32), _dev(k8, torch.uint8), _dev(v8t, torch.uint8),
                                              k8.shape[3], k_scale, v_scale, _stream()))

    def materialize_fp8_rope(self, sel_ids: torch.Tensor, n_sel: torch.Tensor, k8: torch.Tensor, v8t: torch.Tensor,
                             first_position: int = 0, k_scale: float = 1.0, v_scale: float = 1.0, session_first: int = 0) -> None:
        """Position-consistent FP8 view: keys rotated to their compact positions, then quantised; values as materialize_fp8."""
        ns = sel_ids.shape[0]
        _check(self.lib.kvmem_materialize_fp8_rope(self.handle, session_first, ns, _dev(sel_ids, torch.int32), sel_ids.shape[-1],
                                                   _dev(n_sel, torch.int32), _dev(k8, torch.uint8), _dev(v8t, torch.uint8),
                                                   k8.shape[3], first_position, k_scale, v_scale, _stream()))

    def view_attend_fp8(self, q: torch.Tensor, k8: torch.Tensor, v8t: torch.Tensor, n_sel: torch.Tensor, out: torch.Tensor,
                        lse: torch.Tensor, k_scale: float = 1.0, v_scale: float = 1.0, scale: float = 0.0) -> None:
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_view_attend_fp8(self.handle, ns, _dev(q, torch.bfloat16), M, _dev(k8, torch.uint8),
                                              _dev(v8t, torch.uint8), k8.shape[3], _dev(n_sel, torch.int32), scale, k_scale,
                                              v_scale, _dev(out, torch.float32), _dev(lse, torch.float32), ws.data_ptr(),
                                              ws.numel(), _stream()))

    def paged_attend_fp8(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, out: torch.Tensor,
                         lse: torch.Tensor, scale: float = 0.0, session_first: int = 0) -> None:
        """Copy-free view over an FP8 repository (pool created with fp8_pages): attention straight over the pages."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_paged_attend_fp8(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                               _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                               scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                               ws.data_ptr(), ws.numel(), _stream()))

    def paged_attend_fp8_rope(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, out: torch.Tensor,
                              lse: torch.Tensor, first_position: int = 0, scale: float = 0.0, session_first: int = 0) -> None:
        """Copy-free, position-consistent attention over an FP8 repository of in-block-rotated keys: the query is rotated
        back once per block (pool created with fp8_pages and rope_in_block_keys)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_paged_attend_fp8_rope(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                                    _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                    first_position, scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                                    ws.data_ptr(), ws.numel(), _stream()))

    def materialize_attend_fp8(self, q: torch.Tensor, sel_ids: torch.Tensor, n_sel: torch.Tensor, k8: torch.Tensor,
                               v8t: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, scale: float = 0.0,
                               session_first: int = 0) -> None:
        """materialize_fp8 + view_attend_fp8 in one pass over an FP8 repository (pool created with fp8_pages)."""
        ns, M = q.shape[0], q.shape[1]
        ws = self.attend_workspace(ns, M)
        _check(self.lib.kvmem_materialize_attend_fp8(self.handle, session_first, ns, _dev(q, torch.bfloat16), M,
                                                     _dev(sel_ids, torch.int32), sel_ids.shape[-1], _dev(n_sel, torch.int32),
                                                     _dev(k8, torch.uint8), _dev(v8t, torch.uint8), k8.shape[3], scale,
                                                     _dev(out, torch.float32), _dev(lse, torch.float32),
                                                     ws.data_ptr(), ws.numel(), _stream()))

    def view_attend_static(self, q: torch.Tensor, view: View, n_sel: torch.Tensor, out: torch.Tensor,
                           lse: torch.Tensor, scale: float = 0.0) -> None:
        """view_attend without a caller workspace, for hosts that cannot allocate device memory: the
        split-K scratch is a fixed array inside the library (at most 8 (session, layer, KV head)
        triples per call; calls that overlap on the GPU race on it)."""
        ns, M = q.shape[0], q.shape[1]
        _check(self.lib.kvmem_view_attend_static(self.handle, ns, _dev(q, torch.bfloat16), M,
                                                 _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16),
                                                 view.cap_tokens, _dev(n_sel, torch.int32), scale,
                                                 _dev(out, torch.float32), _dev(lse, torch.float32), _stream()))

    def recall_step_host(self, q_host: torch.Tensor, params: SelectParams, sel_ids: torch.Tensor,
                         n_sel: torch.Tensor, view: View, out_host: torch.Tensor, lse_host: torch.Tensor,
                         scale: float = 0.0, session_first: int = 0) -> None:
        """Whole step with HOST query and results (the library does the copies and waits for the stream)."""
        ns, M = q_host.shape[0], q_host.shape[1]
        for t, dt in ((q_host, torch.bfloat16), (out_host, torch.float32), (lse_host, torch.float32)):
            if t.is_cuda or not t.is_contiguous() or t.dtype != dt:
                raise ValueError("expected contiguous CPU tensors (bf16 query, fp32 outputs)")
        need = self.lib.kvmem_step_staging_bytes(C.byref(self.cfg), ns, M)
        if self._staging is None or self._staging.numel() < need:
            self._staging = torch.empty(need, dtype=torch.uint8, device=self.device)
        sws, aws = self.select_workspace(ns, M), self.attend_workspace(ns, M)
        _check(self.lib.kvmem_recall_step_host(
            self.handle, session_first, ns, q_host.data_ptr(), M, C.byref(params), _dev(sel_ids, torch.int32),
            sel_ids.shape[-1], _dev(n_sel, torch.int32), _dev(view.k, torch.bfloat16), _dev(view.v, torch.bfloat16),
            view.cap_tokens, scale, out_host.data_ptr(), lse_host.data_ptr(), self._staging.data_ptr(),
            self._staging.numel(), sws.data_ptr(), sws.numel(), aws.data_ptr(), aws.numel(), _stream()))

    def host_step(self, q_shape, params: SelectParams, sel_ids: torch.Tensor, n_sel: torch.Tensor, view: View,
                  out_host: torch.Tensor, lse_host: torch.Tensor, scale: float = 0.0, session_first: int = 0) -> "HostStep":
        """recall_step_host with everything but the query marshalled once (a decode loop calls the same step with the
        same buffers every token): returns a callable that takes the pinned bf16 query of shape q_shape."""
        return HostStep(self, tuple(q_shape), params, sel_ids, n_sel, view, out_host, lse_host, scale, session_first)

    # ---- helpers that only allocate
    def new_view(self, n_sessions: int, cap_tokens: int) -> View:
        c = self.cfg
        shape = (n_sessions, c.n_layers, c.n_kv_heads, cap_tokens, c.head_dim)
        return View(torch.zeros(shape, dtype=torch.bfloat16, device=self.device),
                    torch.zeros(shape, dtype=torch.bfloat16, device=self.device), cap_tokens)

    def new_outputs(self, n_sessions: int, n_q_tokens: int) -> Tuple[torch.Tensor, torch.Tensor]:
        c = self.cfg
        out = torch.empty(n_sessions, n_q_tokens, c.n_layers, c.n_q_heads, c.head_dim, dtype=torch.float32,
                          device=self.device)
        lse = torch.empty(n_sessions, n_q_tokens, c.n_layers, c.n_q_heads, dtype=torch.float32, device=self.device)
        return out, lse

    # ---- inspection
    def index(self, session: int) -> torch.Tensor:
        """Copy of the session's Mean-K index: bf16 [L][G][n_blocks][d]."""
        ptr, n = C.c_void_p(), C.c_int32()
        _check(self.lib.kvmem_get_index(self.handle, session, C.byref(ptr), C.byref(n)))
        c = self.cfg
        off = (ptr.value - self.storage.data_ptr())
        elems = c.n_layers * c.n_kv_heads * c.max_blocks_per_session * c.head_dim
        full = self.storage[off:off + 2 * elems].view(torch.bfloat16).view(c.n_layers, c.n_kv_heads,
                                                                              c.max_blocks_per_session, c.head_dim)
        return full[:, :, :n.value, :].clone()

    def pages(self) -> torch.Tensor:
        """bf16 [max_blocks][K | V][L][G][B][d]: the pages of a bf16 repository (a view of the pool's storage)."""
        ptr = C.c_void_p()
        _check(self.lib.kvmem_get_pages(self.handle, C.byref(ptr)))
        c = self.cfg
        if c.fp8_pages:
            raise KvmemError(E_STATE, "the pool's pages hold FP8 codes")
        shape = (c.max_blocks, 2, c.n_layers, c.n_kv_heads, c.block_tokens, c.head_dim)
        off, n = (ptr.value or 0) - self.storage.data_ptr(), 2 * c.max_blocks * 2 * c.n_layers * c.n_kv_heads * c.block_tokens * c.head_dim
        return self.storage[off:off + n].view(torch.bfloat16).view(shape)

    def block_table(self, session: int) -> torch.Tensor:
        ptr, n = C.c_void_p(), C.c_int32()
        _check(self.lib.kvmem_get_block_table(self.handle, session, C.byref(ptr), C.byref(n)))
        off = ptr.value - self.storage.data_ptr()
        return self.storage[off:off + 4 * n.value].view(torch.int32).clone()

    def selftest_wait_timeout(self, limit_us: int = 1000) -> int:
        """Run the kernels' bounded wait to its limit on a barrier nobody arrives at; returns the nanoseconds it lasted.
        The status word then holds E_TIMEOUT until device_status() reads it."""
        waited = torch.zeros(1, dtype=torch.int64, device=self.device)
        _check(self.lib.kvmem_selftest_wait_timeout(self.handle, limit_us, waited.data_ptr(), _stream()))
        return int(waited.item())

    def selftest_joint_wait_timeout(self, unmet: int, limit_us: int = 1000) -> int:
        """The same for the wait that asks three barriers together; barrier `unmet` (0 .. 2) is the one nobody arrives at."""
        waited = torch.zeros(1, dtype=torch.int64, device=self.device)
        _check(self.lib.kvmem_selftest_joint_wait_timeout(self.handle, unmet, limit_us, waited.data_ptr(), _stream()))
        return int(waited.item())

    def device_status(self) -> int:
        st = C.c_int32()
        _check(self.lib.kvmem_device_status(self.handle, C.byref(st), _stream()))
        return st.value


class ViewCache:
    """The execution view kept across steps for one session: `cap_blocks` slots of one block each (keys
    encoded for their compact position, values unchanged), updated as a working-set delta."""

    def __init__(self, pool: Pool, cap_blocks: int, max_delta_ropes: int, first_position: int = 0):
        self.pool, self.cap, self.max_delta, self.first_position = pool, cap_blocks, max_delta_ropes, first_position
        need = pool.lib.kvmem_view_cache_bytes(pool.handle, cap_blocks)
        if need == 0:
            raise KvmemError(E_INVALID, "cap_blocks must be in [1, 32768]")
        self.buf = torch.empty(need, dtype=torch.uint8, device=pool.device)
        offs = (C.c_size_t * 6)()
        _check(pool.lib.kvmem_view_cache_layout(pool.handle, cap_blocks, offs))
        self.offsets = list(offs)
        self.stats = torch.zeros(4, dtype=torch.int32, device=pool.device)
        _check(pool.lib.kvmem_view_cache_reset(pool.handle, self.buf.data_ptr(), self.buf.numel(), cap_blocks, _stream()))

    def update(self, session: int, sel_ids: torch.Tensor, n_sel: torch.Tensor) -> None:
        """sel_ids int32 [>= n] ascending (one session's row), n_sel int32 [1]; stats land in self.stats."""
        p = self.pool
        _check(p.lib.kvmem_view_cache_update(p.handle, session, _dev(sel_ids, torch.int32), _dev(n_sel, torch.int32),
                                             self.buf.data_ptr(), self.buf.numel(), self.cap, self.max_delta,
                                             self.first_position, self.stats.data_ptr(), _stream()))

    def attend(self, q: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, scale: float = 0.0) -> None:
        """q bf16 [M][L][H][d] (one session) -> out fp32 [M][L][H][d], lse fp32 [M][L][H]."""
        p = self.pool
        M = q.shape[0]
        ws = p.attend_workspace(1, M)
        _check(p.lib.kvmem_view_cache_attend(p.handle, _dev(q, torch.bfloat16), M, self.buf.data_ptr(), self.buf.numel(),
                                             self.cap, scale, _dev(out, torch.float32), _dev(lse, torch.float32),
                                             ws.data_ptr(), ws.numel(), _stream()))

    # ---- inspection (copies)
    def _ints(self, which: int, n: int) -> torch.Tensor:
        o = self.offsets[which]
        return self.buf[o:o + 4 * n].view(torch.int32).clone()

    def records(self):
        """(slot_block, slot_pos, slot_cnt, view_slots, n_view) as CPU tensors / int."""
        torch.cuda.synchronize(self.pool.device)
        return (self._ints(1, self.cap).cpu(), self._ints(2, self.cap).cpu(), self._ints(3, self.cap).cpu(),
                self._ints(4, self.cap).cpu(), int(self._ints(5, 1).cpu()[0]))

    def pages(self) -> torch.Tensor:
        """bf16 [cap][2][L][G][B][d]: the slots in the pool's page format (a view of the cache buffer)."""
        c = self.pool.cfg
        n = self.cap * 2 * c.n_layers * c.n_kv_heads * c.block_tokens * c.head_dim
        o = self.offsets[0]
        return self.buf[o:o + 2 * n].view(torch.bfloat16).view(self.cap, 2, c.n_layers, c.n_kv_heads, c.block_tokens, c.head_dim)
