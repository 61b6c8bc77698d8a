"""Binding of the attention operators declared in include/kvl_attn.h: new tokens into a paged cache, and attention over it."""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as _b

KVL_BF16, KVL_F16, KVL_E4M3 = 1, 2, 3
KVL_ROPE_HALVES, KVL_ROPE_NEIGHBOURS = 0, 1

_DTYPES = {torch.bfloat16: KVL_BF16, torch.float16: KVL_F16, torch.float8_e4m3fn: KVL_E4M3}


class kvl_attn_layout_t(C.Structure):
    _fields_ = [("block_tokens", C.c_uint32), ("q_heads", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("dtype", C.c_uint32), ("cache_dtype", C.c_uint32), ("window", C.c_uint32), ("sinks", C.c_uint32),
                ("rope_dim", C.c_uint32), ("rope_pairs", C.c_uint32), ("pool_blocks", C.c_uint64)]


class kvl_attn_item_t(C.Structure):
    _fields_ = [(f, C.c_uint32) for f in ("request", "first_row", "n_rows", "begin", "end", "sinks", "gap", "pieces")]


class kvl_append_t(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("q", C.c_void_p), ("q_out", C.c_void_p),
                ("k_stride", C.c_uint64), ("v_stride", C.c_uint64), ("q_stride", C.c_uint64), ("q_out_stride", C.c_uint64),
                ("rope", C.c_void_p), ("rope_positions", C.c_uint64)]


class kvl_attn_t(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("q_stride", C.c_uint64), ("out_stride", C.c_uint64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("scale", C.c_float)]


_PLAN_P = C.c_void_p
SIGNATURES = {
    "kvl_attn_plan": (C.c_int, [C.POINTER(kvl_attn_layout_t), C.POINTER(_b.kvl_request_t), C.c_uint32, C.c_uint32, C.POINTER(_PLAN_P)]),
    "kvl_attn_plan_destroy": (None, [_PLAN_P]),
    "kvl_attn_plan_tokens": (C.c_int, [_PLAN_P, C.POINTER(C.c_uint64)]),
    "kvl_attn_plan_workspace": (C.c_int, [_PLAN_P, C.POINTER(C.c_uint64)]),
    "kvl_attn_plan_items": (C.c_int, [_PLAN_P, C.POINTER(kvl_attn_item_t), C.c_uint64, C.POINTER(C.c_uint64)]),
    "kvl_append_layer": (C.c_int, [_PLAN_P, C.POINTER(kvl_append_t), C.POINTER(C.c_void_p), C.c_void_p]),
    "kvl_attn_layer": (C.c_int, [_PLAN_P, C.POINTER(kvl_attn_t), C.POINTER(C.c_void_p), C.c_void_p]),
}
_lib = _b._lib
for _name, (_res, _args) in SIGNATURES.items():
    _fn = getattr(_lib, _name)
    _fn.restype, _fn.argtypes = _res, _args

if _b._native is not None:
    _b._native.setup_attn(torch.float32, *(C.cast(getattr(_lib, f), C.c_void_p).value for f in ("kvl_append_layer", "kvl_attn_layer")))
    # (as binding.py's: what the library returned, or 1 for a call that is the general path's)
    _fast_append, _fast_attn = _b._native.append_layer, _b._native.attn_layer
else:
    _fast_append = _fast_attn = _b._not_taken


def make_attn_layout(block_tokens: int, q_heads: int, kv_heads: int, head_dim: int, pool_blocks: int, dtype=torch.bfloat16,
                     cache_dtype=None, window: int = 0, sinks: int = 0, rope_dim: int = 0,
                     rope_pairs: int = KVL_ROPE_HALVES) -> kvl_attn_layout_t:
    """Geometry of the operators: dtype is that of queries, new keys and values and outputs (torch.bfloat16 or torch.float16),
    cache_dtype the pool's (dtype if None, or torch.float8_e4m3fn)."""
    cache_dtype = dtype if cache_dtype is None else cache_dtype
    for t in (dtype, cache_dtype):
        if t not in _DTYPES:
            raise ValueError(f"make_attn_layout: no element type {t}")
    for what, x in (("block_tokens", block_tokens), ("q_heads", q_heads), ("kv_heads", kv_heads), ("head_dim", head_dim),
                    ("window", window), ("sinks", sinks), ("rope_dim", rope_dim), ("rope_pairs", rope_pairs)):
        if not 0 <= int(x) < 1 << 32:
            raise ValueError(f"make_attn_layout: {what} is {x}")
    return kvl_attn_layout_t(block_tokens, q_heads, kv_heads, head_dim, _DTYPES[dtype], _DTYPES[cache_dtype], window, sinks,
                             rope_dim, rope_pairs, pool_blocks)


class AttnPlan(_b._native.AttnPlanBase if _b._native is not None else object):
    """Owner of a kvl_attn_plan_t*."""

    def __init__(self, handle: int, layout: kvl_attn_layout_t, flags: int):
        self._h = C.c_void_p(handle)
        self.layout, self.flags = layout, flags
        self.dtype = torch.bfloat16 if layout.dtype == KVL_BF16 else torch.float16
        v = C.c_uint64()
        _b._check(_lib.kvl_attn_plan_tokens(self._h, C.byref(v)), "kvl_attn_plan_tokens")
        self.tokens = int(v.value)                      # new tokens of the batch
        _b._check(_lib.kvl_attn_plan_workspace(self._h, C.byref(v)), "kvl_attn_plan_workspace")
        self.workspace_bytes = int(v.value)             # device memory that kvl_attn_layer wants
        rows = int(layout.pool_blocks) * int(layout.block_tokens) * int(layout.kv_heads) * int(layout.head_dim)
        scales = 4 * int(layout.pool_blocks) * int(layout.kv_heads)
        self.plane_bytes = (rows, rows, scales, scales) if layout.cache_dtype == KVL_E4M3 else (2 * rows, 2 * rows)
        self._pointers = C.c_void_p * len(self.plane_bytes)
        self._q_shape = (self.tokens, int(layout.q_heads), int(layout.head_dim))
        self._kv_shape = (self.tokens, int(layout.kv_heads), int(layout.head_dim))
        if _b._native is not None:
            self._set(handle or 0, self.plane_bytes, self.dtype, self.tokens, layout.q_heads, layout.kv_heads, layout.head_dim,
                      layout.rope_dim // 2, 1 / math.sqrt(layout.head_dim))

    def destroy(self) -> None:
        if self._h:
            if _b._native is not None:
                self._clear()
            _lib.kvl_attn_plan_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()
        return False

    @property
    def handle(self) -> C.c_void_p:
        if not self._h:
            raise ValueError("plan destroyed")
        return self._h

    def items(self) -> np.ndarray:
        """Pieces of attention work as an (n, 8) uint32 array, columns as in kvl_attn_item_t."""
        n = C.c_uint64()
        _b._check(_lib.kvl_attn_plan_items(self.handle, None, 0, C.byref(n)), "kvl_attn_plan_items")
        out = np.zeros((n.value, 8), dtype=np.uint32)
        _b._check(_lib.kvl_attn_plan_items(self.handle, out.ctypes.data_as(C.POINTER(kvl_attn_item_t)), n.value, C.byref(n)),
                  "kvl_attn_plan_items")
        return out


def kvl_attn_plan(layout: kvl_attn_layout_t, hit, app, tables: Sequence[np.ndarray], flags: int) -> AttnPlan:
    """One plan for both operators on a batch (hit prefix, appended tail and block table of each request, as kvl_plan):
    KVL_SCATTER for kvl_append_layer, KVL_GATHER for kvl_attn_layer, with KVL_TOKENS_* for the keys that it sees."""
    reqs, n, _keep = _b._requests(hit, app, tables)
    out = C.c_void_p()
    _b._check(_lib.kvl_attn_plan(C.byref(layout), reqs, n, flags, C.byref(out)), "kvl_attn_plan")
    return AttnPlan(out.value, layout, flags)


def _planes(plan: AttnPlan, planes: Sequence[torch.Tensor], what: str):
    if len(planes) != len(plan.plane_bytes):
        raise ValueError(f"{what}: expected {len(plan.plane_bytes)} planes")
    arr = plan._pointers()
    for p, t in enumerate(planes):
        arr[p] = _b._dev(t, f"{what} pool")
        if t.nbytes < plan.plane_bytes[p]:
            raise ValueError(f"{what}: plane {p} holds {t.nbytes} bytes, pool needs {plan.plane_bytes[p]}")
    return arr


def _rows(plan: AttnPlan, t: torch.Tensor, shape, what: str):
    """(pointer, elements between tokens) of a [tokens, heads, head_dim] tensor whose tokens' heads are dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != plan.dtype:
        raise TypeError(f"{what}: need a device tensor of {plan.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, need {shape}")
    per, heads, dim = t.stride()
    if shape[0] and (dim != 1 or (shape[1] > 1 and heads != shape[2])):
        raise ValueError(f"{what}: a token's heads must be dense")
    dense = shape[1] * shape[2]
    if shape[0] <= 1:
        per = dense
    if per < dense or per % 8 or t.data_ptr() % 16:
        raise ValueError(f"{what}: tokens must lie at least {dense} elements apart, at multiples of 16 bytes")
    return t.data_ptr(), per


def kvl_append_layer(plan: AttnPlan, k: torch.Tensor, v: torch.Tensor, pool_planes: Sequence[torch.Tensor],
                     rope: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """New keys (rotated) and values of one layer into its pool; queries, if given, rotated into q_out (q itself by default).

    k, v: [tokens, kv_heads, head_dim]; q, q_out: [tokens, q_heads, head_dim]; tokens may lie at a stride (parts of one
    projection's output).  rope: float32 [positions, rope_dim / 2, 2], cosines and sines.  An 8-bit pool has four planes: codes
    of keys and of values, float32 [pool_blocks, kv_heads] scales of each."""
    what = "kvl_append_layer"
    rc = _fast_append(plan, k, v, pool_planes, rope, q, q_out, stream)
    if rc <= 0:
        return _b._check(rc, what)
    a = kvl_append_t()
    arr = _planes(plan, pool_planes, what)
    a.k, a.k_stride = _rows(plan, k, plan._kv_shape, f"{what} k")
    a.v, a.v_stride = _rows(plan, v, plan._kv_shape, f"{what} v")
    if q is not None:
        a.q, a.q_stride = _rows(plan, q, plan._q_shape, f"{what} q")
        a.q_out, a.q_out_stride = _rows(plan, q if q_out is None else q_out, plan._q_shape, f"{what} q_out")
    elif q_out is not None:
        raise ValueError(f"{what}: q_out without q")
    if rope is not None:
        half = int(plan.layout.rope_dim) // 2
        if rope.dtype != torch.float32 or rope.dim() != 3 or tuple(rope.shape[1:]) != (half, 2):
            raise ValueError(f"{what}: rope must be float32 [positions, {half}, 2]")
        a.rope, a.rope_positions = _b._dev(rope, f"{what} rope"), rope.shape[0]
    elif plan.layout.rope_dim:
        raise ValueError(f"{what}: the layout rotates, but there is no rope table")
    if plan.tokens == 0:
        a.k = a.v = a.q = a.q_out = None                # (an empty tensor has no address)
    _b._check(_lib.kvl_append_layer(plan.handle, C.byref(a), arr, _b._stream_handle(stream)), what)


def kvl_attn_layer(plan: AttnPlan, q: torch.Tensor, pool_planes: Sequence[torch.Tensor], out: torch.Tensor,
                   workspace: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                   lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of the new tokens' queries over one layer's pool.

    q, out: [tokens, q_heads, head_dim], tokens at a stride of their own; out may be q; scale: 1 / sqrt(head_dim) by default; lse: float32
    [tokens, q_heads], or None; workspace: a device tensor of plan.workspace_bytes (None if that is 0), in nobody else's use
    until the work is done."""
    what = "kvl_attn_layer"
    rc = _fast_attn(plan, q, pool_planes, out, workspace, scale, lse, stream)
    if rc <= 0:
        return _b._check(rc, what)
    a = kvl_attn_t()
    arr = _planes(plan, pool_planes, what)
    a.q, a.q_stride = _rows(plan, q, plan._q_shape, f"{what} q")
    a.out, a.out_stride = _rows(plan, out, plan._q_shape, f"{what} out")
    if lse is not None:
        if lse.dtype != torch.float32 or tuple(lse.shape) != plan._q_shape[:2]:
            raise ValueError(f"{what}: lse must be float32 {plan._q_shape[:2]}")
        a.lse = _b._dev(lse, f"{what} lse")
    if workspace is not None:
        a.workspace, a.workspace_bytes = _b._dev(workspace, f"{what} workspace"), workspace.nbytes
    a.scale = 1 / math.sqrt(plan.layout.head_dim) if scale is None else scale
    _b._check(_lib.kvl_attn_layer(plan.handle, C.byref(a), arr, _b._stream_handle(stream)), what)
