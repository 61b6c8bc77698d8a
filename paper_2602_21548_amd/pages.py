"""Binding of include/kvl_pages.h: whose the blocks of a paged cache are, and copies of blocks."""
from __future__ import annotations

import ctypes as C
import operator
from typing import List, Sequence

import numpy as np
import torch

from . import binding as _b


class kvl_block_copy_t(C.Structure):
    _fields_ = [("from_", C.c_int32), ("to", C.c_int32)]


class kvl_page_layout_t(C.Structure):
    _fields_ = [("n_layers", C.c_uint32), ("n_planes", C.c_uint32), ("block_bytes", C.c_uint64 * _b.KVL_MAX_PLANES), ("pool_blocks", C.c_uint64)]


class kvl_pages_stats_t(C.Structure):
    _fields_ = [(f, C.c_uint64) for f in ("free_blocks", "used_blocks", "shared_blocks", "moves", "sequences")]


# (arrays go by their addresses)
_P = C.c_void_p
SIGNATURES = {
    "kvl_pages": (C.c_int, [C.c_uint32, C.c_uint64, C.POINTER(_P)]),
    "kvl_pages_destroy": (None, [_P]),
    "kvl_pages_adopt": (C.c_int, [_P, C.POINTER(_b.kvl_request_t), C.c_uint32, _P]),
    "kvl_pages_fork": (C.c_int, [_P, _P, C.c_uint32, _P]),
    "kvl_pages_extend": (C.c_int, [_P, _P, _P, C.c_uint32, _P, C.POINTER(C.c_uint32)]),
    "kvl_pages_truncate": (C.c_int, [_P, _P, _P, C.c_uint32]),
    "kvl_pages_free": (C.c_int, [_P, _P, C.c_uint32]),
    "kvl_pages_compact": (C.c_int, [_P, C.c_uint32, _P, C.POINTER(C.c_uint32)]),
    "kvl_pages_tables": (C.c_int, [_P, _P, C.c_uint32, _P, C.c_uint64, _P]),
    "kvl_pages_tokens": (C.c_int, [_P, _P, C.c_uint32, _P]),
    "kvl_pages_stats": (C.c_int, [_P, C.POINTER(kvl_pages_stats_t)]),
    "kvl_page_pools": (C.c_int, [C.POINTER(kvl_page_layout_t), C.POINTER(_P), C.c_uint32, C.POINTER(_P)]),
    "kvl_page_pools_destroy": (None, [_P]),
    "kvl_copy_blocks": (C.c_int, [_P, _P, C.c_uint64, _P]),
}
_lib = _b._lib
for _name, (_res, _args) in SIGNATURES.items():
    _fn = getattr(_lib, _name)
    _fn.restype, _fn.argtypes = _res, _args


def _fork(pages: int, s: np.ndarray, out: np.ndarray) -> int:
    return _lib.kvl_pages_fork(pages, s.ctypes.data, s.size, out.ctypes.data)


def _extend(pages: int, s: np.ndarray, tokens: np.ndarray, copies: np.ndarray) -> int:
    n = C.c_uint32()
    return _lib.kvl_pages_extend(pages, s.ctypes.data, tokens.ctypes.data, s.size, copies.ctypes.data, C.byref(n)) or n.value


def _compact(pages: int, copies: np.ndarray) -> int:
    n = C.c_uint32()
    return _lib.kvl_pages_compact(pages, copies.shape[0], copies.ctypes.data, C.byref(n)) or n.value


def _free(pages: int, s: np.ndarray) -> int:
    return _lib.kvl_pages_free(pages, s.ctypes.data, s.size)


def _tables(pages: int, s: np.ndarray, table: np.ndarray, first: np.ndarray) -> int:
    return _lib.kvl_pages_tables(pages, s.ctypes.data, s.size, table.ctypes.data if table.size else None, table.size, first.ctypes.data)


_copy = _b._not_taken
if _b._native is not None:
    # (by ctypes a call takes some microseconds more)
    _b._native.setup_pages(*(C.cast(getattr(_lib, f), C.c_void_p).value
                             for f in ("kvl_pages_fork", "kvl_pages_extend", "kvl_pages_free", "kvl_pages_tables", "kvl_copy_blocks", "kvl_pages_compact")))
    _fork, _extend, _free, _tables = _b._native.pages_fork, _b._native.pages_extend, _b._native.pages_free, _b._native.pages_tables
    _compact = _b._native.pages_compact
    _copy = _b._native.copy_blocks


class _Owner:
    """Of a handle."""

    def __init__(self, handle: int, destroy):
        self._h, self._destroy = handle, destroy

    def destroy(self) -> None:
        if self._h:
            self._destroy(self._h)
            self._h = None

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
    def handle(self) -> int:
        if not self._h:
            raise ValueError("destroyed")
        return self._h


class Pages(_Owner):
    """Owner of a kvl_pages_t*."""

    def __init__(self, handle: int, block_tokens: int, pool_blocks: int):
        super().__init__(handle, _lib.kvl_pages_destroy)
        self.block_tokens, self.pool_blocks = block_tokens, pool_blocks
        self._longest = 64                      # entries of tables that were asked for


class PagePools(_Owner):
    """Owner of a kvl_page_pools_t*; keeps the planes' tensors."""

    def __init__(self, handle: int, planes: List[torch.Tensor]):
        super().__init__(handle, _lib.kvl_page_pools_destroy)
        self.planes = planes


_UINT64, _UINT32, _INT32 = np.dtype(np.uint64), np.dtype(np.uint32), np.dtype(np.int32)


def _numbers(x, dtype, what: str) -> np.ndarray:
    """A contiguous array of whole numbers of this type."""
    if type(x) is np.ndarray and x.dtype is dtype and x.ndim == 1 and x.flags.c_contiguous:
        return x
    most = int(np.iinfo(dtype).max)
    if type(x) is np.ndarray and x.ndim == 1 and x.dtype.kind in "iu":
        if x.size and (int(x.min()) < 0 or int(x.max()) > most):
            raise ValueError(f"{what}: need whole numbers from 0 to {most}")
        return np.ascontiguousarray(x, dtype=dtype)
    try:
        x = [operator.index(v) for v in x]      # (NumPy makes floats of uint64 numbers beside others)
    except TypeError:
        x = [-1]
    if x and (min(x) < 0 or max(x) > most):
        raise ValueError(f"{what}: need whole numbers from 0 to {most}")
    return np.array(x, dtype=dtype)


def _sequences(x, what: str) -> np.ndarray:
    if type(x) is np.ndarray and x.dtype is _UINT64 and x.ndim == 1 and x.flags.c_contiguous:
        return x
    return _numbers(x, _UINT64, f"{what} sequences")


def _per_sequence(tokens, n: int, what: str) -> np.ndarray:
    """One number for all sequences, or one for each."""
    if type(tokens) is int and 0 <= tokens < 1 << 32:
        out = np.empty(n, dtype=_UINT32)
        out.fill(tokens)
        return out
    if isinstance(tokens, (int, np.integer)):
        tokens = [int(tokens)] * n
    tokens = _numbers(tokens, _UINT32, f"{what} tokens")
    if tokens.size != n:
        raise ValueError(f"{what}: need tokens for every sequence")
    return tokens


def kvl_pages(block_tokens: int, pool_blocks: int) -> Pages:
    """The blocks of a pool, all free."""
    for what, x, most in (("block_tokens", block_tokens, 32), ("pool_blocks", pool_blocks, 64)):
        if not 0 <= int(x) < 1 << most:
            raise ValueError(f"kvl_pages: {what} is {x}")
    out = C.c_void_p()
    _b._check(_lib.kvl_pages(block_tokens, pool_blocks, C.byref(out)), "kvl_pages")
    return Pages(out.value, block_tokens, pool_blocks)


def kvl_pages_adopt(pages: Pages, tables: Sequence[np.ndarray], tokens) -> np.ndarray:
    """New sequences of so many tokens out of tables that are there already; their numbers (uint64)."""
    tables = list(tables)
    reqs, n, _keep = _b._requests(_per_sequence(tokens, len(tables), "kvl_pages_adopt"), np.zeros(len(tables), dtype=np.uint32), tables)
    out = np.zeros(n, dtype=np.uint64)
    _b._check(_lib.kvl_pages_adopt(pages.handle, reqs, n, out.ctypes.data), "kvl_pages_adopt")
    return out


def kvl_pages_fork(pages: Pages, sequences) -> np.ndarray:
    """New sequences that are what these are now; their numbers."""
    s = _sequences(sequences, "kvl_pages_fork")
    out = np.empty(s.size, dtype=_UINT64)
    _b._check(_fork(pages.handle, s, out), "kvl_pages_fork")
    return out


def kvl_pages_extend(pages: Pages, sequences, tokens) -> np.ndarray:
    """Sequences grow by so many tokens (a number, or one for each).  The copies that have to be made before the new tokens are written:
    int32 [copies, 2], from and to."""
    s = _sequences(sequences, "kvl_pages_extend")
    t = _per_sequence(tokens, s.size, "kvl_pages_extend")
    copies = np.empty((s.size, 2), dtype=_INT32)
    n = _extend(pages.handle, s, t, copies)
    if n < 0:
        _b._check(n, "kvl_pages_extend")
    return copies[:n]


def kvl_pages_truncate(pages: Pages, sequences, tokens) -> None:
    """Sequences keep their first tokens."""
    s = _sequences(sequences, "kvl_pages_truncate")
    t = _per_sequence(tokens, s.size, "kvl_pages_truncate")
    _b._check(_lib.kvl_pages_truncate(pages.handle, s.ctypes.data, t.ctypes.data, s.size), "kvl_pages_truncate")


def kvl_pages_free(pages: Pages, sequences) -> None:
    """Sequences end."""
    s = _sequences(sequences, "kvl_pages_free")
    _b._check(_free(pages.handle, s), "kvl_pages_free")


def kvl_pages_compact(pages: Pages, most: int = None) -> np.ndarray:
    """Blocks in use move to the front of the pool, at most so many (all by default).  The copies, int32 [copies, 2], from and to, which have to be made
    before anything else is written."""
    moves = pages.pool_blocks // 2              # (as many blocks in use as free ones change places, at most)
    if most is not None:
        if int(most) < 0:
            raise ValueError(f"kvl_pages_compact: most is {most}")
        moves = min(moves, int(most))
    copies = np.empty((moves, 2), dtype=_INT32)
    n = _compact(pages.handle, copies)
    if n < 0:
        _b._check(n, "kvl_pages_compact")
    return copies[:n] if 4 * n > moves else copies[:n].copy()


def kvl_pages_tables(pages: Pages, sequences) -> List[np.ndarray]:
    """The block table of each sequence (int32; parts of one array, of at most four times their entries, or of 64)."""
    s = _sequences(sequences, "kvl_pages_tables")
    first, table = np.empty(s.size + 1, dtype=_UINT64), np.empty(pages._longest, dtype=_INT32)
    rc = _tables(pages.handle, s, table, first)
    if rc == _b.KVL_ESPACE:
        table = np.empty(int(first[-1]), dtype=np.int32)
        pages._longest = table.size
        rc = _tables(pages.handle, s, table, first)
    _b._check(rc, "kvl_pages_tables")
    at = first.tolist()
    if table.size > 4 * max(at[-1], 16):        # (short tables do not keep the room of the longest ones that were asked for)
        table = table[:at[-1]].copy()
    return [table[a:b] for a, b in zip(at, at[1:])]


def kvl_pages_tokens(pages: Pages, sequences) -> np.ndarray:
    """The tokens of each sequence (uint32)."""
    s = _sequences(sequences, "kvl_pages_tokens")
    out = np.zeros(s.size, dtype=np.uint32)
    _b._check(_lib.kvl_pages_tokens(pages.handle, s.ctypes.data, s.size, out.ctypes.data), "kvl_pages_tokens")
    return out


def kvl_pages_stats(pages: Pages) -> dict:
    """free_blocks, used_blocks, shared_blocks, moves (that kvl_pages_compact would make), sequences."""
    s = kvl_pages_stats_t()
    _b._check(_lib.kvl_pages_stats(pages.handle, C.byref(s)), "kvl_pages_stats")
    return {f: int(getattr(s, f)) for f, _ in s._fields_}


def kvl_page_pools(block_bytes: Sequence[int], pool_blocks: int, pools: Sequence[Sequence[torch.Tensor]], flags: int = 0) -> PagePools:
    """The planes of all layers that copies of blocks go through: pools[layer][plane], device tensors whose blocks have block_bytes[plane] bytes."""
    what = "kvl_page_pools"
    n_layers, n_planes = len(pools), len(block_bytes)
    if not 1 <= n_planes <= _b.KVL_MAX_PLANES or any(len(layer) != n_planes for layer in pools):
        raise ValueError(f"{what}: need 1 to {_b.KVL_MAX_PLANES} planes, the same of every layer")
    if any(not 0 <= int(x) < 1 << 63 for x in (*block_bytes, pool_blocks)):
        raise ValueError(f"{what}: sizes must be whole numbers")
    planes = [t for layer in pools for t in layer]
    arr = (C.c_void_p * max(1, len(planes)))()
    for i, t in enumerate(planes):
        arr[i] = _b._dev(t, what)
        if t.nbytes < block_bytes[i % n_planes] * pool_blocks:
            raise ValueError(f"{what}: plane {i % n_planes} of layer {i // n_planes} holds {t.nbytes} bytes, need {block_bytes[i % n_planes] * pool_blocks}")
    lay, out = kvl_page_layout_t(n_layers, n_planes, (C.c_uint64 * _b.KVL_MAX_PLANES)(*block_bytes), pool_blocks), C.c_void_p()
    _b._check(_lib.kvl_page_pools(C.byref(lay), arr, flags, C.byref(out)), what)
    return PagePools(out.value, planes)


def kvl_copy_blocks(pools: PagePools, copies, stream=None) -> None:
    """Copy blocks of every layer and plane: int32 [copies, 2], from and to.  No block may be the destination of two, or of one and the source of one."""
    c = copies
    if not (type(c) is np.ndarray and c.dtype is _INT32 and c.ndim == 2 and c.shape[1] == 2 and c.flags.c_contiguous):
        c = np.asarray(copies)
        if c.size == 0:
            c = np.empty((0, 2), dtype=np.int32)
        if c.ndim != 2 or c.shape[1] != 2 or (c.size and (c.dtype.kind not in "iu" or int(c.min()) < -(1 << 31) or int(c.max()) >= 1 << 31)):
            raise ValueError("kvl_copy_blocks: copies must be whole numbers [copies, 2]")
        c = np.ascontiguousarray(c, dtype=np.int32)
    rc = _copy(pools.handle, c, stream)
    if rc > 0:
        rc = _lib.kvl_copy_blocks(pools.handle, c.ctypes.data, c.shape[0], _b._stream_handle(stream))
    _b._check(rc, "kvl_copy_blocks")
