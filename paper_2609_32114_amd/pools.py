"""Binding of the state pools' operators (``include/hagdn.h``): moving rows of the pools
that the decode entry points keep their sequences' states in.

    pool_copy(pools, dst=None, src=None, sources=None)   # snapshot, restore, reorder, clear
    slots = pool_fork(pools, slots, parents)              # a beam search's step
    slots = pool_compact(pools, slots)                    # live states to the front

pools: a tensor [S, ..] or a list of them with one S, the layers' states and windows, of any
types; tables are int32.  All on one GPU and contiguous.
"""

from __future__ import annotations

import ctypes

import torch

from . import HagdnError, _check_buffer, _err, _ptr, load_library
from .layer import _stream, _workspace
from .mixer import _call


def pool_workspace_size(slots: int) -> int:
    """Bytes of workspace pool_fork and pool_compact need for pools of so many slots."""
    lib = load_library()
    n = lib.hagdn_pool_workspace_size(slots)
    if n == 0:
        raise HagdnError(1, _err(lib))
    return n


def _pools(pools, name="pools"):
    """(first tensor, its device index, rows, pointers, row sizes, count) of a list of pools."""
    pools = [pools] if isinstance(pools, torch.Tensor) else list(pools)
    if not pools:
        raise ValueError(f"{name} must not be empty")
    first = pools[0]
    rows, di = first.shape[0] if first.dim() else -1, first.get_device()
    for p in pools:
        if p.get_device() != di or di < 0 or not p.is_contiguous():
            raise ValueError(f"{name} must be contiguous tensors on one GPU")
        if p.dim() < 1 or p.shape[0] != rows:
            raise ValueError(f"{name} must have one number of rows (got {[tuple(q.shape) for q in pools]})")
    sizes = [p.numel() // rows * p.element_size() if rows else 0 for p in pools]
    n = len(pools)
    return first, di, rows, (ctypes.c_void_p * n)(*[p.data_ptr() for p in pools]), (ctypes.c_size_t * n)(*sizes), n


def _table(name, t, pool):
    """The length of a table of slots."""
    if t.dim() != 1:
        raise ValueError(f"{name} must be one-dimensional (got {tuple(t.shape)})")
    _check_buffer(name, t, pool.device, torch.int32, t.shape)
    return t.shape[0]


def pool_copy(pools, dst=None, src=None, sources=None):
    """Row dst[i] of every pool receives row src[i] of the same pool, as if all were read
    before any is written (at most 8192 rows), or of the tensor beside it in ``sources``.  A
    table that is None counts rows up: ``pool_copy(pools, slots, sources=finals)`` puts a
    prefill's states in their slots, ``pool_copy(finals, src=slots, sources=pools)`` gets
    them.  dst outside the pool: padding; src outside: a row of zeros, a new sequence's state.
    No two entries may name one destination."""
    lib = load_library()
    first, di, rows, pointers, sizes, n = _pools(pools)
    from_rows, from_pointers = rows, None
    if sources is not None:
        _, other, from_rows, from_pointers, from_sizes, m = _pools(sources, "sources")
        if m != n or other != di:
            raise ValueError("sources must be as many tensors as pools, on the same GPU")
        if rows and from_rows and list(sizes) != list(from_sizes):
            raise ValueError("rows of sources must have the pools' sizes")
    tables = [_table(name, t, first) for name, t in (("dst", dst), ("src", src)) if t is not None]
    if not tables:
        count = min(rows, from_rows)
    elif len(set(tables)) > 1:
        raise ValueError(f"dst and src must have one length (got {tables})")
    else:
        count = tables[0]
    if rows == 0 or count == 0:
        return
    if sources is not None and from_rows == 0:
        raise ValueError("sources have no rows")
    _call(di, lib.hagdn_pool_copy, pointers, from_pointers, sizes, n, _ptr(dst), _ptr(src), count, rows, from_rows,
          _stream(di))


def _plan(pools, workspace):
    first, di, rows, pointers, sizes, n = _pools(pools)
    ws, ws_bytes = _workspace(workspace, lambda: pool_workspace_size(rows), first)
    return first, di, rows, pointers, sizes, n, ws, ws_bytes


def _new_slots(out, count, pool):
    if out is None:
        return torch.empty(count, dtype=torch.int32, device=pool.device)
    _check_buffer("out", out, pool.device, torch.int32, (count,))
    return out


def pool_fork(pools, slots, parents, workspace=None, out=None):
    """Child i goes on from sequence parents[i], whose states are in slot
    slots[parents[i]] of the pools.  The first child of a slot stays in it, each other one, in
    order, gets the lowest slot that no child stays in, and a copy of its parent's rows.  The
    children must be all that the pools hold: every other slot counts as free.  Returns the
    children's slots; -1 where the parent has none, or the free slots did not suffice
    (device_status of the caller's own workspace is then DEV_POOL_FULL)."""
    lib = load_library()
    first, di, rows, pointers, sizes, n, ws, ws_bytes = _plan(pools, workspace)
    N, M = _table("slots", slots, first), _table("parents", parents, first)
    new = _new_slots(out, M, first)
    _call(di, lib.hagdn_pool_fork, pointers, sizes, n, slots.data_ptr(), N, parents.data_ptr(), M, rows,
          new.data_ptr(), ws.data_ptr(), ws_bytes, _stream(di))
    return new


def pool_compact(pools, slots, workspace=None, out=None):
    """Moves the states that the table ``slots`` names to the front of the pools: with L
    live slots those from L on go, in order, to the free ones below L.  Returns the table
    after it (``out`` may be the table itself); entries outside the pools stay as they are."""
    lib = load_library()
    first, di, rows, pointers, sizes, n, ws, ws_bytes = _plan(pools, workspace)
    N = _table("slots", slots, first)
    new = _new_slots(out, N, first)
    _call(di, lib.hagdn_pool_compact, pointers, sizes, n, slots.data_ptr(), N, rows, new.data_ptr(), ws.data_ptr(),
          ws_bytes, _stream(di))
    return new
