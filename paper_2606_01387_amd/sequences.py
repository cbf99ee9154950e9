"""Running sequences on a pool's blocks: block tables, keys and values written
into the blocks, and attention over them.

The calls of ``include/claimkv.h`` under "sequences on a pool", with torch
tensors: argument checks and marshalling only, all work runs in the library's
HIP kernels.  Every call is queued in order with the current stream (the
pool's stream waits for it, and it for the pool's, where they differ) and
nothing waits for the GPU.
"""

from __future__ import annotations

import ctypes

from . import claimkv
from .claimkv import CAttendDesc, CKvDesc, CRows, CSeqs, ENOSPC, _check, _device_ints, _torch, lib

SEQ_OK, SEQ_NO_BLOCKS, SEQ_REFUSED = 0, 1, 2
NONE = -1  # a table entry that names no block (0xFFFFFFFF in 32 bits)


class Sequences:
    """Sequences over the blocks of ``pool``.

    ``tables`` [max_seqs, max_blocks], ``lengths`` [max_seqs] and ``refs``
    [num_blocks] are int32 device tensors that the calls change in place;
    without them, empty ones are made (max_seqs and max_blocks given)."""

    def __init__(self, pool: claimkv.Pool, max_seqs: int | None = None, max_blocks: int | None = None,
                 *, tables=None, lengths=None, refs=None):
        torch = _torch()
        g, dev = pool.geometry, pool.kv.device
        if tables is None:
            if not max_seqs or not max_blocks:
                raise ValueError("max_seqs and max_blocks (or tables) are needed")
            tables = torch.full((max_seqs, max_blocks), NONE, dtype=torch.int32, device=dev)
        if tables.dim() != 2 or tables.numel() == 0:
            raise ValueError("tables must be [max_seqs, max_blocks]")
        if lengths is None:
            lengths = torch.zeros(tables.shape[0], dtype=torch.int32, device=dev)
        if refs is None:
            refs = torch.zeros(g.num_blocks, dtype=torch.int32, device=dev)
        _device_ints(dev, tables=tables, lengths=lengths, refs=refs)
        if lengths.numel() != tables.shape[0] or refs.numel() != g.num_blocks:
            raise ValueError("lengths needs one entry per sequence, refs one per block")
        self.pool, self.tables, self.lengths, self.refs = pool, tables, lengths, refs
        words = 16 + 3 * g.num_blocks + 4 * tables.shape[0]
        self._scratch = torch.empty(words, dtype=torch.int32, device=dev)
        self._seqs = CSeqs(max_seqs=tables.shape[0], max_blocks=tables.shape[1],
                           tables=tables.data_ptr(), lengths=lengths.data_ptr(),
                           refs=refs.data_ptr(), work=self._scratch.data_ptr())
        self._seqs_ref = ctypes.addressof(self._seqs)
        self._state = (tables, lengths, refs, self._scratch)
        self._work = None

    # ------------------------------------------------------------- blocks
    def grow(self, ids, tokens):
        """claim_seqs_grow: ``tokens[i]`` more tokens for sequence ``ids[i]``
        (None: sequences 0..n-1), with blocks for them.  Returns the device
        tensor of statuses (SEQ_OK, SEQ_NO_BLOCKS, SEQ_REFUSED)."""
        return self._entries(lib().claim_seqs_grow, "claim_seqs_grow", ids=ids, tokens=tokens)

    def fork(self, parents, children):
        """claim_seqs_fork: the empty sequence ``children[i]`` becomes a copy
        of ``parents[i]`` that shares its full blocks.  Returns the statuses."""
        return self._entries(lib().claim_seqs_fork, "claim_seqs_fork", parents=parents,
                             children=children)

    def _entries(self, call, what, **given):
        (name, first), (_, second) = given.items()
        pool = self.pool
        _device_ints(pool.kv.device, **given)
        if first is None and name != "ids" or second is None:
            raise ValueError(f"{what} needs {' and '.join(given)}")
        n = second.numel()
        if first is not None and first.numel() != n:
            raise ValueError(f"{' and '.join(given)} need one entry per sequence")
        status = second.new_empty(n)
        with pool.ordered(first, second, status, *self._state):
            _check(call(pool._h, self._seqs_ref, _ptr(first), second.data_ptr(), n,
                        status.data_ptr()), what)
        return status

    def free(self, ids) -> None:
        """claim_seqs_free: sequences ``ids`` give up their blocks."""
        pool = self.pool
        _device_ints(pool.kv.device, ids=ids)
        with pool.ordered(ids, *self._state):
            _check(lib().claim_seqs_free(pool._h, self._seqs_ref, ids.data_ptr(), ids.numel()),
                   "claim_seqs_free")

    def compact(self):
        """claim_seqs_compact: blocks in use move to the front of the pool.
        Returns the device tensor [1] of how many moved."""
        pool = self.pool
        moved = self.refs.new_empty(1)
        with pool.ordered(moved, pool.kv, *self._state):
            _check(lib().claim_seqs_compact(pool._h, self._seqs_ref, moved.data_ptr()),
                   "claim_seqs_compact")
        return moved

    # ---------------------------------------------------- keys and values
    def write(self, layer: int, k, v, *, ids=None, offsets=None, k_scale: float = 1.0,
              v_scale: float = 1.0) -> None:
        """claim_kv_write: rows of ``k`` and ``v`` ([rows, num_kv_heads,
        head_dim], bf16) become the last tokens of their sequences in
        ``layer``: rows offsets[s]..offsets[s + 1] of sequence ids[s] (without
        ``offsets``, row s alone; without ``ids``, sequence s)."""
        pool, g = self.pool, self.pool.geometry
        heads, dim = g.num_kv_heads, g.head_dim
        rows_k, rows_v = self._rows("k", k, heads, dim), self._rows("v", v, heads, dim)
        if k.shape[0] != v.shape[0]:
            raise ValueError("k and v need the same rows")
        kv = self._kv(layer, k.shape[0], ids, offsets, k_scale, v_scale)
        with pool.ordered(k, v, ids, offsets, *self._state):
            _check(lib().claim_kv_write(pool._h, self._seqs_ref, ctypes.addressof(kv),
                                        ctypes.addressof(rows_k), ctypes.addressof(rows_v)),
                   "claim_kv_write")

    def attend(self, layer: int, q, *, ids=None, offsets=None, scale: float | None = None,
               k_scale: float = 1.0, v_scale: float = 1.0, out=None):
        """claim_attend: causal attention of ``q`` ([rows, heads, head_dim],
        bf16) over their sequences' tokens in ``layer``, the rows being the
        sequences' last tokens (as in :meth:`write`, which comes first).
        ``scale`` defaults to head_dim ** -0.5.  Returns ``out``."""
        return self._attend(layer, q, None, ids, offsets, scale, k_scale, v_scale, out)

    def attend_shared(self, layer: int, q, prefix, *, ids=None, offsets=None,
                      scale: float | None = None, k_scale: float = 1.0, v_scale: float = 1.0,
                      out=None):
        """:meth:`attend` for sequences that all begin with the whole blocks
        ``prefix`` (int32 device tensor), which are read once for all of them;
        the tables' own entries for those positions are not read."""
        _device_ints(self.pool.kv.device, prefix=prefix)
        return self._attend(layer, q, prefix, ids, offsets, scale, k_scale, v_scale, out)

    def _attend(self, layer, q, prefix, ids, offsets, scale, k_scale, v_scale, out):
        torch = _torch()
        pool, dim = self.pool, self.pool.geometry.head_dim
        heads = q.shape[1] if q.dim() == 3 else 0
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        d = CAttendDesc(kv=self._kv(layer, q.shape[0], ids, offsets, k_scale, v_scale),
                        q=self._rows("q", q, heads, dim), out=self._rows("out", out, heads, dim),
                        num_heads=heads, prefix_blocks=0 if prefix is None else prefix.numel(),
                        prefix=_ptr(prefix), scale=dim**-0.5 if scale is None else scale)
        if out.shape != q.shape:
            raise ValueError("out needs q's shape")
        at = ctypes.addressof(d)
        with pool.ordered(q, out, ids, offsets, prefix, pool.kv, *self._state):
            if self._work is not None:
                d.work, d.work_bytes = self._work.data_ptr(), self._work.numel()
            rc = lib().claim_attend(pool._h, self._seqs_ref, at)
            if rc == ENOSPC:  # the first call of a larger shape
                need = ctypes.c_uint64()
                _check(lib().claim_attend_work(pool._h, self._seqs_ref, at, ctypes.byref(need)),
                       "claim_attend_work")
                # memory of the pool's stream: what was queued there may use
                # the smaller one until it is done
                with torch.cuda.stream(pool.stream):
                    self._work = torch.empty(need.value, dtype=torch.uint8, device=q.device)
                d.work, d.work_bytes = self._work.data_ptr(), need.value
                rc = lib().claim_attend(pool._h, self._seqs_ref, at)
            _check(rc, "claim_attend")
        return out

    def _kv(self, layer, rows, ids, offsets, k_scale, v_scale) -> CKvDesc:
        _device_ints(self.pool.kv.device, ids=ids, offsets=offsets)
        if offsets is not None:
            n = offsets.numel() - 1
        else:
            n = rows
        if n < 0 or ids is not None and ids.numel() != n:
            raise ValueError("ids needs one entry per sequence, offsets one more")
        if layer < 0:
            raise ValueError("layer must not be negative")
        return CKvDesc(layer=layer, num_seqs=n, num_rows=rows, ids=_ptr(ids), offsets=_ptr(offsets),
                       k_scale=k_scale, v_scale=v_scale)

    def _rows(self, name, x, heads, dim) -> CRows:
        torch = _torch()
        if (x.dtype != torch.bfloat16 or x.device != self.pool.kv.device or x.dim() != 3
                or x.shape[1:] != (heads, dim) or x.numel() and x.stride(2) != 1):
            raise ValueError(f"{name} must be bf16 [rows, {heads}, {dim}] on {self.pool.kv.device}, "
                             "its last dimension contiguous")
        return CRows(data=x.data_ptr(), row_stride=x.stride(0), head_stride=x.stride(1))


def _ptr(t):
    return None if t is None else t.data_ptr()
