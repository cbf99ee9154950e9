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
import struct

from . import claimkv
from .claimkv import (CAttendDesc, CEvictDesc, CKvDesc, CRotateDesc, CRows, CSeqs, CWeighDesc, CWindowDesc,
                      ENOSPC, OK, _check, _torch, lib)

SEQ_OK, SEQ_NO_BLOCKS, SEQ_REFUSED = 0, 1, 2
NONE = -1  # a table entry that names no block (0xFFFFFFFF in 32 bits)

# claim_kv_desc with two claim_rows after it, and the other descriptions, packed in
# one step: filling them field by field takes longer than queueing the work
_WRITE = struct.Struct("<4I2Q2f6Q")
_ATTEND = struct.Struct("<4I2Q2f6Q2IQfI2Q")
assert _WRITE.size == ctypes.sizeof(CKvDesc) + 2 * ctypes.sizeof(CRows)
_ROTATE = struct.Struct("<4I2Q2f12Q2I4Q4I2QfI")
_WINDOW = struct.Struct(_ATTEND.format + "2IQ")
_WEIGH = struct.Struct("<4I2Q2f3Q3If5Q")
assert _WEIGH.size == ctypes.sizeof(CWeighDesc)
_EVICT = struct.Struct("<4I7Q")
assert _EVICT.size == ctypes.sizeof(CEvictDesc)
assert _WINDOW.size == ctypes.sizeof(CWindowDesc)
assert _ATTEND.size == ctypes.sizeof(CAttendDesc)
assert _ROTATE.size == ctypes.sizeof(CRotateDesc)


class Sequences:
    """Sequences over the blocks of ``pool``.

    ``tables`` [max_seqs, max_blocks], ``lengths`` [max_seqs] and ``refs``
    [num_blocks] are int32 device tensors that the calls change in place;
    without them, empty ones are made (max_seqs and max_blocks given).  Tables
    come with their lengths; without refs, those count the tables' entries.  They
    belong to the stream that is current here, and are filled before the pool's
    stream goes on."""

    def __init__(self, pool: claimkv.Pool, max_seqs: int | None = None, max_blocks: int | None = None,
                 *, tables=None, lengths=None, refs=None):
        torch = _torch()
        g, dev = pool.geometry, pool.kv.device
        if tables is None:
            if not max_seqs or not max_blocks:
                raise ValueError("max_seqs and max_blocks (or tables) are needed")
            tables = torch.full((max_seqs, max_blocks), NONE, dtype=torch.int32, device=dev)
            if lengths is None:
                lengths = torch.zeros(max_seqs, dtype=torch.int32, device=dev)
        if tables.dim() != 2 or tables.numel() == 0:
            raise ValueError("tables must be [max_seqs, max_blocks]")
        if lengths is None:
            raise ValueError("tables need their lengths")
        claimkv._device_ints(dev, tables=tables, lengths=lengths, refs=refs)
        if refs is None:
            # a block that a table names is not free; other entries count for none
            named = tables.flatten().long()
            named = named.where((named >= 0) & (named < g.num_blocks), g.num_blocks)
            refs = torch.zeros(g.num_blocks + 1, dtype=torch.int32, device=dev)
            refs = refs.scatter_add_(0, named, torch.ones_like(named, dtype=torch.int32))[:-1]
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
        if pool._current_stream(pool._device_index) != pool._stream_at:
            # the tensors belong to the current stream: the pool's waits until they
            # are filled, and their memory for the pool's work when they are dropped
            pool.stream.wait_stream(torch.cuda.current_stream(dev))
            self.record_stream(pool.stream)
        self._works, self._work_at, self._work_bytes = [], 0, 0
        self._desc = ctypes.create_string_buffer(max(_WINDOW.size, _ROTATE.size))
        self._desc_at = ctypes.addressof(self._desc)
        self._device, self._bf16, self._int32 = dev, torch.bfloat16, torch.int32
        self._float32, self._float64 = torch.float32, torch.float64
        self._heads, self._dim = g.num_kv_heads, g.head_dim
        self._lib = lib()

    # ------------------------------------------------------------- blocks
    def grow(self, ids, tokens):
        """claim_seqs_grow: ``tokens[i]`` more tokens for sequence ``ids[i]``
        (None: sequences 0..n-1), with blocks for them.  Returns the device
        tensor of statuses (SEQ_OK, SEQ_NO_BLOCKS, SEQ_REFUSED)."""
        at = 0 if ids is None else self._ints("ids", ids)
        return self._entries(self._lib.claim_seqs_grow, "claim_seqs_grow", ids, at, "tokens", tokens)

    def fork(self, parents, children):
        """claim_seqs_fork: the empty sequence ``children[i]`` becomes a copy
        of ``parents[i]`` that shares its full blocks.  Returns the statuses."""
        at = self._ints("parents", parents)
        return self._entries(self._lib.claim_seqs_fork, "claim_seqs_fork", parents, at, "children", children)

    def _entries(self, call, what, first, first_at, name, second):
        pool, second_at, n = self.pool, self._ints(name, second), second.numel()
        if first is not None and first.numel() != n:
            raise ValueError(f"{what} needs as many {name}")
        status = second.new_empty(n)
        with pool.ordered(self, first, second, status):
            _check(call(pool._h, self._seqs_ref, first_at, second_at, n, status.data_ptr()), what)
        return status

    def free(self, ids) -> None:
        """claim_seqs_free: sequences ``ids`` give up their blocks."""
        pool, at = self.pool, self._ints("ids", ids)
        with pool.ordered(self, ids):
            _check(self._lib.claim_seqs_free(pool._h, self._seqs_ref, at, ids.numel()), "claim_seqs_free")

    def compact(self):
        """claim_seqs_compact: blocks in use move to the front of the pool, but
        for those that the program holds by a count of its own in ``refs`` (a
        ``prefix`` of :meth:`attend_shared`, a claim's blocks).  Returns the
        device tensor [1] of how many moved."""
        pool = self.pool
        moved = self.refs.new_empty(1)
        with pool.ordered(self, moved):
            _check(self._lib.claim_seqs_compact(pool._h, self._seqs_ref, moved.data_ptr()),
                   "claim_seqs_compact")
        return moved

    def evict(self, ids, weights, tokens: int, *, sinks: int = 0, recent: int = 0):
        """claim_seqs_evict: sequences ``ids`` (None: all) that have more than
        ``tokens`` tokens keep the first ``sinks``, the last ``recent`` and of the
        others those of the largest ``weights`` (float32, as for :meth:`weigh`;
        they come along).  Returns the device tensors of statuses and of the
        kept tokens' old positions [n, tokens] (NONE past the new lengths), which
        is as long as ``tokens`` says, whatever the tables hold.
        Scratch is taken and kept as :meth:`attend` does."""
        at = 0 if ids is None else self._ints("ids", ids)
        n = self.tables.shape[0] if ids is None else ids.numel()
        if not 1 <= tokens < 1 << 31 or sinks < 0 or recent < 0 or sinks + recent > tokens:
            raise ValueError("tokens must be at least 1, and sinks and recent not more than that together")
        weights_at, stride = self._weights(weights)
        status, kept = self.lengths.new_empty(n), self.lengths.new_empty(n, tokens)
        given = (n, tokens, sinks, recent, at, weights_at, stride, kept.data_ptr(), status.data_ptr())
        with self.pool.ordered(self, ids, weights, status, kept):
            self._with_work(_EVICT, given, (), self._lib.claim_seqs_evict, self._lib.claim_seqs_evict_work)
        return status, kept

    # ---------------------------------------------------- keys and values
    def write(self, layer: int, k, v, *, ids=None, offsets=None, k_scale: float = 1.0,
              v_scale: float = 1.0) -> None:
        """claim_kv_write: rows of ``k`` and ``v`` ([rows, num_kv_heads,
        head_dim], bf16) become the last tokens of their sequences in
        ``layer``: rows offsets[s]..offsets[s + 1] of sequence ids[s] (without
        ``offsets``, row s alone; without ``ids``, sequence s)."""
        pool, rows = self.pool, k.shape[0]
        if rows != v.shape[0]:
            raise ValueError("k and v need the same rows")
        _WRITE.pack_into(self._desc, 0, *self._kv(layer, rows, ids, offsets), k_scale, v_scale,
                         *self._rows("k", k, self._heads), *self._rows("v", v, self._heads))
        at = self._desc_at
        with pool.ordered(self, k, v, ids, offsets):
            _check(self._lib.claim_kv_write(pool._h, self._seqs_ref, at, at + 40, at + 64),
                   "claim_kv_write")

    def write_rotated(self, layer: int, q, k, v, freqs, *, positions=None, sections=None, q_norm=None,
                      k_norm=None, eps: float = 1e-6, neighbours: bool = False, ids=None, offsets=None,
                      k_scale: float = 1.0, v_scale: float = 1.0, out=None):
        """claim_kv_write_rotated: :meth:`write` of keys that are first normed by
        head and turned by their positions, as ``q`` ([rows, heads, head_dim],
        bf16) is.  Returns ``out``, the queries for :meth:`attend` (it may be
        ``q``).

        ``freqs`` (float64 [pairs], radians a position; None: nothing turns)
        belong to the pairs (i, i + pairs) of a head, or with ``neighbours`` (2 i,
        2 i + 1).  ``positions`` (int32 [rows] or [rows, axes], up to 4) are the
        rows' positions, each axis's that of ``sections[axis]`` pairs in turn;
        without them, rows have their positions in their sequences.  ``q_norm``
        and ``k_norm`` (bf16 [head_dim]) are the weights of x w / sqrt(mean(x^2)
        + eps); None leaves heads as they are."""
        pool, shape = self.pool, q.shape
        if len(shape) != 3:
            raise ValueError("q must be [rows, heads, head_dim]")
        rows, heads, _ = shape
        given = (*self._rows("q", q, heads), *self._rows("k", k, self._heads, rows),
                 *self._rows("v", v, self._heads, rows))
        if out is None:
            out = q.new_empty(shape)
        elif out.shape != shape:
            raise ValueError("out needs q's shape")
        freqs_at = pairs = 0
        if freqs is not None:
            freqs_at, pairs = freqs.data_ptr(), freqs.numel()
            if freqs.dtype != self._float64 or freqs.device != self._device or not freqs.is_contiguous():
                raise ValueError(f"freqs must be a contiguous float64 tensor on {self._device}")
        sections = (pairs,) if sections is None else tuple(sections)
        at = row_stride = axis_stride = 0
        if positions is not None:
            given_as, strides = positions.shape, positions.stride()
            if (positions.dtype != self._int32 or positions.device != self._device
                    or len(given_as) not in (1, 2) or given_as[0] != rows):
                raise ValueError(f"positions must be int32 [rows] or [rows, axes] on {self._device}")
            if (given_as[1] if len(given_as) == 2 else 1) != len(sections):
                raise ValueError("positions need as many axes as sections")
            at, row_stride, axis_stride = positions.data_ptr(), strides[0], strides[1] if len(strides) == 2 else 0
        if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) != pairs:
            raise ValueError("sections must be up to 4 numbers of pairs that add up to freqs'")
        _ROTATE.pack_into(self._desc, 0, *self._kv(layer, rows, ids, offsets), k_scale, v_scale, *given,
                          *self._rows("out", out, heads), heads, 2 * pairs, freqs_at, at, row_stride,
                          axis_stride, *(sections + (0, 0, 0))[:4], self._norm("q_norm", q_norm),
                          self._norm("k_norm", k_norm), eps, 1 if neighbours else 0)
        with pool.ordered(self, q, k, v, out, freqs, positions, q_norm, k_norm, ids, offsets):
            _check(self._lib.claim_kv_write_rotated(pool._h, self._seqs_ref, self._desc_at),
                   "claim_kv_write_rotated")
        return out

    def attend(self, layer: int, q, *, ids=None, offsets=None, scale: float | None = None,
               k_scale: float = 1.0, v_scale: float = 1.0, out=None):
        """claim_attend: causal attention of ``q`` ([rows, heads, head_dim],
        bf16) over their sequences' tokens in ``layer``, the rows being the
        sequences' last tokens (as in :meth:`write`, which comes first).
        ``scale`` defaults to head_dim ** -0.5.  Returns ``out``.

        The first call of a shape may allocate scratch (so it comes before a
        graph capture of that shape); later ones use it again.  Scratch stays
        where it is, and with it a captured graph, as long as this object does."""
        return self._attend(layer, q, None, 0, 0, ids, offsets, scale, k_scale, v_scale, out)

    def attend_window(self, layer: int, q, window: int | None, *, sinks: int = 0, lse=None, ids=None,
                      offsets=None, scale: float | None = None, k_scale: float = 1.0,
                      v_scale: float = 1.0, out=None):
        """claim_attend_window: :meth:`attend` where a row sees the last
        ``window`` positions (its own among them; None: all) and the first
        ``sinks``.  Table entries of other positions are not read, but their
        blocks are not given up (:meth:`evict` does that).  With
        ``lse`` (float32 [rows, heads]), the logarithms of the rows' sums of
        exponentials are written there, for :meth:`weigh`.  Scratch is taken
        and kept as :meth:`attend` does."""
        return self._attend(layer, q, None, 0, 0, ids, offsets, scale, k_scale, v_scale, out,
                            (*self._window(window, sinks), lse))

    def attend_shared(self, layer: int, q, prefix, *, ids=None, offsets=None,
                      scale: float | None = None, k_scale: float = 1.0, v_scale: float = 1.0,
                      out=None):
        """:meth:`attend` for sequences that all begin with the whole blocks
        ``prefix`` (int32 device tensor), which are read once for all of them;
        the tables' own entries for those positions are not read.  A list that
        is kept over a :meth:`compact` needs a count more of its blocks in
        ``refs``, or they may move."""
        return self._attend(layer, q, prefix, self._ints("prefix", prefix), prefix.numel(), ids,
                            offsets, scale, k_scale, v_scale, out)

    def weigh(self, layer: int, q, lse, weights, *, window: int | None = None, sinks: int = 0, ids=None,
              offsets=None, scale: float | None = None, k_scale: float = 1.0) -> None:
        """claim_weigh: adds to ``weights`` (float32 [max_seqs, columns], a
        column for every position that a table has) what each cached token weighed
        for the rows of ``q``, whose logarithms ``lse`` :meth:`attend_window` gave
        with the same window, sinks and scales.  ``q`` and ``lse`` may be a
        prompt's last rows alone.  :meth:`fork` does not copy a row of weights,
        and :meth:`free` does not clear it.  Scratch is taken and kept as
        :meth:`attend` does."""
        shape = q.shape
        if len(shape) != 3:
            raise ValueError("q must be [rows, heads, head_dim]")
        given = (*self._kv(layer, shape[0], ids, offsets), k_scale, 1.0, *self._rows("q", q, shape[1]), shape[1],
                 *self._window(window, sinks), self._dim**-0.5 if scale is None else scale,
                 self._row_floats("lse", lse, shape), *self._weights(weights))
        with self.pool.ordered(self, q, lse, weights, ids, offsets):
            self._with_work(_WEIGH, given, (), self._lib.claim_weigh, self._lib.claim_weigh_work)

    def _attend(self, layer, q, prefix, prefix_at, blocks, ids, offsets, scale, k_scale, v_scale, out,
                window=None):
        pool, shape, L = self.pool, q.shape, self._lib
        if len(shape) != 3:
            raise ValueError("q must be [rows, heads, head_dim]")
        heads = shape[1]
        rows_q = self._rows("q", q, heads)
        if out is None:
            out = q.new_empty(shape)
        elif out.shape != shape:
            raise ValueError("out needs q's shape")
        given = (*self._kv(layer, shape[0], ids, offsets), k_scale, v_scale, *rows_q,
                 *self._rows("out", out, heads), heads, blocks, prefix_at,
                 self._dim**-0.5 if scale is None else scale, 0)
        lse, record, more, call, need = None, _ATTEND, (), L.claim_attend, L.claim_attend_work
        if window is not None:
            width, sinks, lse = window
            more = (width, sinks, 0 if lse is None else self._row_floats("lse", lse, shape))
            record, call, need = _WINDOW, L.claim_attend_window, L.claim_attend_window_work
        with pool.ordered(self, q, out, ids, offsets, prefix, lse):
            self._with_work(record, given, more, call, need)
        return out

    def _with_work(self, record, given, more, call, work):
        """``call`` with a description that ends in its scratch (and ``more``)."""
        pool = self.pool
        record.pack_into(self._desc, 0, *given, self._work_at, self._work_bytes, *more)
        rc = call(pool._h, self._seqs_ref, self._desc_at)
        if rc == OK:
            return
        if rc == ENOSPC:  # the first call of a larger shape
            need = ctypes.c_uint64()
            _check(work(pool._h, self._seqs_ref, self._desc_at, ctypes.byref(need)), work.__name__)
            # the smaller ones are kept: a captured graph holds their
            # addresses.  Each is at least twice the one before, so all of
            # them together are less than four times what was needed
            size = max(need.value, 2 * self._work_bytes)
            torch = _torch()
            with torch.cuda.stream(pool.stream):
                self._works.append(torch.empty(size, dtype=torch.uint8, device=self._device))
            self._work_at, self._work_bytes = self._works[-1].data_ptr(), size
            record.pack_into(self._desc, 0, *given, self._work_at, self._work_bytes, *more)
            rc = call(pool._h, self._seqs_ref, self._desc_at)
        if rc != OK:
            _check(rc, call.__name__)

    def record_stream(self, stream) -> None:
        """The sequences' own tensors are used on ``stream``."""
        for t in (*self._state, self.pool.kv):
            t.record_stream(stream)

    # ------------------------------------------------------------ checks
    def _ints(self, name, t) -> int:
        """The address of a contiguous int32 tensor on the pool's device."""
        if t.dtype != self._int32 or t.device != self._device or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor on {self._device}")
        return t.data_ptr()

    @staticmethod
    def _window(window, sinks):
        """A window's width and first positions, in 32 bits."""
        width = 0xFFFFFFFF if window is None else window
        if not 1 <= width <= 0xFFFFFFFF or not 0 <= sinks <= 0xFFFFFFFF:
            raise ValueError("window must be at least 1, or None; sinks must not be negative")
        return width, sinks

    def _weights(self, t):
        """The address and row stride of tokens' weights."""
        seqs, blocks = self.tables.shape
        room = blocks * self.pool.geometry.block_size
        if (t.dtype != self._float32 or t.device != self._device or t.dim() != 2 or t.shape[0] != seqs
                or t.shape[1] < room or t.stride(1) != 1 or (seqs > 1 and t.stride(0) < room)):
            raise ValueError(f"weights must be float32 [{seqs}, at least {room}] on {self._device}, rows contiguous")
        return t.data_ptr(), max(t.stride(0), room)

    def _row_floats(self, name, t, shape) -> int:
        """The address of a contiguous float32 tensor [rows, heads]."""
        if (t.dtype != self._float32 or t.device != self._device or t.shape != shape[:2]
                or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous float32 {list(shape[:2])} on {self._device}")
        return t.data_ptr()

    def _kv(self, layer, rows, ids, offsets):
        """claim_kv_desc up to the scales."""
        n, ids_at, offsets_at = rows, 0, 0
        if offsets is not None:
            offsets_at, n = self._ints("offsets", offsets), offsets.numel() - 1
        if ids is not None:
            ids_at = self._ints("ids", ids)
            if ids.numel() != n:
                raise ValueError("ids needs one entry per sequence")
        if n < 0 or layer < 0:
            raise ValueError("offsets needs one entry more than sequences; layer must not be negative")
        return layer, n, rows, 0, ids_at, offsets_at

    def _norm(self, name, w) -> int:
        """The address of a head's weights, or 0."""
        if w is None:
            return 0
        if w.dtype != self._bf16 or w.device != self._device or w.numel() != self._dim or not w.is_contiguous():
            raise ValueError(f"{name} must be contiguous bf16 [{self._dim}] on {self._device}")
        return w.data_ptr()

    def _rows(self, name, x, heads, rows=None):
        """claim_rows."""
        stride, shape = x.stride(), x.shape
        if (x.dtype != self._bf16 or x.device != self._device or len(stride) != 3
                or shape[1] != heads or shape[2] != self._dim or stride[2] != 1):
            raise ValueError(f"{name} must be bf16 [rows, {heads}, {self._dim}] on {self._device}, "
                             "its last dimension contiguous")
        if rows is not None and shape[0] != rows:
            raise ValueError(f"{name} needs {rows} rows")
        # the stride of a single row or head leads nowhere, and may be anything
        return x.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if heads > 1 else 0
