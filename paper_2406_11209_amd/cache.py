"""Thin Python binding of the paged compressed cache (include/pbz_cache.h): keys and values of attention layers held as
compressed arrays, attention taken on the compressed form, and the bookkeeping of pages.

    cache = PagedCache(head_dim=128, heads=8, n_pages=1024, page_size=64)
    seq = cache.open()
    cache.extend_and_append([seq], [k.shape[0]], k, v)          # k, v: [tokens, heads, head_dim]
    out = cache.attend_sequences([seq], [q.shape[0]], q)        # q: [tokens, query heads, head_dim]

The calls on tensors (`append`, `attend`, `copy_pages`) take device tensors for slots, tables and lengths, allocate
nothing but an output and a workspace where none is given, and can be captured into a graph with both given.  As in
`api`, every step runs in the HIP kernels; there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import threading
from typing import List, Optional, Sequence, Tuple

import numpy as np

from . import api

_c = ctypes
_p = _c.c_void_p
_i64, _i32 = _c.c_int64, _c.c_int32


class _Cache(_c.Structure):
    _fields_ = [("n_pages", _i64), ("heads", _i32), ("page_size", _i32), ("k_N", _p), ("k_F", _p), ("v_N", _p), ("v_F", _p)]


class _Lines(_c.Structure):
    _fields_ = [("data", _p), ("token_stride", _i64), ("head_stride", _i64)]


class _Attention(_c.Structure):
    _fields_ = [("q", _p), ("out", _p), ("lse", _p), ("type", _c.c_int), ("q_heads", _i32), ("q_token_stride", _i64),
                ("q_head_stride", _i64), ("out_token_stride", _i64), ("out_head_stride", _i64), ("n_tokens", _i64),
                ("n_seqs", _i64), ("starts", _p), ("lengths", _p), ("table", _p), ("table_stride", _i64),
                ("max_pages", _i64), ("max_new", _i64), ("max_length", _i64), ("causal", _i32), ("window", _i64),
                ("scale", _c.c_float)]


# name -> (restype, argtypes); mirrors include/pbz_cache.h declaration by declaration
_i64p, _i32p, _sizep = _c.POINTER(_i64), _c.POINTER(_i32), _c.POINTER(_c.c_size_t)
SIGNATURES = {
    "pbz_cache_layout": (_c.c_int, [_p, _c.POINTER(_Cache), _sizep, _sizep]),
    "pbz_cache_append": (_c.c_int, [_p, _c.POINTER(_Cache), _i64, _c.POINTER(_Lines), _c.POINTER(_Lines), _c.c_int, _p, _p]),
    "pbz_cache_copy_pages": (_c.c_int, [_p, _c.POINTER(_Cache), _i64, _p, _p]),
    "pbz_cache_attend_workspace": (_c.c_int, [_p, _c.POINTER(_Cache), _c.POINTER(_Attention), _sizep]),
    "pbz_cache_attend": (_c.c_int, [_p, _c.POINTER(_Cache), _c.POINTER(_Attention), _p, _c.c_size_t, _p]),
    "pbz_pages_create": (_c.c_int, [_c.POINTER(_p), _i64, _i32]),
    "pbz_pages_destroy": (None, [_p]),
    "pbz_pages_open": (_c.c_int, [_p, _i64p]),
    "pbz_pages_fork": (_c.c_int, [_p, _i64, _i64p]),
    "pbz_pages_close": (_c.c_int, [_p, _i64]),
    "pbz_pages_extend": (_c.c_int, [_p, _i64, _i64, _p, _i32p, _i32p]),
    "pbz_pages_truncate": (_c.c_int, [_p, _i64, _i64]),
    "pbz_pages_length": (_c.c_int, [_p, _i64, _i64p, _i64p]),
    "pbz_pages_table": (_c.c_int, [_p, _i64, _p, _i64]),
    "pbz_pages_free_count": (_c.c_int, [_p, _i64p]),
    "pbz_pages_compact": (_c.c_int, [_p, _p, _i64, _i64p]),
}

_ERR_PAGES = -15
_declared = None


def _library():
    """libpbz.so with the cache's entry points declared."""
    global _declared
    lib = api.load_library()
    if _declared is not lib:
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
            lib.addresses[name] = _c.cast(fn, _p).value
        _declared = lib
    return lib


def _pairs(pairs) -> np.ndarray:
    """(from, to) pages as the library takes them: contiguous int32 [n, 2]."""
    given = np.asarray(pairs)
    if given.dtype == np.int32 and given.ndim == 2 and given.shape[1] == 2:
        return np.ascontiguousarray(given)
    if given.size == 0:
        return np.empty((0, 2), dtype=np.int32)
    if given.dtype == object and all(isinstance(page, int) for page in given.flat):      # beyond 64 bits
        api.check(_ERR_PAGES)
    if given.dtype.kind not in "iu":
        raise ValueError("pairs of pages have to be integers")
    if given.ndim == 0 or given.size % 2 or (given.ndim > 1 and given.shape[-1] != 2):
        raise ValueError(f"pairs of pages have to be [n, 2], not {given.shape}")
    if given.dtype != np.int32 and (given.min() < 0 or given.max() > 2 ** 31 - 1):        # what int32 would make another page
        api.check(_ERR_PAGES)
    return np.ascontiguousarray(given, dtype=np.int32).reshape(-1, 2)


class Pages:
    """Which sequence owns which page (pbz_pages): host-side, no device work.  Owns the handle."""

    def __init__(self, n_pages: int, page_size: int):
        self._lib = _library()
        self._h = _p()
        api.check(self._lib.pbz_pages_create(_c.byref(self._h), int(n_pages), int(page_size)))
        self.n_pages, self.page_size = int(n_pages), int(page_size)

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            self._lib.pbz_pages_destroy(h)

    def open(self) -> int:
        seq = _i64()
        api.check(self._lib.pbz_pages_open(self._h, _c.byref(seq)))
        return seq.value

    def fork(self, sequence: int) -> int:
        seq = _i64()
        api.check(self._lib.pbz_pages_fork(self._h, sequence, _c.byref(seq)))
        return seq.value

    def close(self, sequence: int) -> None:
        api.check(self._lib.pbz_pages_close(self._h, sequence))

    def extend(self, sequence: int, tokens: int) -> Tuple[np.ndarray, Optional[Tuple[int, int]]]:
        """Slots (int64) of `tokens` more positions, and the (from, to) page copy to make before they are written."""
        slots = np.empty(max(int(tokens), 1), dtype=np.int64)
        copy, n = (_i32 * 2)(), _i32()
        api.check(self._lib.pbz_pages_extend(self._h, sequence, int(tokens), slots.ctypes.data, copy, _c.byref(n)))
        return slots, (copy[0], copy[1]) if n.value else None

    def truncate(self, sequence: int, length: int) -> None:
        api.check(self._lib.pbz_pages_truncate(self._h, sequence, int(length)))

    def length(self, sequence: int) -> int:
        n = _i64()
        api.check(self._lib.pbz_pages_length(self._h, sequence, _c.byref(n), None))
        return n.value

    def table(self, sequence: int, capacity: Optional[int] = None) -> np.ndarray:
        """The sequence's pages in order (int32), padded with -1 to `capacity`."""
        if capacity is None:
            n = _i64()
            api.check(self._lib.pbz_pages_length(self._h, sequence, None, _c.byref(n)))
            capacity = n.value
        table = np.empty(max(int(capacity), 1), dtype=np.int32)
        api.check(self._lib.pbz_pages_table(self._h, sequence, table.ctypes.data, int(capacity)))
        return table[:capacity]

    @property
    def free_count(self) -> int:
        n = _i64()
        api.check(self._lib.pbz_pages_free_count(self._h, _c.byref(n)))
        return n.value

    def compact(self) -> np.ndarray:
        """The page moves [n, 2] (from, to) that bring the pages in use to the front; tables already say so."""
        pairs = np.empty((self.n_pages // 2 + 1, 2), dtype=np.int32)
        n = _i64()
        api.check(self._lib.pbz_pages_compact(self._h, pairs.ctypes.data, pairs.shape[0], _c.byref(n)))
        return pairs[:n.value].copy()


class PagedCache:
    """Pools of compressed keys and values, {N, F} each, with the pages' owners.

    head_dim 32, 64, 128 or 256; page_size a power of two from 16 to 1024; work_type: of N ("f32", "f16", "bf16").
    pools: (k_N, k_F, v_N, v_F) that the program already holds, of `pool_shapes`; otherwise they are allocated here.
    """

    def __init__(self, head_dim: int, heads: int, n_pages: int, page_size: int = 64, work_type: str = "f32",
                 transform: str = "dct", pools: Optional[Sequence] = None, device="cuda"):
        self._lib = _library()
        self.codec = api.Codec((int(head_dim),), work_type, "i8", transform=transform)
        self.head_dim, self.heads, self.n_pages, self.page_size = int(head_dim), int(heads), int(n_pages), int(page_size)
        self._struct = _Cache(n_pages=self.n_pages, heads=self.heads, page_size=self.page_size)
        self._ref = _c.byref(self._struct)
        self._h = self.codec._h
        api.check(self._lib.pbz_cache_layout(self._h, self._ref, None, None))
        self.pages = Pages(self.n_pages, self.page_size)
        torch = api._torch()
        if pools is None:
            pools = [torch.zeros(shape, dtype=dtype, device=device) for shape, dtype in self.pool_shapes]
        for pool, (shape, dtype) in zip(pools, self.pool_shapes):
            if pool.dtype != dtype or tuple(pool.shape) != shape:
                raise ValueError(f"a pool has to be {dtype} of shape {shape}, not {pool.dtype} of {tuple(pool.shape)}")
        self.pools = self.k_N, self.k_F, self.v_N, self.v_F = tuple(pools)
        for name, pool in zip(("k_N", "k_F", "v_N", "v_F"), self.pools):
            setattr(self._struct, name, api._ptr(pool))
        self.device = self.k_N.device
        self._own = threading.local()     # of each thread: stream -> workspace, its bytes.  (A call is several launches through it.)
        # for the native side of the calls: entry points, codec and pools, and what tensors are held against
        self._append, self._copy, self._attend = (self._lib.addresses["pbz_cache_" + name] for name in ("append", "copy_pages", "attend"))
        self._handle, self._at = self._h.value, _c.addressof(self._struct)
        self._held = (self.device, torch.int32, torch.int64, torch.float32, self.heads, self.head_dim)
        self._need = {}              # sizes of an attention call -> bytes of its workspace

    @property
    def pool_shapes(self):
        torch = api._torch()
        lines = (self.n_pages, self.heads, self.page_size)
        n_type = api._torch_ftype(self.codec.work_type)
        return [(lines, n_type), (lines + (self.head_dim,), torch.int8)] * 2

    # ---- calls on tensors (checked and handed over by csrc/pbz_binding.c) --------------------
    def append(self, k, v, slots) -> None:
        """pbz_cache_append: compress keys and values [tokens, heads, head_dim] into their slots (int64, device;
        page * page_size + place, -1 leaves a token out)."""
        type_ = api._FTYPE_OF.get(k.dtype)
        if type_ is None or v.dtype != k.dtype:
            raise ValueError("keys and values have to be of one float type")
        api.check(api._binding.cache_append(self._append, self._handle, self._at, self._held, type_, k, v, slots))

    def copy_pages(self, pairs) -> None:
        """pbz_cache_copy_pages: pairs [n, 2] (from, to), on the host."""
        pairs = _pairs(pairs)
        if len(pairs):
            api.check(api._binding.cache_copy(self._copy, self._handle, self._at, pairs))

    def attend(self, q, table, lengths, starts=None, max_new: Optional[int] = None, max_length: int = 0,
               causal: bool = True, window: int = 0, scale: Optional[float] = None, out=None, lse=None, workspace=None):
        """pbz_cache_attend: q [tokens, query heads, head_dim] (bfloat16 or float16) over the cache -> out, alike.

        table [sequences, pages] and lengths [sequences], int32; starts [sequences + 1] int32, the rows of each
        sequence's new tokens (None: one token a sequence).  max_new, max_length: the host's bounds of the runs of new
        tokens and of the lengths, by which the work is dealt out (defaults: all tokens; the table's width).
        lse: float32 [tokens, query heads], written.  scale: 1 / sqrt(head_dim) when None.  workspace: the cache's own, one for every
        thread and stream, when None; a call that is captured into a graph has to be given one."""
        if q.dim() != 3:
            raise ValueError("q has to be [tokens, query heads, head_dim]")
        torch = api._torch()
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif out.dtype != q.dtype:
            raise ValueError("out has to be of q's type")
        args = _Attention()
        api._binding.cache_attention(args, self._held, q, out, lse, starts, lengths, table)
        tokens = args.n_tokens
        if tokens == 0:
            return out
        args.type = api._FTYPE_OF.get(q.dtype, -1)
        args.max_new = tokens if max_new is None else int(max_new)
        args.max_length, args.causal, args.window = int(max_length), 1 if causal else 0, int(window)
        args.scale = 1.0 / math.sqrt(self.head_dim) if scale is None else float(scale)
        if workspace is None:
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a graph's call has to be given its workspace: the cache's own is replaced when a later call needs more")
            sizes = (tokens, args.q_heads, args.n_seqs, args.max_pages, args.max_new, args.max_length, args.window, starts is None, args.type)
            need = self._need.get(sizes)
            if need is None:
                need = self.workspace_bytes(args)
                if len(self._need) < 256:
                    self._need[sizes] = need
            stream = api._stream()
            spaces = self._own.__dict__
            workspace, room = spaces.get(stream, (None, 0))
            if room < need:
                workspace, room = spaces[stream] = torch.empty(need, dtype=torch.uint8, device=self.device), need
        else:
            room = workspace.numel() * workspace.element_size()
        api.check(api._binding.cache_attend(self._attend, self._handle, self._at, args, workspace, room))
        return out

    def workspace_bytes(self, args: _Attention) -> int:
        need = _c.c_size_t()
        api.check(self._lib.pbz_cache_attend_workspace(self._h, self._ref, _c.byref(args), _c.byref(need)))
        return need.value

    # ---- sequences -------------------------------------------------------------------------
    def open(self) -> int:
        """A new, empty sequence."""
        return self.pages.open()

    def fork(self, sequence: int) -> int:
        """A sequence that shares all of `sequence`'s pages; whichever is written first gets a copy of the last one."""
        return self.pages.fork(sequence)

    def close(self, sequence: int) -> None:
        """Let a sequence's pages go."""
        self.pages.close(sequence)

    def truncate(self, sequence: int, length: int) -> None:
        self.pages.truncate(sequence, length)

    def length(self, sequence: int) -> int:
        return self.pages.length(sequence)

    def compact(self) -> int:
        """Bring the pages in use to the front of the pools; returns how many were moved."""
        pairs = self.pages.compact()
        self.copy_pages(pairs)
        return len(pairs)

    def extend_and_append(self, sequences: Sequence[int], counts: Sequence[int], k, v) -> None:
        """Append the next counts[b] tokens of each sequence; their rows follow one another in k and v.  Where that is refused, the sequences
        are as they were."""
        torch = api._torch()
        if len(sequences) != len(counts) or sum(counts) != k.shape[0]:
            raise ValueError("counts have to name every row of k, sequence by sequence")
        if len(set(sequences)) != len(sequences):
            raise ValueError("a sequence is named twice")
        slots: List[np.ndarray] = []
        before = [(seq, self.pages.length(seq)) for seq in sequences]
        try:
            for seq, count in zip(sequences, counts):
                if count == 0:
                    continue
                found, copy = self.pages.extend(seq, count)
                if copy:
                    self.copy_pages([copy])      # at once: the page copied to may be copied from by the next
                slots.append(found)
            if slots:
                self.append(k, v, torch.from_numpy(np.concatenate(slots)).to(self.device))
        except BaseException:                    # too few pages, or lines that are refused: the sequences stay as long as they were
            for seq, length in before:
                self.pages.truncate(seq, length)
            raise

    def tables(self, sequences: Sequence[int]):
        """(table, lengths) of the sequences, on the device, for `attend`."""
        torch = api._torch()
        lengths = [self.pages.length(s) for s in sequences]
        width = max([1] + [-(-n // self.page_size) for n in lengths])
        table = np.empty((len(lengths), width), dtype=np.int32)
        for row, s in zip(table, sequences):
            row[:] = self.pages.table(s, width)
        return torch.from_numpy(table).to(self.device), torch.tensor(lengths, dtype=torch.int32).to(self.device)

    def attend_sequences(self, sequences: Sequence[int], counts: Sequence[int], q, **options):
        """Attention of the last counts[b] tokens of each sequence (appended before); rows as in extend_and_append."""
        torch = api._torch()
        if len(sequences) != len(counts) or sum(counts) != q.shape[0] or min(counts, default=0) < 0:
            raise ValueError("counts have to name every row of q, sequence by sequence")
        table, lengths = self.tables(sequences)
        starts = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(self.device)
        return self.attend(q, table, lengths, starts=starts, max_new=max(counts, default=0) or 1, **options)
