"""Attention over exchanged keys and values, and serving from a cache of them: device-memory plumbing around the C entry points cf_kv_append, cf_attn_prompt,
cf_attn_paged and cf_attn_join, and around those of the cache in 8 bits, cf_kv_plan, cf_kv_append8, cf_attn_select and cf_attn_paged8, for torch tensors.  Checks types, shapes and devices, allocates outputs that are not given,
and keeps a workspace.  No arithmetic happens here, and nothing has a gradient: tensors that want one are refused while gradients are
recorded.

Queries, keys, values and outputs are [tokens, heads, head_dim] with the last dimension contiguous; tokens and heads may be
strided (slices of a wider projection).  Calls enqueue work on the session's stream, or on torch's current one, and return.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct
import threading
import types
from typing import NamedTuple, Optional, Sequence

import torch

import paper_2507_17511_amd as cf

_CF_DT = {torch.bfloat16: cf.CF_BF16, torch.float16: cf.CF_F16, torch.float32: cf.CF_F32}

# The arguments of a call, as one struct.pack writes them: filling a ctypes structure field by field takes several times as long
# as the call itself.  A cf_rows is "Pqq".  What is packed is the call's own, so that threads may call at once: the interpreter's lock is free during a call.
_APPEND = struct.Struct("@q Pqq Pqq P Pqq Pqq PPP q ii")
_PROMPT = struct.Struct("@ii qqq PP Pqq Pqq Pqq Pqq P")
_PAGED = struct.Struct("@ii qq PP Pqq Pqq P")
_JOIN = struct.Struct("@ii q PP Pqq P")
_BLOCKS = struct.Struct("@P i4x")
_SELECT = struct.Struct("@ii qq PP Pqq iii4x P")
_PLAN = struct.Struct("@iiii qq PPPPPPPPPPP")
for _layout, _args in ((_APPEND, cf.cf_append), (_PROMPT, cf.cf_prompt), (_PAGED, cf.cf_paged), (_JOIN, cf.cf_join), (_BLOCKS, cf.cf_blocks),
                       (_SELECT, cf.cf_select), (_PLAN, cf.cf_plan)):
    assert _layout.size == ctypes.sizeof(_args), _args


def _entries() -> types.SimpleNamespace:
    """The library's entry points, with packed arguments as bytes."""
    desc, cache, args, workspace, stream = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_char_p, (ctypes.c_void_p, ctypes.c_size_t), ctypes.c_void_p
    takes = {"cf_kv_append": (desc, cache, args, stream), "cf_attn_prompt": (desc, args, *workspace, stream),
             "cf_attn_paged": (desc, cache, args, *workspace, stream), "cf_attn_join": (desc, args, stream), "cf_kv_append8": (desc, cache, args, stream),
             "cf_attn_paged8": (desc, cache, args, args, *workspace, stream), "cf_attn_select": (desc, cache, args, *workspace, stream), "cf_kv_plan": (args, *workspace, stream)}
    return types.SimpleNamespace(**{name: ctypes.CFUNCTYPE(ctypes.c_int32, *given)((name, cf.lib())) for name, given in takes.items()})


# device index -> hipStream_t, without a Stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_written = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)     # [tensors]: autograd notices where it had kept one of them
_NO_GRADIENT = "has no gradient: call under torch.no_grad() or torch.inference_mode(), or detach it"


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


class _Held:
    """Tensors that calls know by their addresses.  One that is put in another's place is checked as the first ones were, and is what the next call is given."""
    _given: tuple = ()

    def __setattr__(self, name, x):
        if name in self._given:
            self.__init__(**{**{n: getattr(self, n) for n in self._given}, name: x})
        else:
            super().__setattr__(name, x)


class PagedCache(_Held):
    """Pages of keys and values: two tensors [pages, kv_heads, page_size, head_dim], dense within a page.  They may be views
    of one tensor, [pages, 2, ...] say, or of one that holds all layers."""
    _given = ("k", "v")

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _require(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device, "k and v are [pages, kv_heads, page_size, head_dim], alike")
        pages, heads, page, dim = k.shape
        for x in (k, v):
            _require(x.numel() > 0 and x[0].is_contiguous() and (pages == 1 or x.stride(0) == k.stride(0) >= heads * page * dim),
                     "pages are dense, do not overlap, and are as far apart in k as in v")
        _require(not ((k.requires_grad or v.requires_grad) and torch.is_grad_enabled()), f"a cache {_NO_GRADIENT}")
        vars(self).update(k=k, v=v)
        self.heads, self.page_size, self.head_dim, self.dtype, self.index = heads, page, dim, k.dtype, k.get_device()
        self.struct = cf.cf_kv_cache(k.data_ptr(), v.data_ptr(), pages, k.stride(0) if pages > 1 else 0, page)
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page_size: int = 64, dtype: torch.dtype = torch.bfloat16,
              device: str | torch.device = "cuda:0") -> "PagedCache":
        kv = torch.empty((2, pages, kv_heads, page_size, head_dim), dtype=dtype, device=device)
        return cls(kv[0], kv[1])


class PagedCache8(_Held):
    """Pages of 8-bit codes: two tensors [pages, kv_heads, page_size, head_dim] of torch.float8_e4m3fn, dense within a page, and their scales, two of
    torch.float32 [pages, kv_heads], powers of two.  bounds: torch.bfloat16 [pages, kv_heads, 2, head_dim], the least and the largest of each
    channel of a page's keys, which AttentionSession.select reads."""
    _given = ("k", "v", "k_scale", "v_scale", "bounds")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, bounds: Optional[torch.Tensor] = None):
        _require(k.dim() == 4 and k.shape == v.shape and k.dtype is v.dtype is torch.float8_e4m3fn and k.device == v.device,
                 "k and v are [pages, kv_heads, page_size, head_dim] of torch.float8_e4m3fn, alike")
        pages, heads, page, dim = k.shape
        for x in (k, v):
            _require(x.numel() > 0 and x[0].is_contiguous() and (pages == 1 or x.stride(0) == k.stride(0) >= heads * page * dim),
                     "pages are dense, do not overlap, and are as far apart in k as in v")
        for x in (k_scale, v_scale):
            _require(x.shape == (pages, heads) and x.dtype is torch.float32 and x.device == k.device and x.is_contiguous(), "scales are dense [pages, kv_heads] of torch.float32")
        _require(bounds is None or (bounds.shape == (pages, heads, 2, dim) and bounds.dtype is torch.bfloat16 and bounds.device == k.device and bounds.is_contiguous()),
                 "bounds are dense [pages, kv_heads, 2, head_dim] of torch.bfloat16")
        written = [x for x in (k, v, k_scale, v_scale, bounds) if x is not None]
        _require(not (any(x.requires_grad for x in written) and torch.is_grad_enabled()), f"a cache {_NO_GRADIENT}")
        vars(self).update(k=k, v=v, k_scale=k_scale, v_scale=v_scale, bounds=bounds, written=written)
        self.heads, self.page_size, self.head_dim, self.index = heads, page, dim, k.get_device()
        self.struct = cf.cf_kv_cache8(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), None if bounds is None else bounds.data_ptr(),
                                      pages, k.stride(0) if pages > 1 else 0, page)
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page_size: int = 64, bounds: bool = True, device: str | torch.device = "cuda:0") -> "PagedCache8":
        kv = torch.empty((2, pages, kv_heads, page_size, head_dim), dtype=torch.float8_e4m3fn, device=device)
        scales = torch.ones((2, pages, kv_heads), device=device)
        return cls(kv[0], kv[1], scales[0], scales[1], torch.zeros((pages, kv_heads, 2, head_dim), dtype=torch.bfloat16, device=device) if bounds else None)


class Plan(NamedTuple):
    slots: torch.Tensor         # int64 [tokens]: for append and append8
    positions: torch.Tensor     # int32 [tokens]
    cu: torch.Tensor            # int32 [sequences + 1]: where each sequence's tokens begin, as prompt takes it
    refused: torch.Tensor       # int32 [1]: sequences whose tokens are not served


class PageTables(_Held):
    """Which pages the sequences of a batch hold, table [sequences, max_pages] int32 and lens [sequences] int32, and which are free: pages ring[i % len(ring)] (int32),
    state[0] <= i < state[1] (int64 [2]: taken and put, ever).  All of it stays on the device; AttentionSession.plan updates it."""
    _given = ("table", "lens", "ring", "state", "page_size")

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, ring: torch.Tensor, state: torch.Tensor, page_size: int):
        _require(table.dim() == 2 and table.dtype is torch.int32 and table.shape[1] > 0 and (table.shape[1] == 1 or table.stride(1) == 1) and
                 (table.shape[0] < 2 or table.stride(0) >= table.shape[1]), "table is [sequences, pages] int32, its rows dense")
        for x, dtype, n, name in ((lens, torch.int32, table.shape[0], "lens"), (ring, torch.int32, ring.numel(), "ring"), (state, torch.int64, 2, "state")):
            _require(x.shape == (n,) and x.dtype is dtype and x.device == table.device and x.is_contiguous(), f"{name} is {n} dense values of {dtype} on {table.device}")
        vars(self).update(table=table, lens=lens, ring=ring, state=state, page_size=page_size)
        self.seqs, self.index = table.shape[0], table.get_device()
        self.head = (self.seqs, page_size, table.shape[1], ring.numel(), table.stride(0) if self.seqs > 1 else 0)
        self.at = (table.data_ptr(), ring.data_ptr(), state.data_ptr())

    @classmethod
    def empty(cls, seqs: int, max_pages: int, pages: int, page_size: int = 64, device: str | torch.device = "cuda:0") -> "PageTables":
        return cls(torch.zeros((seqs, max_pages), dtype=torch.int32, device=device), torch.zeros(seqs, dtype=torch.int32, device=device),
                   torch.arange(pages, dtype=torch.int32, device=device), torch.tensor([0, pages], dtype=torch.int64, device=device), page_size)


class AttentionSession:
    """The geometry of a model's attention on one device, and the workspace of its calls: one stream at a time, from any threads.  Calls go to the session's own
    stream, if it has one, or to the current one.  As with every stream but their own, tensors are kept until the work on them is done, or recorded on that stream; the workspace is."""

    def __init__(self, q_heads: int, kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, scale: float = 0.0,
                 device: str | torch.device = "cuda:0", stream: Optional[torch.cuda.Stream] = None,
                 workspace_bytes: int = cf.CF_ATTN_WORKSPACE_BYTES):
        _require(dtype in (torch.bfloat16, torch.float16), "dtype is torch.bfloat16 or torch.float16")
        self.q_heads, self.kv_heads, self.head_dim, self.dtype = q_heads, kv_heads, head_dim, dtype
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index if self.device.type == "cuda" else -1
        self.desc = cf.cf_attn_desc(_CF_DT[dtype], q_heads, kv_heads, head_dim, scale)
        self._lib = _entries()
        self._desc = ctypes.byref(self.desc)
        self.ws_bytes = workspace_bytes
        self._stream = stream
        self._handle = stream.cuda_stream if stream is not None else None if self._index >= 0 else 0       # None: torch's current one
        self._settled = set()       # streams on which there is nothing more to do for a call than to make it
        self.workspace = self._ws = None
        self._unset = False         # whether the workspace's zeros were captured into a graph, which is yet to run
        if workspace_bytes:         # memory of the session's stream, or else of the current one, and recorded on those that calls go to
            with torch.cuda.device(self._index), torch.cuda.stream(stream):
                self.workspace = torch.zeros(workspace_bytes, dtype=torch.uint8, device=self.device)
                self._unset = self._index >= 0 and torch.cuda.is_current_stream_capturing()
            self._ws = self.workspace.data_ptr()
            if stream is None and self._index >= 0 and not self._unset:
                torch.cuda.current_stream(self.device).synchronize()        # zeros on whichever stream the first call is
        self._one = threading.Lock() if workspace_bytes else contextlib.nullcontext()      # a call's kernels are enqueued one after another, as they share the workspace

    # The library launches on the device that is current, and the null stream, torch's default one, is that device's.
    def _call(self, entry, name: str, *args) -> None:
        on = _raw_stream(self._index) if self._handle is None else self._handle
        if on in self._settled and _current_device() == self._index:
            status = entry(*args, on)
        else:
            status = self._call_elsewhere(entry, args, on)
        if status:
            raise cf.CFError(status, name)

    # ... on a stream for the first time, or with another device current.
    def _call_elsewhere(self, entry, args, on: int) -> int:
        if self._index < 0:
            raise ValueError(f"attention runs on a GPU: the session's device is {self.device}")
        with torch.cuda.device(self._index):
            if on not in self._settled and self._stream is None and self.workspace is not None:
                self.workspace.record_stream(torch.cuda.current_stream(self.device))
            if self._unset:
                with torch.cuda.stream(self._stream):
                    self.workspace[:cf.CF_ATTN_COUNTER_BYTES].zero_()
                    self._unset = torch.cuda.is_current_stream_capturing()
            if not self._unset:
                self._settled.add(on)
            return entry(*args, on)

    # An output is memory of the stream that it is written on: of another's it might still be in use there.
    def _new(self, shape, dtype: torch.dtype) -> torch.Tensor:
        if self._stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self._stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    # What a call reads of its tensors is most of its time on the host: each attribute once, and those that tell a wrong tensor.
    def _rows(self, x: torch.Tensor, tokens: int, heads: int, name: str):
        """-> data, token stride, head stride."""
        if x.shape == (tokens, heads, self.head_dim) and x.dtype is self.dtype and x.get_device() == self._index:
            token, head, last = x.stride()
            if last == 1:
                if x.requires_grad and torch.is_grad_enabled():
                    raise ValueError(f"attention {_NO_GRADIENT} ({name})")
                return x.data_ptr(), token, head
        raise ValueError(f"{name} is [{tokens}, {heads}, {self.head_dim}] of {self.dtype} on {self.device}, the elements of a head next to one another: "
                         f"got {tuple(x.shape)} of {x.dtype} on {x.device}, strides {x.stride()}")

    def _list(self, x: torch.Tensor, dtype: torch.dtype, n: int, name: str) -> int:
        if x.numel() != n or x.dtype is not dtype or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name} is {n} dense values of {dtype} on {self.device}: got {tuple(x.shape)} of {x.dtype} on {x.device}")
        return x.data_ptr()

    def _plain(self, x: torch.Tensor, dtype: torch.dtype, shape, name: str) -> int:
        if x.shape != shape or x.dtype is not dtype or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name} is dense {tuple(shape)} of {dtype} on {self.device}: got {tuple(x.shape)} of {x.dtype} on {x.device}")
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"attention {_NO_GRADIENT} ({name})")
        return x.data_ptr()

    def _cache(self, cache: PagedCache):
        if cache.heads != self.kv_heads or cache.head_dim != self.head_dim or cache.dtype is not self.dtype or cache.index != self._index:
            raise ValueError(f"the cache has {self.kv_heads} heads of {self.head_dim} of {self.dtype} on {self.device}: got {cache.heads} of "
                             f"{cache.head_dim} of {cache.dtype} on {cache.k.device}")
        return cache.ref

    def _cache8(self, cache: PagedCache8):
        if cache.heads != self.kv_heads or cache.head_dim != self.head_dim or cache.index != self._index:
            raise ValueError(f"the cache has {self.kv_heads} heads of {self.head_dim} on {self.device}: got {cache.heads} of {cache.head_dim} on {cache.k.device}")
        return cache.ref

    def _pages(self, table: torch.Tensor, n: int):
        """-> its columns, and the stride of its rows."""
        shape = table.shape
        _require(len(shape) == 2 and shape[0] == n and table.dtype is torch.int32 and table.get_device() == self._index, "table is [sequences, pages] int32")
        row, entry = table.stride()
        cols = shape[1]
        _require((cols == 1 or entry == 1) and (n < 2 or row >= cols), "the rows of the table are dense and do not overlap")
        return cols, row if n > 1 else 0

    def _listed(self, blocks: torch.Tensor, n: int) -> int:
        shape = blocks.shape
        if len(shape) != 3 or shape[:2] != (n, self.kv_heads) or blocks.dtype is not torch.int32 or blocks.get_device() != self._index or not blocks.is_contiguous():
            raise ValueError(f"blocks are dense [{n}, {self.kv_heads}, count] of torch.int32 on {self.device}: got {tuple(shape)} of {blocks.dtype} on {blocks.device}")
        return blocks.data_ptr()

    def append(self, cache: PagedCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
               cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, interleaved: bool = False) -> Optional[torch.Tensor]:
        """Stores k and v at `slots` (int64) of the cache, k (and q) rotated by `positions` (int32), rows of cos and sin
        [n_positions, rotary_dim / 2] (fp32); without positions nothing is rotated.  Returns the rotated queries, if any: in q_out,
        which may be q."""
        return self._append(self._lib.cf_kv_append, "cf_kv_append", self._cache, cache, [cache.k, cache.v], k, v, slots, positions, cos, sin, q, q_out, interleaved)

    def append8(self, cache: PagedCache8, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
                cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                q_out: Optional[torch.Tensor] = None, interleaved: bool = False) -> Optional[torch.Tensor]:
        """append, into a cache of 8-bit codes.  Tokens that go to the same page are neighbours in the call; one at a page's first place
        begins the page anew."""
        return self._append(self._lib.cf_kv_append8, "cf_kv_append8", self._cache8, cache, cache.written.copy(), k, v, slots, positions, cos, sin, q, q_out, interleaved)

    def _append(self, entry, name: str, ref, cache, written, k, v, slots, positions, cos, sin, q, q_out, interleaved) -> Optional[torch.Tensor]:
        n = k.shape[0]
        rows_q = rows_out = (0, 0, 0)
        if q is not None:
            if q_out is not None:
                written.append(q_out)
            else:
                q_out = self._new(q.shape, self.dtype)
            rows_q = self._rows(q, n, self.q_heads, "q")
            rows_out = rows_q if q_out is q else self._rows(q_out, n, self.q_heads, "q_out")
        elif q_out is not None:
            raise ValueError("q_out goes with q")
        at = table = (0, 0, 0)
        if positions is not None:
            _require(cos is not None and sin is not None and cos.dim() == 2, "positions go with cos and sin [n_positions, rotary_dim / 2]")
            shape = cos.shape
            at = (self._list(positions, torch.int32, n, "positions"), self._plain(cos, torch.float32, shape, "cos"),
                  self._plain(sin, torch.float32, shape, "sin"))
            table = (shape[0], 2 * shape[1], interleaved)
        args = _APPEND.pack(n, *self._rows(k, n, self.kv_heads, "k"), *self._rows(v, n, self.kv_heads, "v"),
                            self._list(slots, torch.int64, n, "slots"), *rows_q, *rows_out, *at, *table)
        self._call(entry, name, self._desc, ref(cache), args)
        _written(written)
        return q_out

    def prompt(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: Optional[torch.Tensor] = None,
               causal: bool = True, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, max_k: int = 0) -> torch.Tensor:
        """Attention of packed sequences: sequence b has rows cu_q[b] .. cu_q[b + 1] of q and cu_k[b] .. of k and v (int32; cu_k is
        cu_q if not given).  `lse`: fp32 [tokens, q_heads], filled with the rows' log-sum-exps.  max_k: keys of the longest sequence, a hint."""
        n, n_q, n_k = cu_q.shape[0] - 1, q.shape[0], k.shape[0]
        if n < 0:
            raise ValueError("cu_q has an entry more than there are sequences")
        at_q = self._list(cu_q, torch.int32, n + 1, "cu_q")
        at_k = at_q if cu_k is None or cu_k is cu_q else self._list(cu_k, torch.int32, n + 1, "cu_k")
        given = () if out is None else (out,)
        if out is None:
            out = self._new(q.shape, self.dtype)
        args = _PROMPT.pack(n, causal, n_q, n_k, max_k, at_q, at_k, *self._rows(q, n_q, self.q_heads, "q"), *self._rows(k, n_k, self.kv_heads, "k"),
                            *self._rows(v, n_k, self.kv_heads, "v"), *self._rows(out, n_q, self.q_heads, "out"), 0 if lse is None else self._plain(lse, torch.float32, (n_q, self.q_heads), "lse"))
        with self._one:
            self._call(self._lib.cf_attn_prompt, "cf_attn_prompt", self._desc, args, self._ws, self.ws_bytes)
        if given or lse is not None:
            _written(given if lse is None else (*given, lse))
        return out

    def paged(self, cache: PagedCache, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, out: Optional[torch.Tensor] = None,
              lse: Optional[torch.Tensor] = None, max_len: int = 0) -> torch.Tensor:
        """Attention of one token per sequence, q [sequences, q_heads, head_dim], over its context: lens[b] tokens in the pages
        table[b] (int32 both).  max_len: the longest context, a hint."""
        n = q.shape[0]
        given = () if out is None else (out,)
        if out is None:
            out = self._new(q.shape, self.dtype)
        shape = table.shape
        _require(len(shape) == 2 and shape[0] == n and table.dtype is torch.int32 and table.get_device() == self._index, "table is [sequences, pages] int32")
        row, entry = table.stride()
        cols = shape[1]
        _require((cols == 1 or entry == 1) and (n < 2 or row >= cols), "the rows of the table are dense and do not overlap")
        args = _PAGED.pack(n, cols, row if n > 1 else 0, max_len, table.data_ptr(), self._list(lens, torch.int32, n, "lens"),
                         *self._rows(q, n, self.q_heads, "q"), *self._rows(out, n, self.q_heads, "out"),
                         0 if lse is None else self._plain(lse, torch.float32, (n, self.q_heads), "lse"))
        with self._one:
            self._call(self._lib.cf_attn_paged, "cf_attn_paged", self._desc, self._cache(cache), args, self._ws, self.ws_bytes)
        if given or lse is not None:
            _written(given if lse is None else (*given, lse))
        return out

    def select(self, cache: PagedCache8, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, count: int, first: int = 1, recent: int = 1,
               out: Optional[torch.Tensor] = None, max_len: int = 0) -> torch.Tensor:
        """The `count` pages of each context whose keys may score highest for the queries that share them, by the cache's bounds, among them its `first` and its
        `recent` (last) ones: int32 [sequences, kv_heads, count], in order, then -1.  For paged8; q, table, lens and max_len as there."""
        n = q.shape[0]
        given = out is not None
        if out is None:
            out = self._new((n, self.kv_heads, count), torch.int32)
        elif out.shape[2:] != (count,):
            raise ValueError(f"out is [{n}, {self.kv_heads}, {count}]: got {tuple(out.shape)}")
        _require(cache.bounds is not None, "the cache has no bounds")
        args = _SELECT.pack(n, *self._pages(table, n), max_len, table.data_ptr(), self._list(lens, torch.int32, n, "lens"), *self._rows(q, n, self.q_heads, "q"),
                            count, first, recent, self._listed(out, n))
        with self._one:
            self._call(self._lib.cf_attn_select, "cf_attn_select", self._desc, self._cache8(cache), args, self._ws, self.ws_bytes)
        if given:
            _written((out,))
        return out

    def paged8(self, cache: PagedCache8, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, blocks: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, max_len: int = 0) -> torch.Tensor:
        """paged, over a cache of 8-bit codes.  blocks (int32 [sequences, kv_heads, count]): which of its context's pages each head of keys is
        attended on, entries of its row of the table: as select gives them, the first ones count, and those outside of the context are none."""
        n = q.shape[0]
        given = () if out is None else (out,)
        if out is None:
            out = self._new(q.shape, self.dtype)
        args = _PAGED.pack(n, *self._pages(table, n), max_len, table.data_ptr(), self._list(lens, torch.int32, n, "lens"), *self._rows(q, n, self.q_heads, "q"),
                           *self._rows(out, n, self.q_heads, "out"), 0 if lse is None else self._plain(lse, torch.float32, (n, self.q_heads), "lse"))
        listed = None if blocks is None else _BLOCKS.pack(self._listed(blocks, n), blocks.shape[2])
        with self._one:
            self._call(self._lib.cf_attn_paged8, "cf_attn_paged8", self._desc, self._cache8(cache), args, listed, self._ws, self.ws_bytes)
        if given or lse is not None:
            _written(given if lse is None else (*given, lse))
        return out

    def plan(self, tables: PageTables, news: torch.Tensor, tokens: int, slots: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
             cu: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
             refused: Optional[torch.Tensor] = None) -> Plan:
        """Makes room for news[b] new tokens (int32) of every sequence, in order, while free pages suffice; -1 says that a sequence has ended, and its pages come
        back.  `tokens`: rows of slots and positions; those behind the last token, and those of sequences that are not served, are -1.
        The tables' table and ring are updated, and their lens and state, unless lens_out or state_out are given."""
        n = tables.seqs
        _require(tables.index == self._index, f"the tables are on {self.device}")
        slots = self._new((tokens,), torch.int64) if slots is None else slots
        positions = self._new((tokens,), torch.int32) if positions is None else positions
        cu = self._new((n + 1,), torch.int32) if cu is None else cu
        refused = self._new((1,), torch.int32) if refused is None else refused
        lens_out = tables.lens if lens_out is None else lens_out
        state_out = tables.state if state_out is None else state_out
        args = _PLAN.pack(*tables.head, tokens, tables.lens.data_ptr(), self._list(news, torch.int32, n, "news"), *tables.at,
                          self._list(state_out, torch.int64, 2, "state_out"), self._list(lens_out, torch.int32, n, "lens_out"),
                          self._list(cu, torch.int32, n + 1, "cu"), self._list(slots, torch.int64, tokens, "slots"),
                          self._list(positions, torch.int32, tokens, "positions"), self._list(refused, torch.int32, 1, "refused"))
        with self._one:
            self._call(self._lib.cf_kv_plan, "cf_kv_plan", args, self._ws, self.ws_bytes)
        _written((tables.table, tables.ring, lens_out, state_out, slots, positions, cu, refused))
        return Plan(slots, positions, cu, refused)

    def join(self, parts: Sequence[torch.Tensor], lses: Sequence[torch.Tensor], out: Optional[torch.Tensor] = None,
             lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention over the union of disjoint sets of keys: parts [tokens, q_heads, head_dim], all of the session's dtype or all fp32,
        and their log-sum-exps."""
        n = len(parts)
        _require(n > 0 and n == len(lses), "a log-sum-exp for every part, and one part at least")
        shape, pdt = parts[0].shape, parts[0].dtype
        if len(shape) != 3 or shape[1] != self.q_heads or shape[2] != self.head_dim or (pdt is not self.dtype and pdt is not torch.float32):
            raise ValueError(f"parts are [tokens, {self.q_heads}, {self.head_dim}] of {self.dtype} or torch.float32")
        tokens = shape[0]
        given = () if out is None else (out,)
        if out is None:
            out = self._new(shape, self.dtype)
        p = (ctypes.c_void_p * n)(*[self._plain(x, pdt, shape, "a part") for x in parts])
        s = (ctypes.c_void_p * n)(*[self._plain(x, torch.float32, shape[:2], "a log-sum-exp") for x in lses])
        args = _JOIN.pack(n, _CF_DT[pdt], tokens, ctypes.addressof(p), ctypes.addressof(s), *self._rows(out, tokens, self.q_heads, "out"),
                        0 if lse is None else self._plain(lse, torch.float32, shape[:2], "lse"))
        self._call(self._lib.cf_attn_join, "cf_attn_join", self._desc, args)
        if given or lse is not None:
            _written(given if lse is None else (*given, lse))
        return out
