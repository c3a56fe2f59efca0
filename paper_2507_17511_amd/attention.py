"""Attention over exchanged keys and values: device-memory plumbing around the C entry points cf_kv_append, cf_attn_prompt,
cf_attn_paged and cf_attn_join, for torch tensors.  Checks types, shapes and devices, allocates outputs that are not given,
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
from typing import Optional, Sequence

import torch

import paper_2507_17511_amd as cf

_CF_DT = {torch.bfloat16: cf.CF_BF16, torch.float16: cf.CF_F16, torch.float32: cf.CF_F32}

# The arguments of a call, as one struct.pack writes them: filling a ctypes structure field by field takes several times as long
# as the call itself.  A cf_rows is "Pqq".  What is packed is the call's own, so that threads may call at once: the interpreter's lock is free during a call.
_APPEND = struct.Struct("@q Pqq Pqq P Pqq Pqq PPP q ii")
_PROMPT = struct.Struct("@ii qqq PP Pqq Pqq Pqq Pqq P")
_PAGED = struct.Struct("@ii qq PP Pqq Pqq P")
_JOIN = struct.Struct("@ii q PP Pqq P")
for _layout, _args in ((_APPEND, cf.cf_append), (_PROMPT, cf.cf_prompt), (_PAGED, cf.cf_paged), (_JOIN, cf.cf_join)):
    assert _layout.size == ctypes.sizeof(_args), _args


def _entries() -> types.SimpleNamespace:
    """The library's entry points, with packed arguments as bytes."""
    desc, cache, args, workspace, stream = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_char_p, (ctypes.c_void_p, ctypes.c_size_t), ctypes.c_void_p
    takes = {"cf_kv_append": (desc, cache, args, stream), "cf_attn_prompt": (desc, args, *workspace, stream),
             "cf_attn_paged": (desc, cache, args, *workspace, stream), "cf_attn_join": (desc, args, stream)}
    return types.SimpleNamespace(**{name: ctypes.CFUNCTYPE(ctypes.c_int32, *given)((name, cf.lib())) for name, given in takes.items()})


# device index -> hipStream_t, without a Stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_written = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)     # [tensors]: autograd notices where it had kept one of them
_NO_GRADIENT = "has no gradient: call under torch.no_grad() or torch.inference_mode(), or detach it"


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


class PagedCache:
    """Pages of keys and values: two tensors [pages, kv_heads, page_size, head_dim], dense within a page.  They may be views
    of one tensor, [pages, 2, ...] say, or of one that holds all layers."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _require(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device, "k and v are [pages, kv_heads, page_size, head_dim], alike")
        pages, heads, page, dim = k.shape
        for x in (k, v):
            _require(x.numel() > 0 and x[0].is_contiguous() and (pages == 1 or x.stride(0) == k.stride(0) >= heads * page * dim),
                     "pages are dense, do not overlap, and are as far apart in k as in v")
        _require(not ((k.requires_grad or v.requires_grad) and torch.is_grad_enabled()), f"a cache {_NO_GRADIENT}")
        self.k, self.v = k, v
        self.heads, self.page_size, self.head_dim, self.dtype, self.index = heads, page, dim, k.dtype, k.get_device()
        self.struct = cf.cf_kv_cache(k.data_ptr(), v.data_ptr(), pages, k.stride(0) if pages > 1 else 0, page)
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page_size: int = 64, dtype: torch.dtype = torch.bfloat16,
              device: str | torch.device = "cuda:0") -> "PagedCache":
        kv = torch.empty((2, pages, kv_heads, page_size, head_dim), dtype=dtype, device=device)
        return cls(kv[0], kv[1])


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

    def append(self, cache: PagedCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
               cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, interleaved: bool = False) -> Optional[torch.Tensor]:
        """Stores k and v at `slots` (int64) of the cache, k (and q) rotated by `positions` (int32), rows of cos and sin
        [n_positions, rotary_dim / 2] (fp32); without positions nothing is rotated.  Returns the rotated queries, if any: in q_out,
        which may be q."""
        n = k.shape[0]
        rows_q = rows_out = (0, 0, 0)
        written = [cache.k, cache.v]
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
        self._call(self._lib.cf_kv_append, "cf_kv_append", self._desc, self._cache(cache), args)
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
