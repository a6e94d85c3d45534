"""Attention over a paged key-value cache: what a decoder block's step does between its projections.

``PagedCache`` is the cache with its bookkeeping: sequences that own pages, grow, are forked (sharing pages until one of
them writes), cut and freed, and the pool compacted. ``PagedAttention`` is the module: it writes a step's keys and values
into the cache and attends over it (operators ``usp::cache_append`` and ``usp::paged_attention``). All of it is for
inference: nothing here has a backward pass.

    cache = PagedCache(pages=4096, kv_heads=8, head_dim=128, layers=80)
    attend = PagedAttention(heads=64, kv_heads=8, head_dim=128)
    sequence = cache.add()
    rows = cache.extend([sequence], [prompt_tokens])
    for layer in range(80):
        y = attend(q, cache, rows, k, v, layer=layer)
"""
from __future__ import annotations

import heapq
from typing import List, Optional, Sequence

import torch

from . import usp
from .linear import Workspaces, _operand, _seen


class OutOfPages(RuntimeError):
    """The cache has fewer free pages than a call needs; nothing was changed."""


class PagedCache(usp.KVCache):
    """A cache whose pages belong to sequences (arguments as usp.KVCache).

    Sequences are numbered by ``add`` and ``fork``. The bookkeeping is the host's and immediate; copies of pages are enqueued on
    the current stream, and a page that one call gives back the next may hand out: keep a cache's calls on one
    stream, or order the streams. Not for several threads at once."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self._free = list(range(self.pages))  # a heap: the lowest page first
        self._users = [0] * self.pages
        self._pages: dict[int, List[int]] = {}
        self._lengths: dict[int, int] = {}
        self._next = 0

    # ---- sequences

    @property
    def free_pages(self) -> int:
        return len(self._free)

    @property
    def sequences(self) -> List[int]:
        return list(self._pages)

    def length(self, sequence: int) -> int:
        return self._lengths[self._known(sequence)]

    def pages_of(self, sequence: int) -> List[int]:
        return list(self._pages[self._known(sequence)])

    def _known(self, sequence: int) -> int:
        if sequence not in self._pages:
            raise KeyError(f"no sequence {sequence} in the cache")
        return sequence

    def add(self) -> int:
        """A new sequence without tokens."""
        sequence, self._next = self._next, self._next + 1
        self._pages[sequence], self._lengths[sequence] = [], 0
        return sequence

    def fork(self, sequence: int) -> int:
        """A new sequence with the tokens of another. They share its pages; the first of them to grow into a shared page
        gets a copy of it."""
        pages, length = self._pages[self._known(sequence)], self._lengths[sequence]
        new = self.add()
        self._pages[new], self._lengths[new] = list(pages), length
        for p in pages:
            self._users[p] += 1
        return new

    def _give_back(self, pages: Sequence[int]) -> None:
        for p in pages:
            self._users[p] -= 1
            if self._users[p] == 0:
                heapq.heappush(self._free, p)

    def free(self, sequence: int) -> None:
        """Ends a sequence; pages that no other has are free again."""
        pages = self._pages.pop(self._known(sequence))
        del self._lengths[sequence]
        self._give_back(pages)

    def truncate(self, sequence: int, length: int) -> None:
        """Cuts a sequence to its first `length` tokens."""
        if not 0 <= length <= self.length(sequence):
            raise ValueError(f"a sequence of {self.length(sequence)} tokens cannot be cut to {length}")
        pages, keep = self._pages[sequence], -(-length // self.page_tokens)
        self._pages[sequence], self._lengths[sequence] = pages[:keep], length
        self._give_back(pages[keep:])

    def extend(self, sequences: Sequence[int], tokens: Optional[Sequence[int]] = None) -> usp.CacheRows:
        """Room for `tokens` new tokens of each sequence (default: one), and the step's rows: append their keys and values
        in every layer before anything reads them. Raises OutOfPages, and changes nothing, where pages lack."""
        sequences = [self._known(s) for s in sequences]
        counts = [1] * len(sequences) if tokens is None else [int(n) for n in tokens]
        if len(set(sequences)) != len(sequences):
            raise ValueError("a sequence is named twice")
        if len(counts) != len(sequences) or min(counts, default=0) < 0:
            raise ValueError("tokens must be one count >= 0 for each sequence")
        capacity = (2**31 - 1 - 4096) // self.page_tokens * self.page_tokens
        new, copies, users = [], [], {}  # users: pages that this call changes the number of users of
        for s, n in zip(sequences, counts):
            length, pages = self._lengths[s], self._pages[s]
            if length + n > capacity:
                raise ValueError(f"a sequence holds at most {capacity} tokens")
            new.append(-(-(length + n) // self.page_tokens) - len(pages))
            if n and length % self.page_tokens:
                last = pages[-1]
                left = users.get(last, self._users[last])
                if left > 1:  # of the sequences that grow in this step the last one of a page keeps it
                    users[last] = left - 1
                    copies.append(s)
        if sum(new) + len(copies) > len(self._free):
            raise OutOfPages(f"{sum(new) + len(copies)} pages needed, {len(self._free)} free")
        src, dst = [], []
        for s in copies:
            page = heapq.heappop(self._free)
            src.append(self._pages[s][-1])
            dst.append(page)
            self._users[page] = 1
            self._users[src[-1]] -= 1
            self._pages[s][-1] = page
        for s, n, add in zip(sequences, counts, new):
            for _ in range(add):
                page = heapq.heappop(self._free)
                self._users[page] = 1
                self._pages[s].append(page)
            self._lengths[s] += n
        if src:
            self.copy(src, dst)
        return self.rows(sequences, counts)

    def compact(self) -> int:
        """Moves the pages in use to the lowest numbers (one copy of each that moves) and returns how many they are.
        Rows made before name the old pages."""
        used = self.pages - len(self._free)
        holes = sorted(p for p in self._free if p < used)
        above = [p for p in range(used, self.pages) if self._users[p]]
        if holes:
            self.copy(above, holes)
        moved = dict(zip(above, holes))
        for old, page in moved.items():
            self._users[page], self._users[old] = self._users[old], 0
        for s, pages in self._pages.items():
            self._pages[s] = [moved.get(p, p) for p in pages]
        self._free = list(range(used, self.pages))
        return used

    # ---- steps

    def _step(self, sequences: Sequence[int], tokens: Optional[Sequence[int]]):
        """(tables, lengths, offsets) of a step as host lists."""
        counts = [1] * len(sequences) if tokens is None else [int(n) for n in tokens]
        if not sequences or len(counts) != len(sequences):
            raise ValueError("a step has at least one sequence, and one count for each")
        offsets = [0]
        for s, n in zip(sequences, counts):
            if not 0 <= n <= self.length(s):
                raise ValueError(f"sequence {s} of {self.length(s)} tokens has no {n} last ones")
            offsets.append(offsets[-1] + n)
        return [self._pages[s] for s in sequences], [self._lengths[s] for s in sequences], offsets

    def _upload(self, values: List[int]) -> torch.Tensor:
        """int32 values on the cache's GPU, without waiting for it."""
        return torch.tensor(values, dtype=torch.int32).pin_memory().to(self.data.device, non_blocking=True)

    def rows(self, sequences: Sequence[int], tokens: Optional[Sequence[int]] = None) -> usp.CacheRows:
        """The last `tokens` tokens of each sequence (default: one) as a step's rows."""
        pages, lengths, offsets = self._step(sequences, tokens)
        S, most = len(pages), max(1, max(map(len, pages)))
        flat = [p for own in pages for p in own + [0] * (most - len(own))] + lengths + offsets
        on_gpu = self._upload(flat)
        table, lengths, offsets = on_gpu[:S * most].view(S, most), on_gpu[S * most:S * most + S], on_gpu[S * most + S:]
        single = tokens is None or all(int(n) == 1 for n in tokens)
        return usp.CacheRows(table, lengths, None if single else offsets)

    def update(self, rows: usp.CacheRows, sequences: Sequence[int], tokens: Optional[Sequence[int]] = None) -> None:
        """Writes a step into the tensors of `rows`, which a captured graph reads: as many sequences, a table as wide as the
        longest needs, and offsets if the step is not one token each."""
        pages, lengths, offsets = self._step(sequences, tokens)
        S, width = rows.table.shape
        if len(pages) != S or max(map(len, pages)) > width:
            raise ValueError(f"the rows have room for {S} sequences of {width} pages")
        if rows.offsets is None and offsets != list(range(S + 1)):
            raise ValueError("the rows are of one token for each sequence")
        on_gpu = self._upload([p for own in pages for p in own + [0] * (width - len(own))] + lengths + offsets)
        rows.table.copy_(on_gpu[:S * width].view(S, width))
        rows.lengths.copy_(on_gpu[S * width:S * width + S])
        if rows.offsets is not None:
            rows.offsets.copy_(on_gpu[S * width + S:])


# ---- the operators


def _cache_of(data: torch.Tensor, geometry: List[int]) -> usp.KVCache:
    kv_heads, head_dim, page_tokens, eight_bit = geometry
    return usp.KVCache(data.shape[1], kv_heads, head_dim, page_tokens, data.shape[0], torch.int8 if eight_bit else torch.float16,
                       data=data)


def _geometry(cache: usp.KVCache) -> List[int]:
    return [cache.kv_heads, cache.head_dim, cache.page_tokens, int(cache.dtype is torch.int8)]


def _attend(cache: usp.KVCache, rows: usp.CacheRows, q: torch.Tensor, workspace: Optional[torch.Tensor], layer: int,
            scale: Optional[float], cap: float, slopes: Optional[torch.Tensor], window: int, first: Optional[torch.Tensor],
            last: Optional[torch.Tensor]) -> torch.Tensor:
    out = q.new_empty(q.shape) if rows.offsets is None else q.new_zeros(q.shape)  # offsets may leave rows out
    usp.usp_attention(cache, rows, q, out, workspace, layer, scale, cap, slopes, window, first, last)
    return out


@torch.library.custom_op("usp::paged_attention", mutates_args=("workspace",))
def paged_attention(q: torch.Tensor, data: torch.Tensor, geometry: List[int], table: torch.Tensor, lengths: torch.Tensor,
                    offsets: Optional[torch.Tensor], workspace: Optional[torch.Tensor], layer: int, scale: Optional[float],
                    cap: float, slopes: Optional[torch.Tensor], window: int, first: Optional[torch.Tensor],
                    last: Optional[torch.Tensor]) -> torch.Tensor:
    """usp_attention of q [T, heads, head_dim] over the cache whose memory is `data`; geometry: kv_heads, head_dim,
    page_tokens and whether it holds 8-bit values."""
    return _attend(_cache_of(data, geometry), usp.CacheRows(table, lengths, offsets), q, workspace, layer, scale, cap, slopes,
                   window, first, last)


@paged_attention.register_fake
def _(q, data, geometry, table, lengths, offsets, workspace, layer, scale, cap, slopes, window, first, last):
    return q.new_empty(q.shape, dtype=torch.float16)


@torch.library.custom_op("usp::cache_append", mutates_args=("data",))
def cache_append(k: torch.Tensor, v: torch.Tensor, data: torch.Tensor, geometry: List[int], table: torch.Tensor,
                 lengths: torch.Tensor, offsets: Optional[torch.Tensor], layer: int) -> None:
    """usp_cache_append of k and v [T, kv_heads, head_dim] into the cache whose memory is `data`."""
    usp.usp_cache_append(_cache_of(data, geometry), usp.CacheRows(table, lengths, offsets), k, v, layer)


@cache_append.register_fake
def _(k, v, data, geometry, table, lengths, offsets, layer):
    return None


def _heads(x: torch.Tensor, heads: int, dim: int, name: str) -> torch.Tensor:
    """x [T, heads, dim] or [T, heads * dim] as fp16 [T, heads, dim] with unit inner stride."""
    if x.dim() == 2 and x.shape[1] == heads * dim:
        x = x.unflatten(1, (heads, dim))
    if x.dim() != 3 or x.shape[1] != heads or x.shape[2] != dim:
        raise ValueError(f"{name} must be [T, {heads}, {dim}] or [T, {heads * dim}], got {tuple(x.shape)}")
    if x.dtype is not torch.float16 or x.stride(2) != 1:
        x = x.to(torch.float16).contiguous()
    return x


class _DeviceWorkspaces(Workspaces):
    """The workspaces of calls on one GPU."""

    def __init__(self, device: int):
        self.device = device
        self._no_workspaces()

    def _stream(self) -> int:
        return usp.current_stream_handle(self.device)


class PagedAttention(torch.nn.Module):
    """Attention of a step's rows over a paged cache: softmax(bias(cap(scale q K^T))) V with the keys that each row sees.

    heads, kv_heads, head_dim: of q and of the cache (each of its heads serves heads / kv_heads of q's); scale: default
    head_dim ** -0.5; cap: scores become cap * tanh(score / cap) (0: not); slopes: [heads], scores lose slope * distance (None:
    not); window: a row sees its last `window` tokens (0: all); device: of the slopes (default: theirs, or the current GPU).

    Calls and captured graphs may overlap as SparseLinear's may."""

    def __init__(self, heads: int, kv_heads: int, head_dim: int, scale: Optional[float] = None, cap: float = 0.0,
                 slopes: Optional[torch.Tensor] = None, window: int = 0, device=None):
        super().__init__()
        if kv_heads < 1 or heads < 1 or heads % kv_heads:
            raise ValueError(f"heads must be a multiple of kv_heads, got {heads} and {kv_heads}")
        if slopes is not None and tuple(slopes.shape) != (heads,):
            raise ValueError(f"slopes must be [{heads}]")
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.scale, self.cap, self.window = scale, cap, window
        if slopes is not None:
            dev = f"cuda:{device}" if isinstance(device, int) else device or (slopes.device if slopes.is_cuda else "cuda")
            slopes = slopes.detach().to(device=dev, dtype=torch.float32).contiguous()
        self.register_buffer("slopes", slopes)
        self._spaces: dict[int, _DeviceWorkspaces] = {}

    def _apply(self, fn, recurse=True):
        """Moves and casts: slopes stay fp32, as the kernels take them, in a model that is cast."""
        slopes = self._buffers["slopes"]
        super()._apply(fn, recurse)
        if slopes is not None and self._buffers["slopes"].dtype is not torch.float32:
            self._buffers["slopes"] = slopes.to(self._buffers["slopes"].device)
        return self

    def forward(self, q: torch.Tensor, cache: usp.KVCache, rows: usp.CacheRows, k: Optional[torch.Tensor] = None,
                v: Optional[torch.Tensor] = None, layer: int = 0, first: Optional[torch.Tensor] = None,
                last: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q [T, heads, head_dim] or [T, heads * head_dim]; the result has its shape, in fp16. k, v: the rows' keys and values
        [T, kv_heads, head_dim] or [T, kv_heads * head_dim], written into the cache first; None where they are there already.
        first, last: int32 [T], the keys first <= j < last that each row sees (default: 0 and its own place + 1). Rows that no
        sequence has are zeros."""
        if cache.kv_heads != self.kv_heads or cache.head_dim != self.head_dim:
            raise ValueError(f"the cache holds {cache.kv_heads} heads of {cache.head_dim}, not {self.kv_heads} of {self.head_dim}")
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        q3 = _heads(q, self.heads, self.head_dim, "q")
        T = q3.shape[0]
        if T == 0:
            return q.to(torch.float16)
        slopes = self._buffers["slopes"]
        seen = _seen((q, k, v, first, last))
        if k is not None:
            k3, v3 = _heads(k, self.kv_heads, self.head_dim, "k"), _heads(v, self.kv_heads, self.head_dim, "v")
            if seen:
                torch.ops.usp.cache_append(k3, v3, cache.data, _geometry(cache), rows.table, rows.lengths, rows.offsets, layer)
            else:
                usp.usp_cache_append(cache, rows, k3, v3, layer)
        ws = self._workspace_of(cache, rows, T)
        if seen:
            out = torch.ops.usp.paged_attention(q3, cache.data, _geometry(cache), rows.table, rows.lengths, rows.offsets,
                                                _operand(ws, q3), layer, self.scale, self.cap, slopes, self.window, first, last)
        else:
            out = _attend(cache, rows, q3, ws, layer, self.scale, self.cap, slopes, self.window, first, last)
        return out if q.dim() == 3 else out.flatten(1)

    def _workspace_of(self, cache: usp.KVCache, rows: usp.CacheRows, T: int) -> Optional[torch.Tensor]:
        spaces = self._spaces.get(cache.device) or self._spaces.setdefault(cache.device, _DeviceWorkspaces(cache.device))
        return spaces._workspace(cache.workspace_size(rows, T, self.heads), lambda: cache.make_workspace(rows, T, self.heads))

    def extra_repr(self) -> str:
        return (f"heads={self.heads}, kv_heads={self.kv_heads}, head_dim={self.head_dim}, scale={self.scale}, cap={self.cap}, "
                f"slopes={self.slopes is not None}, window={self.window}")
