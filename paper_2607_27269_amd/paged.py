"""Serving from a paged latent cache: pages, sequences that share them, and the calls on them.

``PageAllocator`` keeps, on the host, which pages of a pool each sequence owns or shares.
``PagedLatentCache`` adds the pools of all layers on the GPU and the calls of the C ABI that
work on them.  One model step over some sequences is a ``Batch``::

    batch = cache.batch(seqs, counts)             # pages reserved, tables uploaded
    for layer in range(n_layers):
        ...                                       # rows [c^KV | k^PE] and q of the new tokens
        q = batch.append(layer, rows, q, inv_freq)    # rotated, rows written to the pages
        o = batch.attend(layer, q, Wuk, Wuv)          # prefill or decode
    batch.commit()                                # the new tokens count as cached

The pools hold bf16 rows or, with ``format="e4m3"``, rows whose latents take eight bits (about half
the bytes, so twice the tokens and a quicker decoding; a latent is off by up to 2^-4 of itself).
Forked sequences share pages: a step of single tokens made with ``share=True`` attends to the
pages that neighbours in the batch have in common once for all of them, where that is quicker.

All device work is enqueued on the current HIP stream; calls from more than one stream are the
caller's to order (the layers of a batch share its workspace).
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import _lib as L


class OutOfPages(RuntimeError):
    """The pool has too few free pages; nothing was changed."""


class PageAllocator:
    """Pages of a pool and the sequences that hold them.

    A sequence holds ceil(length / page_size) pages in order.  Forked sequences share their
    pages; a page that is shared is never written: the first of its holders that grows into a
    shared, partly filled page gets a copy of it (``extend`` returns the page pairs to copy)."""

    def __init__(self, n_pages: int, page_size: int):
        if n_pages < 1 or page_size < 1:
            raise ValueError("n_pages and page_size must be positive")
        self.n_pages, self.page_size = n_pages, page_size
        self.holders = np.zeros(n_pages, dtype=np.int32)   # sequences that hold the page
        self.free_pages = list(range(n_pages - 1, -1, -1))  # the lowest page is taken first
        self.pages: dict[int, list[int]] = {}
        self.length: dict[int, int] = {}
        self._next = 0

    def _new(self, pages, length) -> int:
        seq, self._next = self._next, self._next + 1
        self.pages[seq], self.length[seq] = pages, length
        return seq

    def add(self) -> int:
        """A new, empty sequence."""
        return self._new([], 0)

    def fork(self, seq: int) -> int:
        """A new sequence with the same cached tokens, in the same pages."""
        pages = self.pages[seq][:-(-self.length[seq] // self.page_size)]  # none of those reserved
        for p in pages:
            self.holders[p] += 1
        return self._new(pages, self.length[seq])

    def _release(self, page: int):
        self.holders[page] -= 1
        if self.holders[page] == 0:
            self.free_pages.append(page)

    def truncate(self, seq: int, length: int):
        """Drop the tokens behind the first ``length`` (rejected drafts)."""
        if not 0 <= length <= self.length[seq]:
            raise ValueError(f"sequence {seq} has {self.length[seq]} tokens, not {length}")
        keep = -(-length // self.page_size)
        for p in self.pages[seq][keep:]:
            self._release(p)
        del self.pages[seq][keep:]
        self.length[seq] = length

    def free(self, seq: int):
        """Give up a sequence and the pages that nobody else holds."""
        self.truncate(seq, 0)
        del self.pages[seq], self.length[seq]

    def extend(self, seqs, counts, copy=None) -> list[tuple[int, int]]:
        """Room for counts[i] more tokens of seqs[i] (lengths stay as they are; pages reserved
        before are kept).  Returns the page pairs (from, to) to copy before anything is written
        to them; ``copy`` is called with them before anything here has changed (nothing has if it
        raises).  Raises OutOfPages, having changed nothing, if the pool has too few."""
        seqs, counts = list(seqs), [int(c) for c in counts]
        if len(set(seqs)) != len(seqs) or len(seqs) != len(counts):
            raise ValueError("one count for each of different sequences")
        if any(c < 0 for c in counts):
            raise ValueError("counts must not be negative")
        ps, shared, need = self.page_size, [], 0
        holders = {}   # of the shared pages, as the copies give them up
        for s, c in zip(seqs, counts):
            n, held = self.length[s], self.pages[s]
            need += max(0, -(-(n + c) // ps) - len(held))
            if c and n % ps:
                page = held[n // ps]
                k = holders.setdefault(page, int(self.holders[page]))
                if k > 1:
                    holders[page] = k - 1
                    shared.append((s, n // ps))
                    need += 1
        if need > len(self.free_pages):
            raise OutOfPages(f"{need} pages needed, {len(self.free_pages)} free")
        # (the pages that _take gives next)
        pairs = [(self.pages[s][at], self.free_pages[-1 - i]) for i, (s, at) in enumerate(shared)]
        if copy is not None:
            copy(pairs)
        for (s, at), (old, _) in zip(shared, pairs):
            self.pages[s][at] = self._take()
            self._release(old)
        for s, c in zip(seqs, counts):
            for _ in range(-(-(self.length[s] + c) // ps) - len(self.pages[s])):
                self.pages[s].append(self._take())
        return pairs

    def _take(self) -> int:
        page = self.free_pages.pop()
        self.holders[page] = 1
        return page

    def compact(self, copy=None) -> list[tuple[int, int]]:
        """Move the pages in use to the front of the pool.  Returns the page pairs (from, to) to
        copy (``copy`` as for ``extend``); afterwards pages >= the number in use are free."""
        used = np.flatnonzero(self.holders)
        holes = np.flatnonzero(self.holders[:len(used)] == 0)
        moved = dict(zip(used[used >= len(used)].tolist(), holes.tolist()))
        if copy is not None:
            copy(list(moved.items()))
        for pages in self.pages.values():
            pages[:] = [moved.get(p, p) for p in pages]
        for old, new in moved.items():
            self.holders[new], self.holders[old] = self.holders[old], 0
        self.free_pages = list(range(self.n_pages - 1, len(used) - 1, -1))
        return list(moved.items())


def shared_prefixes(table: np.ndarray, page_size: int) -> list[tuple[int, int, int]]:
    """Groups (first sequence, sequences, shared rows) of neighbours in a page table whose rows begin
    with the same pages.  A sequence joins its neighbour's group unless fewer rows would then be spared
    (those of all but one); a group has two sequences at least."""
    if len(table) < 2:
        return []
    differ = (table[1:] != table[:-1]) | (table[1:] < 0)
    alike = np.where(differ.any(1), differ.argmax(1), table.shape[1])   # pages in common with the one before
    groups, first, pages = [], 0, 0
    for i, n in enumerate(list(alike) + [0], start=1):
        n = int(n)
        if n and (i == first + 1 or (i - first) * min(n, pages) >= (i - first - 1) * pages):
            pages = n if i == first + 1 else min(n, pages)
            continue
        if i - first >= 2:
            groups.append((first, i - first, pages * page_size))
        first = i
    return groups


def worth_sharing(groups, cfg, format: str) -> list[tuple[int, int, int]]:
    """Those of a step's groups whose rows are to be read once for all: the others, and every group of a step
    in which too few bytes would be spared (those of all sequences but one of each group), are quicker apart,
    where the caches serve what is read again.

    Whole calls, us apart / shared (groups x sequences, shared rows each; 64 rows of their own).  bf16, the
    8B layer (1152 bytes a row): 1 x 8, 4096 rows 32 / 46; 8 x 8, 4096 73 / 62; 16 x 4, 8192 120 / 85; 8 x 8, 16384
    202 / 126; 32 x 2, 16384 212 / 226; 2 x 3, 131072 164 / 125; 1 x 64, 2048 48 / 51, 8192 92 / 75; 1 x 128, 4096
    78 / 85, 8192 125 / 120; 1 x 192, 16384 454 / 256; 1 x 256, 4096 140 / 145, 16384 419 / 391.  The 0.5B one
    (576 bytes): 8 x 8, 4096 37 / 38; 1 x 64, 4096 34 / 41; 32 x 4, 4096 60 / 52; 8 x 8, 16384 99 / 73.  e4m3 rows,
    about half as many bytes, gain less: the 8B layer 7 x 6, 20032 109 / 113; 1 x 32, 16384 70 / 72; 1 x 64, 8192
    71 / 70, 16384 110 / 103; 1 x 192, 8192 200 / 144; the 0.5B one 1 x 64, 8192 48 / 49; 1 x 128, 16384 128 / 117.
    With more than 32 heads a row is worked on longer once it is read (64 heads: 8 x 8, 4096 83 / 94; 16 x 3,
    8192 120 / 135)."""
    if cfg.n_heads > 32:
        return []
    row, least, spared = cfg.kv_rank + 2 * cfg.rope_dim + 4, 16, 384 << 20
    if format == "bf16":
        row, least, spared = 2 * (cfg.kv_rank + cfg.rope_dim), 3, 144 << 20
    groups = [g for g in groups if g[1] >= least and (g[1] <= 64 or g[2] >= 8192)]
    return groups if sum((n - 1) * rows for _, n, rows in groups) * row >= spared else []


class PagedLatentCache:
    """The paged latent cache of ``n_layers`` layers of shape ``cfg`` (a configs.LayerConfig).

    All layers share one page table: page p of a sequence lies at the same place of every
    layer's pool: [n_pages, page_size, r_kv + d_rope] in bf16, or [n_pages, bytes of a page] where
    ``format`` is "e4m3".  Shapes that the attention over pages does not
    serve (fp32, more than one positional key, other widths) are refused here."""

    format = "bf16"

    def __init__(self, cfg, n_layers: int, n_pages: int, page_size: int, device: str = "cuda:0",
                 format: str = "bf16"):
        if format not in ("bf16", "e4m3"):
            raise ValueError(f"format {format!r}: bf16 or e4m3")
        # (the library's load fails loudly if it is not built)
        ccfg = L.make_cfg(cfg.replace(batch=1, seq=1))
        if L.mla_recon_decode_paged_workspace_size(ccfg, 1) == 0:
            raise L.MlaError(L.MLA_ERR_UNSUPPORTED, L.last_error())
        if not torch.cuda.is_available():
            raise RuntimeError("PagedLatentCache needs a ROCm GPU")
        self.cfg, self.dtype, self.format = cfg, torch.bfloat16, format
        self.alloc = PageAllocator(n_pages, page_size)
        self.width = cfg.kv_rank + cfg.rope_dim
        if format == "e4m3":
            self.pool = torch.zeros(n_layers, n_pages,
                                    L.mla_recon_cache_page_bytes(ccfg, L.MLA_CACHE_E4M3, page_size),
                                    dtype=torch.uint8, device=device)
        else:
            self.pool = torch.zeros(n_layers, n_pages, page_size, self.width, dtype=self.dtype,
                                    device=device)
        self.device = self.pool.device  # (with its index: "cuda" would follow the current device)
        self._open = None  # the batch that has reserved pages and is not committed

    def _copy(self, pairs):
        if not pairs:
            return
        arr = np.ascontiguousarray(pairs, dtype=np.int32)
        size = self.pool.element_size()
        with torch.cuda.device(self.device):
            L.mla_recon_cache_copy_pages(self.pool.data_ptr(), self.pool.shape[0],
                                         self.pool.stride(0) * size, self.pool.shape[1],
                                         self.pool.stride(1) * size,
                                         arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                         len(arr), torch.cuda.current_stream().cuda_stream)

    def _closed(self):
        if self._open is not None:
            raise RuntimeError("a batch is open: commit or abandon it first")

    def add(self) -> int:
        return self.alloc.add()

    def length(self, seq: int) -> int:
        """Cached tokens of a sequence."""
        return self.alloc.length[seq]

    def fork(self, seq: int) -> int:
        self._closed()
        return self.alloc.fork(seq)

    def truncate(self, seq: int, length: int):
        self._closed()
        self.alloc.truncate(seq, length)

    def free(self, seq: int):
        self._closed()
        self.alloc.free(seq)

    def compact(self) -> int:
        """Move the pages in use to the front of the pools; returns how many moved."""
        self._closed()
        return len(self.alloc.compact(self._copy))

    def _handle(self, layer: int, table: torch.Tensor) -> L.PagedCache:
        pool = self.pool[layer]
        return L.PagedCache(pool.data_ptr(), table.data_ptr(), pool.shape[0], self.alloc.page_size,
                            table.shape[1])

    @property
    def _format(self) -> int:
        return L.MLA_CACHE_E4M3 if self.format == "e4m3" else L.MLA_CACHE_STORAGE

    def read(self, layer: int, seq: int, start: int = 0, count: int | None = None) -> torch.Tensor:
        """Cached rows start .. start + count - 1 of a sequence (default: all from start), as one bf16 tensor
        [count, r_kv + d_rope] = [c^KV | k^PE rotated]: for another cache, or a look at what is stored.  Up to
        8388608 rows a call."""
        have = self.alloc.length[seq]
        count = have - start if count is None else int(count)
        if start < 0 or count < 0 or start + count > have:
            raise ValueError(f"rows {start} .. {start + count - 1} of the {have} of sequence {seq}")
        out = torch.empty(count, self.width, dtype=self.dtype, device=self.device)
        if count == 0:
            return out
        pages = self.alloc.pages[seq]
        flat = torch.from_numpy(np.asarray([0, count, start] + pages, dtype=np.int32)).to(self.device)
        offsets, first, table = flat.split([2, 1, len(pages)])
        with torch.cuda.device(self.device):
            L.mla_recon_cache_read(L.make_cfg(self.cfg.replace(batch=1, seq=1)),
                                   self._handle(layer, table.view(1, -1)), self._format, out.data_ptr(), count,
                                   offsets.data_ptr(), first.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return out

    def batch(self, seqs, counts, share: bool = False) -> "Batch":
        """A step that adds counts[i] >= 1 tokens to seqs[i]: pages are reserved (and shared ones
        copied).  One batch is open at a time.  Sequences past 2^31 - 1 tokens are refused with nothing
        changed.  share: where every sequence has one new token, pages that neighbours in seqs have in
        common are attended to once for all of them, if that is quicker (``worth_sharing``; put forks of
        one sequence next to each other)."""
        self._closed()
        step = Batch(self, list(seqs), [int(c) for c in counts], share)
        self.alloc.extend(step.seqs, step.counts, self._copy)
        try:
            step._upload()
        except BaseException:
            step._give_back()
            raise
        self._open = step
        return step


class Batch:
    """One model step over some sequences of a PagedLatentCache: the packed new tokens of
    sequence i follow those of sequence i - 1."""

    def __init__(self, cache: PagedLatentCache, seqs, counts, share: bool = False):
        if not seqs or len(seqs) != len(counts) or any(c < 1 for c in counts):
            raise ValueError("a batch has sequences, and one new token or more of each")
        self.cache, self.seqs, self.counts = cache, seqs, counts
        self._before = [cache.alloc.length[s] for s in seqs]
        self._after = [n + c for n, c in zip(self._before, counts)]
        self.n_new, self.n_kv, self.max_len = sum(counts), sum(self._after), max(self._after)
        self.ccfg = L.make_cfg(cache.cfg.replace(batch=len(seqs), seq=1))
        self.single = all(c == 1 for c in counts)
        self.share, self.groups = share and self.single, []
        self._ws = None
        if self.max_len >= 2**31:
            raise L.MlaError(L.MLA_ERR_UNSUPPORTED, f"a sequence of {self.max_len} tokens")

    def _upload(self):
        """The page table (pages are reserved by now), offsets and lengths, to the GPU."""
        a, seqs, counts, before, after = self.cache.alloc, self.seqs, self.counts, self._before, self._after
        table = np.full((len(seqs), max(len(a.pages[s]) for s in seqs)), -1, dtype=np.int32)
        for row, s in zip(table, seqs):
            row[:len(a.pages[s])] = a.pages[s]
        if self.share:
            # (pages in common are full: a shared page that is not has been copied)
            self.groups = worth_sharing(shared_prefixes(table, a.page_size), self.cache.cfg, self.cache.format)
            # (a step of more rows than the call for groups takes is still decoded, apart)
            if self.groups and L.mla_recon_decode_shared_workspace_size(self.ccfg, self.cache._format, self.max_len,
                                                                        len(seqs)) == 0:
                self.groups = []
        zero = [0]
        # one upload: offsets, starts, offsets of the cached rows, lengths, the table
        parts = [np.cumsum(zero + counts), before, np.cumsum(zero + after), after, table.ravel()]
        if self.groups:  # all sequences between the groups' ends: those between two groups are groups without rows
            bounds, shared = [self.groups[0][0]], []
            for first, n, rows in self.groups:
                if first > bounds[-1]:
                    bounds.append(first)
                    shared.append(0)
                bounds.append(first + n)
                shared.append(rows)
            self.n_groups = len(shared)
            parts += [bounds, shared]
        flat = torch.from_numpy(np.concatenate([np.asarray(p, dtype=np.int32) for p in parts]))
        flat = flat.to(self.cache.device)
        self.offsets, self.start, self.kv_offsets, self.lengths, t, *g = flat.split([len(p) for p in parts])
        if self.groups:
            self.group_offsets, self.shared_len = g
        self.table = t.view(table.shape)

    def _handle(self, layer: int) -> L.PagedCache:
        if self.cache._open is not self:
            raise RuntimeError("this batch is not open")
        return self.cache._handle(layer, self.table)

    def _check(self, name, x, shape, dtype):
        if tuple(x.shape) != shape or x.dtype != dtype or x.device != self.cache.pool.device \
                or not x.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor {shape} on {self.cache.pool.device} "
                             f"is needed, not {x.dtype} {tuple(x.shape)} on {x.device}")

    def append(self, layer: int, rows: torch.Tensor, q: torch.Tensor, inv_freq: torch.Tensor) -> torch.Tensor:
        """Write the new tokens' rows [n_new, r_kv + d_rope] = [c^KV | k^PE], k^PE rotated at its
        position, into the pages of ``layer``; returns q [n_new, H, d_nope + d_rope] with its
        rotary part rotated likewise (a new tensor).  inv_freq [1, d_rope / 2] fp32."""
        c, cfg = self.cache, self.cache.cfg
        self._check("rows", rows, (self.n_new, c.width), c.dtype)
        self._check("q", q, (self.n_new, cfg.n_heads, cfg.nope_dim + cfg.rope_dim), c.dtype)
        self._check("inv_freq", inv_freq, (1, cfg.rope_dim // 2), torch.float32)
        out = torch.empty_like(q)
        append = L.mla_recon_cache_append_e4m3 if c.format == "e4m3" else L.mla_recon_cache_append
        with torch.cuda.device(c.device):
            append(self.ccfg, self._handle(layer), rows.data_ptr(), q.data_ptr(), out.data_ptr(), self.n_new,
                   self.offsets.data_ptr(), self.start.data_ptr(), inv_freq.data_ptr(),
                   torch.cuda.current_stream().cuda_stream)
        return out

    def attend(self, layer: int, q: torch.Tensor, Wuk: torch.Tensor, Wuv: torch.Tensor) -> torch.Tensor:
        """The per-head attention outputs [n_new, H, d_k] of the new tokens (q rotated, their rows
        appended), each over the cached rows of its sequence up to its own.  Wuk
        [G_kv d_nope, r_kv], Wuv [G_kv d_k, r_kv].  Of a step made with share=True the results are
        those of the step without it up to rounding.

        Where every sequence has one new token the call is the absorbed form's (decoding), else keys
        and values are written out (prefill) for all of the batch.  Single tokens by decoding and by
        prefill, whole calls of the 8B layer: 64 sequences of 4096 rows 79 and 1197 us, 512 of 16 rows
        88 and 162, one of 300 rows 21 and 29, 8 of 64 rows 25 and 22 (prefill is ahead in a few short
        sequences only, by 6 us at most).  One sequence of two tokens among 63 of one, 4096 rows each,
        makes the step a prefill: 1.3 ms.  A prefill takes 1048576 new tokens and as many cached rows of all
        its sequences: a larger step is refused here, with nothing enqueued (``append`` serves it)."""
        c, cfg = self.cache, self.cache.cfg
        self._check("q", q, (self.n_new, cfg.n_heads, cfg.nope_dim + cfg.rope_dim), c.dtype)
        self._check("Wuk", Wuk, (cfg.s_kv_groups * cfg.nope_dim, cfg.kv_rank), c.dtype)
        self._check("Wuv", Wuv, (cfg.s_kv_groups * cfg.head_dim, cfg.kv_rank), c.dtype)
        o = torch.empty(self.n_new, cfg.n_heads, cfg.head_dim, dtype=c.dtype, device=c.device)
        with torch.cuda.device(c.device):
            if self._ws is None:  # kept for the other layers
                self._ws = torch.empty(self._workspace_bytes(), dtype=torch.uint8, device=c.device)
            stream = torch.cuda.current_stream().cuda_stream
            e4m3 = c.format == "e4m3"
            if self.groups:
                L.mla_recon_decode_shared(self.ccfg, q.data_ptr(), self._handle(layer), c._format, self.max_len,
                                          self.lengths.data_ptr(), self.n_groups, self.group_offsets.data_ptr(),
                                          self.shared_len.data_ptr(), Wuk.data_ptr(), Wuv.data_ptr(), o.data_ptr(),
                                          self._ws.data_ptr(), self._ws.numel(), stream)
            elif self.single:
                decode = L.mla_recon_decode_e4m3 if e4m3 else L.mla_recon_decode_paged
                decode(self.ccfg, q.data_ptr(), self._handle(layer), self.max_len, self.lengths.data_ptr(),
                       Wuk.data_ptr(), Wuv.data_ptr(), o.data_ptr(), self._ws.data_ptr(), self._ws.numel(), stream)
            else:
                prefill = L.mla_recon_prefill_e4m3 if e4m3 else L.mla_recon_prefill_paged
                prefill(self.ccfg, q.data_ptr(), self.n_new, self.offsets.data_ptr(), self._handle(layer), self.n_kv,
                        self.kv_offsets.data_ptr(), Wuk.data_ptr(), Wuv.data_ptr(), o.data_ptr(),
                        self._ws.data_ptr(), self._ws.numel(), stream)
        return o

    def _workspace_bytes(self) -> int:
        if not self.single and self.n_kv >= 2**31:
            raise L.MlaError(L.MLA_ERR_UNSUPPORTED, f"a prefill over {self.n_kv} cached rows")
        e4m3 = self.cache.format == "e4m3"
        if self.groups:
            size = L.mla_recon_decode_shared_workspace_size(self.ccfg, self.cache._format, self.max_len, self.n_groups)
        elif self.single:
            size = (L.mla_recon_decode_e4m3_workspace_size if e4m3 else
                    L.mla_recon_decode_paged_workspace_size)(self.ccfg, self.max_len)
        else:
            size = (L.mla_recon_prefill_e4m3_workspace_size if e4m3 else
                    L.mla_recon_prefill_paged_workspace_size)(self.ccfg, self.n_new, self.n_kv)
        if size == 0:
            raise L.MlaError(L.MLA_ERR_UNSUPPORTED, L.last_error())
        return size

    def commit(self):
        """The new tokens count as cached."""
        self._handle(0)
        for s, c in zip(self.seqs, self.counts):
            self.cache.alloc.length[s] += c
        self.cache._open = None

    def abandon(self):
        """Give the batch up: its new tokens do not count, the pages reserved for them go back."""
        self._handle(0)
        self._give_back()
        self.cache._open = None

    def _give_back(self):
        for s in self.seqs:
            self.cache.alloc.truncate(s, self.cache.alloc.length[s])
