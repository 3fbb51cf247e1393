"""PagedLatentCache's steps on the host (no GPU): what is refused and what fails leaves the books as they were,
and page tables name copied pages only after the copies were enqueued."""
import copy
import os

import pytest
import torch

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs
from paper_2607_27269_amd.paged import PageAllocator, PagedLatentCache

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH),
                                reason="libmlarecon.so not built (run __graft_entry__.build())")


def host_cache(n_pages, page_size, cfg=None, copies=None):
    """A cache without a GPU's pools; page copies go to the list `copies`."""
    c = object.__new__(PagedLatentCache)
    c.cfg, c.device, c._open = cfg or configs.get(2), torch.device("cpu"), None
    c.alloc = PageAllocator(n_pages, page_size)
    c.pool = torch.zeros(1, n_pages, 1, 1)
    c._copy = copies.extend if copies is not None else lambda pairs: None
    return c


def grown(c, n):
    """A sequence of n cached tokens."""
    s = c.add()
    c.alloc.extend([s], [n])
    c.alloc.length[s] = n
    return s


def state(c):
    a = c.alloc
    return copy.deepcopy((a.pages, a.length, a.holders.tolist(), a.free_pages, c._open))


@pytest.mark.parametrize("kw", [dict(dtype="fp32"), dict(s_rope_groups=2), dict(kv_rank=384), dict(head_dim=32)])
def test_caches_that_no_attention_serves_are_refused(kw):
    """At the constructor, before a pool exists: append would fill them, and the first attend refuse."""
    with pytest.raises(L.MlaError) as e:
        PagedLatentCache(configs.get(1).replace(**kw), 1, 4, 16)
    assert e.value.code == L.MLA_ERR_UNSUPPORTED and str(e.value)


@pytest.mark.parametrize("page_size,tokens,forks,counts", [
    (1 << 16, 700_000, 2, [1, 2]),          # 1400003 rows
    (1 << 16, 1 << 20, 4096, [1] * 4095 + [2]),   # a little more than 2^32 rows
    (1 << 16, 10, 1, [(1 << 20) + 1]),      # too many new tokens
])
def test_steps_that_only_append_serves(page_size, tokens, forks, counts):
    """More new tokens, or more cached rows for a step of several tokens a sequence, than the attention
    takes: their rows can be appended, attend refuses (and does not take their low 32 bits), and the
    pages go back."""
    c = host_cache(6000, page_size)
    seqs = [grown(c, tokens)]
    seqs += [c.alloc.fork(seqs[0]) for _ in range(forks - 1)]
    free = len(c.alloc.free_pages)
    step = c.batch(seqs, counts)
    with pytest.raises(L.MlaError) as e:
        step._workspace_bytes()
    assert e.value.code == L.MLA_ERR_UNSUPPORTED and str(e.value)
    step.abandon()
    assert c._open is None and [c.alloc.length[s] for s in seqs] == [tokens] * forks
    assert len(c.alloc.free_pages) >= free - (forks - 1)     # (copies of the shared page stay)
    assert c.batch(seqs[:1], [1])._workspace_bytes() > 0     # single tokens over as many rows are served


def test_a_sequence_past_32_bits_is_refused():
    c = host_cache(40000, 1 << 16)
    s = grown(c, 2**31 - 1)
    before = state(c)
    with pytest.raises(L.MlaError):
        c.batch([s], [1])
    assert state(c) == before


class Failed(Exception):
    pass


def failing(pairs):
    if pairs:
        raise Failed


def test_a_failed_page_copy_leaves_the_tables_as_they_were():
    """Forked sequences grow into a shared page, and a pool is compacted: if the copy fails, no table names
    the page that did not get one, and the same call can be made again."""
    copies = []
    c = host_cache(12, 4, copies=copies)
    drop, s = grown(c, 8), grown(c, 6)
    t = c.alloc.fork(s)
    working, c._copy = c._copy, failing
    before = state(c)
    with pytest.raises(Failed):
        c.batch([s, t], [3, 1])
    assert state(c) == before
    c._copy = working
    step = c.batch([s, t], [3, 1])
    assert copies == [(c.alloc.pages[t][1], c.alloc.pages[s][1])]
    step.commit()
    c.alloc.free(drop)
    c._copy, before = failing, state(c)
    with pytest.raises(Failed):
        c.compact()
    assert state(c) == before
    c._copy = working
    del copies[:]
    assert c.compact() == len(copies) > 0
    assert max(p for pages in c.alloc.pages.values() for p in pages) == (c.alloc.holders > 0).sum() - 1


def test_a_failed_upload_gives_the_pages_back():
    c = host_cache(12, 4)
    s = grown(c, 6)
    before = (c.alloc.length[s], list(c.alloc.pages[s]), sorted(c.alloc.free_pages))
    c.device = "no such device"
    with pytest.raises(RuntimeError):
        c.batch([s], [9])
    assert before == (c.alloc.length[s], c.alloc.pages[s], sorted(c.alloc.free_pages)) and c._open is None
