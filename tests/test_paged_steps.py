"""PagedLatentCache's steps on the host (no GPU): what is refused is refused before anything has changed,
and page tables name copied pages only after the copies were enqueued."""
import copy
import os

import numpy as np
import pytest
import torch

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs
from paper_2607_27269_amd.paged import PageAllocator, PagedLatentCache

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH),
                                reason="libmlarecon.so not built (run __graft_entry__.build())")


def host_cache(n_pages, page_size, cfg=None, copies=None):
    """A cache without pools; page copies go to the list `copies`."""
    c = object.__new__(PagedLatentCache)
    c.cfg, c.device, c._open = cfg or configs.get(2), torch.device("cpu"), None
    c.alloc = PageAllocator(n_pages, page_size)
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
