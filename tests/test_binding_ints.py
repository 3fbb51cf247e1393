"""Sizes that 32 bits do not hold are refused by the binding: ctypes alone would pass their low bits on,
and the call would work on other sizes than its caller's."""
import ctypes
import os

import pytest

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH),
                                reason="libmlarecon.so not built (run __graft_entry__.build())")

CFG = L.make_cfg(configs.get(3).replace(batch=4, seq=1))


@pytest.mark.parametrize("n", [2**31, 2**32 + 5, -2**31 - 1])
def test_sizes_past_32_bits_are_refused(n):
    cache = L.PagedCache(256, 256, 10, 64, 8)
    for f, args in ((L.mla_recon_prefill_paged_workspace_size, (CFG, 4, n)),
                    (L.mla_recon_prefill_paged_workspace_size, (CFG, n, 4)),
                    (L.mla_recon_decode_paged_workspace_size, (CFG, n)),
                    (L.mla_recon_decode_workspace_size, (CFG, n)),
                    # (low bits of 0 rows, tokens or pairs: no launch in any case)
                    (L.mla_recon_cache_append, (CFG, cache, 256, 256, 256, n & ~0xff, 256, 256, 256, None)),
                    (L.mla_recon_cache_copy_pages, (256, 1, 0, 10, 1024, None, n & ~0xff, None))):
        with pytest.raises(ctypes.ArgumentError):
            f(*args)


def test_whole_numbers_of_any_type_pass():
    np = pytest.importorskip("numpy")
    want = L.mla_recon_prefill_paged_workspace_size(CFG, 100, 300)
    assert L.mla_recon_prefill_paged_workspace_size(CFG, np.int64(100), np.int32(300)) == want > 0
    with pytest.raises(ctypes.ArgumentError):
        L.mla_recon_prefill_paged_workspace_size(CFG, 100.0, 300)
