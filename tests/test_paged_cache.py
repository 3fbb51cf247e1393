"""Refusals of the paged-cache operators, without a GPU: every check returns before the library
touches one."""
import ctypes

import pytest

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs
import os

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH),
                                reason="libmlarecon.so not built (run __graft_entry__.build())")

CFG = L.make_cfg(configs.get(3).replace(batch=4, seq=1))
FP32 = L.make_cfg(configs.get(3).replace(batch=4, seq=1, dtype="fp32"))
PER_HEAD = L.make_cfg(configs.get(4).replace(batch=4, seq=1))
OK = L.PagedCache(256, 256, 10, 64, 8)
BIG = 1 << 40


def caches():
    return [(None, "no cache"), (L.PagedCache(None, 256, 10, 64, 8), "no pool"),
            (L.PagedCache(256, None, 10, 64, 8), "no table"), (L.PagedCache(264, 256, 10, 64, 8), "pool alignment"),
            (L.PagedCache(256, 256, 0, 64, 8), "no pages"), (L.PagedCache(256, 256, 10, 0, 8), "empty pages"),
            (L.PagedCache(256, 256, 10, -64, 8), "negative pages"), (L.PagedCache(256, 256, 10, 64, 0), "no entries"),
            (L.PagedCache(256, 256, 2**31 - 1, 2**31 - 1, 8), "too large")]


def refused(code, f, *args):
    with pytest.raises(L.MlaError) as e:
        f(*args)
    assert e.value.code == code and L.last_error(), args
    return str(e.value)


@pytest.mark.parametrize("cache,why", caches())
def test_bad_caches_are_refused(cache, why):
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_append, CFG, cache, 256, 256, 256, 4, 256, 256, 256, None)
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_decode_paged, CFG, 256, cache, 64, 256, 256, 256, 256, 256, BIG, None)
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_prefill_paged, CFG, 256, 4, 256, cache, 9, 256, 256, 256, 256, 256,
            BIG, None)


def test_append_refusals():
    def args(**kw):
        a = dict(cfg=CFG, cache=OK, rows=256, q=256, q_out=512, n_rows=4, offsets=256, start=256, inv_freq=256)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(rows=None, q=None, q_out=None), dict(q=None), dict(q_out=None), dict(n_rows=-1),
               dict(offsets=None), dict(start=None), dict(inv_freq=None), dict(rows=264), dict(q=264),
               dict(q_out=520), dict(cfg=L.make_cfg(configs.get(3).replace(rope_dim=60)))):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_append, *args(**kw))
    refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_cache_append, *args(n_rows=(1 << 23) + 1))
    # nothing to do: no launch
    L.mla_recon_cache_append(*args(n_rows=0))


def test_decode_refusals():
    size = L.mla_recon_decode_paged_workspace_size(CFG, 512)
    assert size > 0

    def args(**kw):
        a = dict(cfg=CFG, q=256, cache=OK, max_len=512, lengths=256, Wuk=256, Wuv=256, o=256, ws=256, ws_bytes=size)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(q=None), dict(lengths=None), dict(Wuk=None), dict(Wuv=None), dict(o=None), dict(ws=None),
               dict(q=264), dict(Wuv=264), dict(ws=264), dict(max_len=0), dict(max_len=-1)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_decode_paged, *args(**kw))
    refused(L.MLA_ERR_WORKSPACE, L.mla_recon_decode_paged, *args(ws_bytes=size - 1))
    for cfg in (FP32, PER_HEAD):
        assert L.mla_recon_decode_paged_workspace_size(cfg, 512) == 0
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_decode_paged, *args(cfg=cfg, ws_bytes=BIG))
    assert L.mla_recon_decode_paged_workspace_size(CFG, 0) == 0
    # a workspace for many sequences or long ones is enough for fewer and shorter ones
    sizes = [L.mla_recon_decode_paged_workspace_size(CFG, n) for n in (1, 100, 5000, 1 << 20, 2**31 - 1)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_prefill_refusals():
    size = L.mla_recon_prefill_paged_workspace_size(CFG, 100, 300)
    assert size > 0

    def args(**kw):
        a = dict(cfg=CFG, q=256, n_q=100, q_offsets=256, cache=OK, n_kv=300, kv_offsets=256, Wuk=256, Wuv=256,
                 o=256, ws=256, ws_bytes=size)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(q=None), dict(q_offsets=None), dict(kv_offsets=None), dict(Wuk=None), dict(Wuv=None),
               dict(o=None), dict(ws=None), dict(q=264), dict(Wuv=264), dict(o=264), dict(ws=264), dict(n_q=-1),
               dict(n_kv=-1)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_prefill_paged, *args(**kw))
    refused(L.MLA_ERR_WORKSPACE, L.mla_recon_prefill_paged, *args(ws_bytes=size - 1))
    for kw in (dict(cfg=FP32), dict(cfg=PER_HEAD), dict(n_q=(1 << 20) + 1), dict(n_kv=(1 << 20) + 1)):
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_prefill_paged, *args(ws_bytes=BIG, **kw))
    assert L.mla_recon_prefill_paged_workspace_size(CFG, (1 << 20) + 1, 1) == 0
    # no tokens: no launch
    L.mla_recon_prefill_paged(*args(n_q=0))


def test_copy_refusals():
    def call(pairs, **kw):
        flat = [v for p in pairs for v in p]
        a = dict(pool=256, n_layers=2, layer_stride=10 * 1024, n_pages=10, page_bytes=1024)
        a.update(kw)
        arr = (ctypes.c_int32 * max(1, len(flat)))(*flat)
        return tuple(a.values()) + (arr, len(pairs), None)
    for pairs in ([(0, 10)], [(10, 0)], [(-1, 0)], [(0, -1)], [(0, 1), (2, 1)], [(0, 0)], [(0, 1), (1, 2)],
                  [(k, k + 1) for k in range(8)]):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages, *call(pairs))
    many = [(k, 100 + k) for k in range(90)]      # beyond the list that is sorted in place
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages,
            *call(many + [(5, 100)], n_pages=200, layer_stride=200 * 1024))
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages,
            *call(many + [(100, 195)], n_pages=200, layer_stride=200 * 1024))
    for kw in (dict(pool=None), dict(pool=264), dict(page_bytes=1000), dict(page_bytes=0), dict(n_layers=0),
               dict(n_pages=0), dict(layer_stride=10 * 1024 - 16), dict(layer_stride=10 * 1024 + 8),
               dict(page_bytes=1 << 35, layer_stride=1 << 50)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages, *call([(0, 1)], **kw))
    refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_cache_copy_pages, *call([(0, 1)], n_layers=65536))
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages, 256, 1, 0, 10, 1024, None, 1, None)
    refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_copy_pages, 256, 1, 0, 10, 1024, None, -1, None)
    # nothing to copy: no launch
    L.mla_recon_cache_copy_pages(256, 1, 0, 10, 1024, None, 0, None)


def test_prefill_scale_too_small_is_refused():
    cfg = L.make_cfg(configs.get(1).replace(batch=2, seq=1))
    cfg.softmax_scale = 1e-31
    assert L.mla_recon_prefill_paged_workspace_size(cfg, 4, 4) == 0
    assert "softmax_scale" in L.last_error()


def test_prefill_head_widths_without_a_kernel_are_refused():
    cfg = L.make_cfg(configs.get(3).replace(batch=2, seq=1, nope_dim=0))      # keys of 64, values of 128
    assert L.mla_recon_prefill_paged_workspace_size(cfg, 4, 4) == 0
    assert "not supported" in L.last_error()
