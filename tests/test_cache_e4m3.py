"""The eight-bit cache format and decoding behind shared prefixes without a GPU: the oracle's quantisation
against its definition, sizes of pages and workspaces, refusals."""
import os

import numpy as np
import pytest

from oracle import cache_e4m3_oracle as EO
from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs

needs_lib = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libmlarecon.so not built (run __graft_entry__.build())")

CFG = L.make_cfg(configs.get(3).replace(batch=4, seq=1))
FP32 = L.make_cfg(configs.get(3).replace(batch=4, seq=1, dtype="fp32"))
PER_HEAD = L.make_cfg(configs.get(4).replace(batch=4, seq=1))
OK = L.PagedCache(256, 256, 10, 64, 8)
BIG = 1 << 40


# ---- the format ----------------------------------------------------------------------------
def test_codes_round_trip():
    codes = np.arange(256, dtype=np.uint8)
    v = EO.value(codes)
    assert np.isnan(v[[127, 255]]).all() and v[126] == 448 and v[1] == 2.0 ** -9 and v[0x38] == 1.0
    fine = np.isfinite(v)
    assert (EO.code(v)[fine] == codes[fine]).all()


def test_code_is_the_nearest_and_halves_go_to_even():
    m = EO.MAGNITUDES
    mid = (m[1:] + m[:-1]) / 2
    k = EO.code(mid)
    assert (k % 2 == 0).all() and (np.abs(k.astype(int) - np.arange(len(mid)) - 0.5) == 0.5).all()
    assert (EO.code(mid * (1 + 1e-12)) == np.arange(1, 127)).all()
    assert (EO.code(mid * (1 - 1e-12)) == np.arange(126)).all()


def test_powers_are_the_least_that_fit():
    x = np.array([[448.0], [448.1], [224.0], [225.0], [1.0], [0.0], [2.0 ** -90], [3.38e38], [np.inf], [np.nan]])
    assert EO.exponent(x).tolist() == [0, 1, -1, 0, -8, -80, -80, 120, -80, -80]
    got = EO.stored(np.array([[1.0, np.nan, -3.0, np.inf]]), 4)
    assert got[0, 0] == 1 and got[0, 2] == -3 and np.isnan(got[0, [1, 3]]).all()


def test_error_is_half_a_step_at_most():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 512)) * np.exp(rng.standard_normal((200, 1)) * 20)
    y = EO.stored(x, 512)
    top = np.abs(x).max(-1, keepdims=True)
    power = 2.0 ** EO.exponent(x)[:, None]
    assert (np.abs(x - y) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * power)).all()
    # (a power half as large would not do, unless it is the smallest there is)
    assert (power * 448 >= top).all() and ((power * 224 < top) | (power == 2.0 ** -80)).all()


def test_pack_and_unpack():
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 256, (3, 5, 128)).astype(np.uint8)
    pe = rng.integers(-4, 5, (3, 5, 32)) / 4.0
    power = 2.0 ** rng.integers(-80, 121, (3, 5))
    pages = EO.pack(codes, pe, power)
    assert pages.shape == (3, -(-5 * (128 + 64 + 4) // 16) * 16)
    for a, b in zip(EO.unpack(pages, 5, 128, 32), (codes, pe, power)):
        assert (a == b).all()


# ---- the library's sizes and refusals --------------------------------------------------------
def refused(code, f, *args):
    with pytest.raises(L.MlaError) as e:
        f(*args)
    assert e.value.code == code and L.last_error(), args
    return str(e.value)


@needs_lib
def test_page_bytes():
    assert L.mla_recon_cache_page_bytes(CFG, L.MLA_CACHE_E4M3, 64) == 64 * 644
    assert L.mla_recon_cache_page_bytes(CFG, L.MLA_CACHE_STORAGE, 64) == 64 * 1152
    assert L.mla_recon_cache_page_bytes(FP32, L.MLA_CACHE_STORAGE, 3) == 3 * 2304
    assert L.mla_recon_cache_page_bytes(CFG, L.MLA_CACHE_E4M3, 1) == 656       # padded to 16
    assert L.mla_recon_cache_page_bytes(PER_HEAD, L.MLA_CACHE_E4M3, 16) == 16 * (1024 + 2 * 512 + 4)
    assert L.mla_recon_cache_page_bytes(CFG, L.MLA_CACHE_E4M3, 2**31 - 1) == -(-(2**31 - 1) * 644 // 16) * 16
    for cfg, fmt, n in ((CFG, 2, 64), (CFG, -1, 64), (CFG, 1, 0), (CFG, 1, -5), (FP32, 1, 64)):
        assert L.mla_recon_cache_page_bytes(cfg, fmt, n) == 0 and L.last_error()


@needs_lib
@pytest.mark.parametrize("cache", [None, L.PagedCache(None, 256, 10, 64, 8), L.PagedCache(256, None, 10, 64, 8),
                                   L.PagedCache(264, 256, 10, 64, 8), L.PagedCache(256, 256, 0, 64, 8),
                                   L.PagedCache(256, 256, 10, 0, 8), L.PagedCache(256, 256, 10, 64, 0),
                                   L.PagedCache(256, 256, 2**31 - 1, 2**31 - 1, 8)])
def test_bad_caches_are_refused(cache):
    bad = L.MLA_ERR_INVALID_ARG
    refused(bad, L.mla_recon_cache_append_e4m3, CFG, cache, 256, 256, 256, 4, 256, 256, 256, None)
    refused(bad, L.mla_recon_cache_read, CFG, cache, 1, 256, 4, 256, 256, None)
    refused(bad, L.mla_recon_decode_e4m3, CFG, 256, cache, 64, 256, 256, 256, 256, 256, BIG, None)
    refused(bad, L.mla_recon_prefill_e4m3, CFG, 256, 4, 256, cache, 9, 256, 256, 256, 256, 256, BIG, None)
    refused(bad, L.mla_recon_decode_shared, CFG, 256, cache, 0, 64, 256, 1, 256, 256, 256, 256, 256, 256, BIG, None)


@needs_lib
def test_append_and_read_refusals():
    def args(**kw):
        a = dict(cfg=CFG, cache=OK, rows=256, q=256, q_out=512, n_rows=4, offsets=256, start=256, inv_freq=256)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(rows=None, q=None, q_out=None), dict(q=None), dict(q_out=None), dict(n_rows=-1),
               dict(offsets=None), dict(start=None), dict(inv_freq=None), dict(rows=264), dict(q=264), dict(q_out=520)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_append_e4m3, *args(**kw))
    for kw in (dict(n_rows=(1 << 23) + 1), dict(cfg=FP32)):
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_cache_append_e4m3, *args(**kw))
    L.mla_recon_cache_append_e4m3(*args(n_rows=0))

    def read(**kw):
        a = dict(cfg=CFG, cache=OK, fmt=1, rows=256, n_rows=4, offsets=256, start=256)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(fmt=2), dict(fmt=-1), dict(rows=None), dict(rows=264), dict(n_rows=-1), dict(offsets=None),
               dict(start=None)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_cache_read, *read(**kw))
    for kw in (dict(n_rows=(1 << 23) + 1), dict(cfg=FP32)):
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_cache_read, *read(**kw))
    L.mla_recon_cache_read(*read(n_rows=0))
    L.mla_recon_cache_read(*read(n_rows=0, cfg=FP32, fmt=0))


@needs_lib
def test_decode_and_prefill_refusals():
    size = L.mla_recon_decode_e4m3_workspace_size(CFG, 512)
    assert size > 0

    def args(**kw):
        a = dict(cfg=CFG, q=256, cache=OK, max_len=512, lengths=256, Wuk=256, Wuv=256, o=256, ws=256, ws_bytes=size)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(q=None), dict(lengths=None), dict(Wuk=None), dict(Wuv=None), dict(o=None), dict(ws=None),
               dict(q=264), dict(Wuv=264), dict(ws=264), dict(max_len=0), dict(max_len=-1)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_decode_e4m3, *args(**kw))
    refused(L.MLA_ERR_WORKSPACE, L.mla_recon_decode_e4m3, *args(ws_bytes=size - 1))
    for cfg in (FP32, PER_HEAD):
        assert L.mla_recon_decode_e4m3_workspace_size(cfg, 512) == 0
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_decode_e4m3, *args(cfg=cfg, ws_bytes=BIG))
    refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_prefill_e4m3, FP32, 256, 4, 256, OK, 9, 256, 256, 256, 256, 256, BIG, None)
    size = L.mla_recon_prefill_e4m3_workspace_size(CFG, 100, 300)
    assert size > 0
    refused(L.MLA_ERR_WORKSPACE, L.mla_recon_prefill_e4m3, CFG, 256, 100, 256, OK, 300, 256, 256, 256, 256, 256,
            size - 1, None)
    L.mla_recon_prefill_e4m3(CFG, 256, 0, 256, OK, 300, 256, 256, 256, 256, 256, size, None)


@needs_lib
def test_shared_refusals():
    size = L.mla_recon_decode_shared_workspace_size(CFG, 0, 512, 2)
    assert size > 0

    def args(**kw):
        a = dict(cfg=CFG, q=256, cache=OK, fmt=0, max_len=512, lengths=256, n_groups=2, group_offsets=256,
                 shared_len=256, Wuk=256, Wuv=256, o=256, ws=256, ws_bytes=size)
        a.update(kw)
        return tuple(a.values()) + (None,)
    for kw in (dict(q=None), dict(lengths=None), dict(Wuk=None), dict(Wuv=None), dict(o=None), dict(ws=None),
               dict(q=264), dict(Wuv=264), dict(ws=264), dict(max_len=0), dict(fmt=2), dict(n_groups=-1),
               dict(n_groups=5), dict(group_offsets=None), dict(shared_len=None)):
        refused(L.MLA_ERR_INVALID_ARG, L.mla_recon_decode_shared, *args(**kw))
    refused(L.MLA_ERR_WORKSPACE, L.mla_recon_decode_shared, *args(ws_bytes=size - 1))
    for cfg in (FP32, PER_HEAD):
        assert L.mla_recon_decode_shared_workspace_size(cfg, 0, 512, 2) == 0
        refused(L.MLA_ERR_UNSUPPORTED, L.mla_recon_decode_shared, *args(cfg=cfg, ws_bytes=BIG))
    assert L.mla_recon_decode_shared_workspace_size(CFG, 0, 512, 5) == 0
    big = L.make_cfg(configs.get(3).replace(batch=60000, seq=1))
    assert L.mla_recon_decode_shared_workspace_size(big, 0, 2**31 - 1, 2) == 0


@needs_lib
@pytest.mark.parametrize("heads,groups", [(14, 2), (32, 8), (40, 8), (128, 128)])
def test_sizes_grow_with_sequences_lengths_and_groups(heads, groups):
    def size(b, n, g):
        c = L.make_cfg(configs.get(1).replace(batch=b, seq=1, n_heads=heads, s_kv_groups=groups, n_kv_groups=groups))
        return L.mla_recon_decode_shared_workspace_size(c, 1, n, min(b, g))
    bs, ns, gs = (1, 2, 3, 7, 64, 255, 257, 5000), (1, 31, 33, 500, 4096, 100000), (0, 1, 2, 5, 70, 5000)
    t = np.array([[[size(b, n, g) for g in gs] for n in ns] for b in bs], dtype=np.float64)
    assert t.min() > 0
    for axis in range(3):
        assert (np.diff(t, axis=axis) >= 0).all(), axis
