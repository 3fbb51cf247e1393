"""Which sequences of a step share their first pages (paged.shared_prefixes, Batch), on the host."""
import os

import numpy as np
import pytest
import torch

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs, paged
from paper_2607_27269_amd.paged import PagedLatentCache, shared_prefixes, worth_sharing
from test_paged_steps import grown, host_cache


def table(*rows):
    out = np.full((len(rows), max(map(len, rows))), -1, dtype=np.int32)
    for t, r in zip(out, rows):
        t[:len(r)] = r
    return out


@pytest.mark.parametrize("rows,groups", [
    ([[1, 2, 3]], []),
    ([[1, 2, 3], [4, 5]], []),
    ([[1, 2, 3], [1, 2, 4]], [(0, 2, 32)]),
    ([[1, 2], [1, 2]], [(0, 2, 32)]),
    ([[1, 2, 3], [1, 2, 4], [5], [6, 7, 8, 9], [6, 7, 8, 1], [6, 7, 8]], [(0, 2, 32), (3, 3, 48)]),
    ([[0, 1, 2, 3, 9], [0, 1, 2, 3, 8], [0, 1, 5], [0, 6]], [(0, 3, 32)]),   # 4 pages spared, 2 x 2, 3 x 1
    ([[0, 1, 2, 3, 9], [0, 1, 2, 3, 8], [0, 5], [0, 6]], [(0, 2, 64), (2, 2, 16)]),
    ([[1], [2], [3], [3]], [(2, 2, 16)]),
    ([[-1, -1], [-1, -1]], []),
])
def test_groups_of_a_table(rows, groups):
    assert shared_prefixes(table(*rows), 16) == groups


@pytest.mark.parametrize("groups,name,format,kept", [
    ([], 3, "bf16", []),
    ([(0, 9, 16384)], 3, "bf16", [(0, 9, 16384)]),            # 2^17 rows spared, of 1152 bytes
    ([(0, 9, 16368)], 3, "bf16", []),
    ([(0, 9, 16384)], 1, "bf16", []),                         # of 576 bytes
    ([(0, 9, 32768)], 1, "bf16", [(0, 9, 32768)]),
    ([(0, 2, 1 << 20)], 3, "bf16", []),                       # pairs do not count
    ([(0, 2, 1 << 20), (2, 5, 16384), (9, 5, 16384)], 3, "bf16", [(2, 5, 16384), (9, 5, 16384)]),
    ([(0, 64, 8192)], 3, "bf16", [(0, 64, 8192)]),
    ([(0, 65, 8176)], 3, "bf16", []),                         # large groups behind few rows
    ([(0, 200, 8192)], 3, "bf16", [(0, 200, 8192)]),
    ([(0, 41, 16384)], 3, "e4m3", [(0, 41, 16384)]),          # of 644 bytes
    ([(0, 38, 16384)], 3, "e4m3", []),
    ([(0, 15, 1 << 18)], 3, "e4m3", []),
])
def test_what_is_worth_sharing(groups, name, format, kept):
    cfg = configs.get(name)
    assert worth_sharing(groups, cfg, format) == kept
    assert worth_sharing(groups, cfg.replace(n_heads=64), format) == []


def test_the_first_and_last_rows_hold_for_any_table():
    """Random tables: groups are disjoint, in order, and share what they say."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        t = rng.integers(0, 2, (rng.integers(1, 12), rng.integers(1, 6))).astype(np.int32)
        t[rng.random(t.shape) < 0.05] = -1
        end = 0
        for first, n, rows in shared_prefixes(t, 4):
            assert first >= end and n >= 2 and rows % 4 == 0
            end = first + n
            part = t[first:end, :rows // 4]
            assert (part == part[0]).all() and (part >= 0).all()
        assert end <= len(t)


@pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libmlarecon.so not built")
def test_a_step_shares_full_pages_only(monkeypatch):
    """Forks of a sequence with a partly filled last page: each that grows has its own copy of that page;
    sequences between two groups are a group without shared rows."""
    c = host_cache(200, 16)
    monkeypatch.setattr(paged, "worth_sharing", lambda groups, cfg, format: groups)
    a = grown(c, 16 * 9 + 3)
    b = c.alloc.fork(a)
    alone = grown(c, 20)
    d = grown(c, 16 * 8)
    e = c.alloc.fork(d)
    step = c.batch([a, b, alone, d, e], [1] * 5, share=True)
    assert step.groups == [(0, 2, 144), (3, 2, 128)]
    assert step.group_offsets.tolist() == [0, 2, 3, 5] and step.shared_len.tolist() == [144, 0, 128]
    assert step.n_groups == 3 and step.lengths.tolist() == [148, 148, 21, 129, 129]
    step.abandon()
    step = c.batch([alone, a, d, b], [1] * 4, share=True)       # no neighbours
    assert not step.groups
    step.abandon()
    step = c.batch([a, b], [1, 2], share=True)                  # not single tokens
    assert not step.groups
    step.abandon()
    step = c.batch([alone, a, b], [1] * 3)
    assert not step.groups
    step.abandon()
    monkeypatch.undo()
    step = c.batch([a, b], [1] * 2, share=True)                 # too few
    assert not step.groups
    step.abandon()


@pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libmlarecon.so not built")
def test_steps_too_large_for_groups_are_decoded_apart(monkeypatch):
    """More rows than decode_shared numbers (2^35 over all blocks of 32 heads): the step is served as without sharing."""
    monkeypatch.setattr(paged, "worth_sharing", lambda groups, cfg, format: groups)
    c = host_cache(3000, 1 << 16, configs.get(3).replace(n_heads=64, batch=1, seq=1))
    a = grown(c, 1 << 26)
    seqs = [a] + [c.alloc.fork(a) for _ in range(299)]          # (full pages: each grows into one of its own)
    ccfg = L.make_cfg(c.cfg.replace(batch=300))
    assert L.mla_recon_decode_shared_workspace_size(ccfg, 0, (1 << 26) + 1, 1) == 0
    assert L.mla_recon_decode_paged_workspace_size(ccfg, (1 << 26) + 1) > 0
    step = c.batch(seqs, [1] * 300, share=True)
    assert not step.groups and step._workspace_bytes() > 0
    step.abandon()


def test_unknown_formats_are_refused():
    with pytest.raises(ValueError):
        PagedLatentCache(configs.get(1), 1, 4, 16, format="fp8")
