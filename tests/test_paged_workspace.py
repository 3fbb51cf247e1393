"""The paged attention's workspace sizes (no GPU): a workspace of the size reported for some tokens, rows
and sequences holds every call of fewer of them, so that a program can keep one of its largest step's."""
import os
import random

import pytest

from paper_2607_27269_amd import _lib as L
from paper_2607_27269_amd import configs

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH),
                                reason="libmlarecon.so not built (run __graft_entry__.build())")


def size(cfg, batch, n_q, n_kv):
    return L.mla_recon_prefill_paged_workspace_size(L.make_cfg(cfg.replace(batch=batch, seq=1)), n_q, n_kv)


SHAPES = [configs.get(1), configs.get(2), configs.get(3),
          configs.get(1).replace(n_heads=1, s_kv_groups=1, n_kv_groups=1),
          configs.get(3).replace(n_heads=128, s_kv_groups=128, n_kv_groups=128)]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_sizes_grow_with_tokens_rows_and_sequences(shape):
    cfg = SHAPES[shape]
    tokens = [0, 1, 63, 64, 77, 463, 1024, 1400, 1599, 1600, 2047, 2048, 4096, 65536, 1 << 20]
    rows = [0, 1, 255, 256, 511, 512, 3000, 4096, 16384, 100000, 1 << 20]
    batches = [1, 2, 8, 64, 300]
    t = {(b, q, k): size(cfg, b, q, k) for b in batches for q in tokens for k in rows}
    assert min(t.values()) > 0
    for (b, q, k), v in t.items():
        for b2, q2, k2 in ((batches[min(batches.index(b) + 1, len(batches) - 1)], q, k),
                           (b, tokens[min(tokens.index(q) + 1, len(tokens) - 1)], k),
                           (b, q, rows[min(rows.index(k) + 1, len(rows) - 1)])):
            assert t[b2, q2, k2] >= v, ((b, q, k), (b2, q2, k2))


def test_a_workspace_of_the_largest_step_serves_smaller_ones():
    rng = random.Random(5)
    for _ in range(3000):
        cfg = rng.choice(SHAPES)
        big = [rng.randint(1, 64), rng.randint(0, 6000), int(2 ** rng.uniform(0, 18))]
        small = [rng.randint(1, big[0]), rng.randint(0, big[1]), rng.randint(0, big[2])]
        assert size(cfg, *small) <= size(cfg, *big), (cfg.n_heads, small, big)


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_decode_sizes_grow_with_sequences_and_lengths(shape):
    def size(batch, max_len):
        return L.mla_recon_decode_paged_workspace_size(L.make_cfg(SHAPES[shape].replace(batch=batch, seq=1)), max_len)
    t = [[size(b, n) for n in (1, 31, 33, 500, 4096, 100000)] for b in (1, 2, 7, 64, 255, 257, 5000)]
    assert t[0][0] > 0
    for row in t + [list(c) for c in zip(*t)]:
        assert row == sorted(row)
