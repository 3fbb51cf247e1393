"""GPU tests of decoding over so many rows that sums of them lose bits: a wavefront puts its state down every few
thousand tiles.  The caches are a few pages of 65536 rows that stand in every place of the tables, so that a sequence's
attention is that over their rows, each counted as often as it stands there.  Random pages differ in the mean of
their latents and stand in a random order, and one has logits so much larger that the six places where it stands in
a long sequence take about half of all weight: a part of a sequence that is lost or counted twice shows.

Tolerance of the rows alike.  All latents are one row of whole numbers, so that whatever the weights the output is that row
through W_UV, but for the output's rounding (2^-8), the weights' (fp16 2^-11), the weighted latents' as two bf16
values (2^-15) and the sums': up to 4096 tiles a run, two additions a tile for the latents and one for the weights, each
off by half a step of the sum so far at most, which is n 2^-25 of the last: 2^-12 + 2^-13.  (Rows alike are the worst case:
every addition errs in the same direction.  With weights of e^-1/8 added one by one, 16 a tile, the sum of 65536 tiles is
off by 0.7 % and of 262144 by 5 %.)  Of random rows: that of decoding (tests/test_gpu_paged.py)."""
import numpy as np
import pytest

from test_gpu_cache_e4m3 import E4m3Layer
from test_gpu_decode_shared import FORMATS
from test_gpu_paged import REL, Layer, bf16, ints, shape, up

pytestmark = pytest.mark.gpu

PS = 1 << 16
ALIKE = 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -12 + 2.0 ** -13 + 2.0 ** -15


class Pages:
    """The layer with two pages, calls over tables of them, and what they should give."""

    def __init__(self, fmt, seed, pages=None):
        """pages: places of the longest random sequence; None for rows alike."""
        n = 2 if pages is None else 3
        lay = self.lay = (E4m3Layer if fmt else Layer)(shape("tiny"), [n * PS], PS, seed=seed, spare=0)
        self.fmt, self.cfg, rkv = int(fmt), lay.cfg, lay.cfg.kv_rank
        if fmt:                                              # (made again of the rows below)
            del lay.codes, lay.power
        if pages is None:
            lay.pool[:] = 0
            lay.pool[..., :rkv] = lay.rng.integers(1, 4, rkv)
            lay.pool[:, ::32, rkv] = 1.0                     # the largest weight is in every tile
        else:
            lay.pool[..., :rkv] = bf16(lay.pool[..., :rkv] + lay.rng.standard_normal((n, 1, rkv)))
            lay.pool[..., rkv] = 0
            lay.pool[2, :, rkv] = bf16(np.array([2 * np.log(pages / 6)]))[0]   # (queries of 4, a scale of 1/8)
        lay.upload()

    def queries(self, n, alike=False):
        q = self.lay.queries(n)
        q[..., self.cfg.nope_dim] = 4.0
        if alike:
            q[:] = 0
            q[..., self.cfg.nope_dim] = 1.0                  # logits of 1/8 and 0
        return q

    def tables(self, lens, long=()):
        """Pages 0 and 1 in any order, page 2 in six places of the sequences `long`."""
        rng, width = self.lay.rng, -(-max(lens) // PS)
        tables = rng.integers(0, 2, (len(lens), width))
        for b in long:
            tables[b, rng.choice(lens[b] // PS, 6, replace=False)] = 2
        return tables

    def call(self, q, lens, tables, groups=None, shared=None, paged=False):
        import torch
        from paper_2607_27269_amd import _lib as L
        lay, stream, most = self.lay, torch.cuda.current_stream().cuda_stream, max(lens)
        cfg = L.make_cfg(self.cfg.replace(batch=len(lens), seq=1))
        d_q, d_table, d_lens = up(q), ints(tables), ints(lens)
        cache = L.PagedCache(lay.d_pool.data_ptr(), d_table.data_ptr(), len(lay.d_pool), PS, tables.shape[1])
        o = torch.empty(len(lens), self.cfg.n_heads, self.cfg.head_dim, dtype=torch.bfloat16, device="cuda")
        n_groups = 0 if shared is None else len(shared)
        off, rows = (ints(groups), ints(shared)) if n_groups else (None, None)
        if paged:
            size = L.mla_recon_decode_paged_workspace_size(cfg, most)
        else:
            size = L.mla_recon_decode_shared_workspace_size(cfg, self.fmt, most, n_groups)
        assert size > 0, L.last_error()
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        rest = (lay.d_Wuk.data_ptr(), lay.d_Wuv.data_ptr(), o.data_ptr(), ws.data_ptr(), size, stream)
        if paged:
            L.mla_recon_decode_paged(cfg, d_q.data_ptr(), cache, most, d_lens.data_ptr(), *rest)
        else:
            L.mla_recon_decode_shared(cfg, d_q.data_ptr(), cache, self.fmt, most, d_lens.data_ptr(), n_groups,
                                      off.data_ptr() if n_groups else None, rows.data_ptr() if n_groups else None, *rest)
        return o.double().cpu().numpy()

    def want(self, q, n, table):
        """One sequence's output in float64."""
        c, lay = self.cfg, self.lay
        count = np.zeros((len(lay.pool), PS))
        for page, k in zip(*np.unique(table[:n // PS], return_counts=True)):
            count[page] += k
        if n % PS:
            count[table[n // PS], :n % PS] += 1
        rows, count = lay.pool.reshape(-1, lay.W), count.ravel()
        out = np.zeros((c.n_heads, c.head_dim))
        for h in range(c.n_heads):
            g = h // (c.n_heads // c.s_kv_groups)
            x = np.concatenate([q[h, :c.nope_dim] @ lay.Wuk[g * c.nope_dim:(g + 1) * c.nope_dim], q[h, c.nope_dim:]])
            s = rows @ x * float(np.float32(c.softmax_scale))
            p = np.exp(s - s[count > 0].max()) * count
            out[h] = lay.Wuv[g * c.head_dim:(g + 1) * c.head_dim] @ (p / p.sum() @ rows[:, :c.kv_rank])
        return out

    def check(self, got, q, lens, tables, only, bound):
        for b in only:
            ref = self.want(q[b], lens[b], tables[b])
            e = (np.linalg.norm(got[b] - ref, axis=-1) / np.linalg.norm(ref, axis=-1)).max()
            print(f"[sums] sequence {b}, {lens[b]} rows: {e:.2e}", flush=True)
            assert e <= bound, (b, lens[b], e)


MOST = 2**31 - 1


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("call", ["paged", "own bf16", "own e4m3", "shared bf16", "shared e4m3"])
def test_rows_alike(call, n):
    """The longest sequences, each row by itself, and shared by all."""
    print(f"[sums] {call}: {n} of {MOST} rows", flush=True)
    p = Pages("e4m3" in call, 1)
    lens, q = [MOST] * n, p.queries(n, alike=True)
    tables = p.tables([MOST])[[0] * n]
    shared = dict(groups=[0, n], shared=[MOST]) if "shared" in call else {}
    p.check(p.call(q, lens, tables, paged=call == "paged", **shared), q, lens, tables, range(n), ALIKE)


@pytest.mark.parametrize("call", ["paged", "bf16", "e4m3"])
def test_random_rows_of_many_sequences(call):
    """Runs of several thousand tiles that cross from sequence to sequence, one of which fills many workgroups; a page
    that is missing early in a long sequence is not forgotten."""
    print(f"[sums] many sequences, {call}", flush=True)
    p = Pages(call == "e4m3", 2, 1 << 26 >> 16)
    lens = [int(n) for n in p.lay.rng.integers(300000, 600000, 300)]
    lens[4], lens[77], lens[150], lens[299] = 0, 1 << 26, 5 * PS, 33
    tables, q = p.tables(lens, [77]), p.queries(300)
    tables[200, 1] = -1
    got = p.call(q, lens, tables, paged=call == "paged")
    assert np.isnan(got[200]).all() and not got[4].any()
    p.check(got, q, lens, tables, [0, 1, 2, 3, 5, 76, 77, 78, 149, 150, 151, 199, 201, 298, 299], REL)


@pytest.mark.parametrize("call", ["paged", "bf16", "e4m3"])
def test_random_rows_of_few_sequences(call):
    p = Pages(call == "e4m3", 5, 3000)
    lens = [3000 * PS + 17, 1000 * PS, 2 * PS + 5, 2000 * PS - 40]
    tables, q = p.tables(lens, [0, 1, 3]), p.queries(4)
    p.check(p.call(q, lens, tables, paged=call == "paged"), q, lens, tables, range(4), REL)


@FORMATS
def test_random_rows_behind_long_prefixes(fmt):
    """Pieces of the shared rows of about 16000 tiles each."""
    p = Pages(fmt, 3, 1 << 27 >> 16)
    shared = [1 << 27, 0, 3 * PS]
    lens = [shared[0] + k for k in (1, 70000, 33)] + [123456] + [shared[2] + k for k in (1, 5, 40000, 70)]
    tables, q = p.tables(lens, [0]), p.queries(8)
    tables[1:3], tables[5:8] = tables[0], tables[4]
    p.check(p.call(q, lens, tables, groups=[0, 3, 4, 8], shared=shared), q, lens, tables, range(8), REL)


@FORMATS
def test_random_rows_behind_a_long_prefix_of_a_large_group(fmt):
    """520 sequences behind 640000 rows: a piece, of rows that the launch before copies, has 10000 tiles."""
    p = Pages(fmt, 4, 10)
    lens = [640000 + 1 + b % 90 for b in range(520)]
    tables, q = p.tables(lens), p.queries(520)
    tables[:] = [0, 1, 2, 0, 0, 1, 0, 1, 1, 1]
    got = p.call(q, lens, tables, groups=[0, 520], shared=[640000])
    p.check(got, q, lens, tables, [0, 1, 2, 3, 4, 130, 257, 516, 517, 518, 519], REL)
