"""GPU tests of the eight-bit latent cache against float64 (oracle/paged_oracle.py over the values that
oracle/cache_e4m3_oracle.py gives the stored rows).

Tolerances.  Latents are quantised by an exact rule from bf16 values: append's codes and powers, and read's
values, are compared bit by bit.  Rotated values: one rounding to bf16 (2^-8 of the value) and the fp32
rotation (1e-6 of |lo| + |hi|).  decode and prefill: what tests/test_gpu_paged.py allows their bf16 forms (1e-2
of the norm), since the stored values themselves are exact operands.
"""
import numpy as np
import pytest

from oracle import cache_e4m3_oracle as EO
from oracle import paged_oracle as PO
from test_gpu_paged import EDGES, Decode, Layer, bf16, check_decode, ints, scatter, shape, up

pytestmark = pytest.mark.gpu


class E4m3Layer(Layer):
    """A layer whose pool is in eight bits; ``pool`` holds the values that it stands for."""

    def upload(self):
        import torch
        codes, power = EO.quantise(self.pool[..., :self.cfg.kv_rank])
        if not hasattr(self, "codes"):
            self.codes, self.power = codes, power
        self.pool = np.concatenate([EO.value(self.codes) * self.power[..., None], self.pool[..., self.cfg.kv_rank:]], -1)
        self.d_pool = torch.from_numpy(EO.pack(self.codes, self.pool[..., self.cfg.kv_rank:], self.power)).cuda()
        self.d_table = ints(self.table)
        self.d_Wuk, self.d_Wuv = up(self.Wuk), up(self.Wuv)

    def edit(self, page, row, latents=None, positional=None):
        """Give a cached row other values."""
        if latents is not None:
            self.codes[page, row], self.power[page, row] = EO.quantise(latents)
        if positional is not None:
            self.pool[page, row, self.cfg.kv_rank:] = positional

    def handle(self, batch=None):
        from paper_2607_27269_amd import _lib as L
        c = L.make_cfg(self.cfg.replace(batch=batch or len(self.table), seq=1))
        assert self.d_pool.shape[1] == L.mla_recon_cache_page_bytes(c, L.MLA_CACHE_E4M3, self.ps)
        return c, L.PagedCache(self.d_pool.data_ptr(), self.d_table.data_ptr(), len(self.d_pool), self.ps,
                               self.d_table.shape[1])


class DecodeE4m3(Decode):
    GUARD = 4096

    def __init__(self, layer, q, lens, max_len):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.layer, self.max_len, self.c = layer, max_len, layer.handle()
        self.q, self.lens, self.Wuk = up(q), ints(lens), layer.d_Wuk
        self.o = torch.full((len(q), layer.cfg.n_heads, layer.cfg.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        self.size = L.mla_recon_decode_e4m3_workspace_size(self.c[0], max_len)
        assert self.size > 0, L.last_error()
        self.ws = torch.full((self.size + self.GUARD,), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.ws[self.size:] = 0xA5
        L.mla_recon_decode_e4m3(self.c[0], self.q.data_ptr(), self.c[1], self.max_len, self.lens.data_ptr(),
                                self.Wuk.data_ptr(), self.layer.d_Wuv.data_ptr(), self.o.data_ptr(),
                                self.ws.data_ptr(), self.size, torch.cuda.current_stream().cuda_stream)
        return self.o

    def guard(self):
        assert bool((self.ws[self.size:] == 0xA5).all()), "written behind the workspace"


# ---- append ----------------------------------------------------------------------------------
class Append:
    def __init__(self, cfg, new, start, ps, seed, latents=None, lo=0, hi=0):
        """new[b] rows of sequence b at positions start[b] ..; `lo` packed rows before the first
        sequence's and `hi` behind the last's belong to nobody."""
        import torch
        rng = np.random.default_rng(seed)
        self.cfg, self.ps, c = cfg, ps, cfg
        pe = c.s_rope_groups * c.rope_dim
        self.table, total = scatter(rng, [a + b for a, b in zip(start, new)], ps)
        n = lo + sum(new) + hi
        self.rows = bf16(rng.standard_normal((n, c.kv_rank + pe)) * np.exp(rng.standard_normal((n, 1))))
        if latents is not None:
            latents(self.rows, rng)
        self.q = bf16(rng.standard_normal((n, c.n_heads, c.nope_dim + c.rope_dim)))
        self.inv = (1e4 ** (-np.arange(pe // 2) / (pe / 2))).astype(np.float32).reshape(c.s_rope_groups, -1)
        self.offsets, self.start = np.concatenate([[0], np.cumsum(new)]) + lo, np.array(start)
        size = -(-ps * (c.kv_rank + 2 * pe + 4) // 16) * 16
        self.before = rng.integers(0, 256, (total, size)).astype(np.uint8)
        self.d_pool = torch.from_numpy(self.before).cuda()
        self.d_rows, self.d_q, self.d_inv = up(self.rows), up(self.q), up(self.inv, "fp32")
        self.d_out = torch.full_like(self.d_q, 9.0)
        self.d_off, self.d_start, self.d_table = ints(self.offsets), ints(start), ints(self.table)

    def __call__(self, rows=True, q=True, in_place=False):
        import torch
        from paper_2607_27269_amd import _lib as L
        cfg = L.make_cfg(self.cfg.replace(batch=len(self.start), seq=1))
        cache = L.PagedCache(self.d_pool.data_ptr(), self.d_table.data_ptr(), len(self.d_pool), self.ps, self.table.shape[1])
        out = self.d_q if in_place else self.d_out
        L.mla_recon_cache_append_e4m3(cfg, cache, self.d_rows.data_ptr() if rows else None,
                                      self.d_q.data_ptr() if q else None, out.data_ptr() if q else None,
                                      len(self.rows), self.d_off.data_ptr(), self.d_start.data_ptr(),
                                      self.d_inv.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return self.d_pool.cpu().numpy(), out.double().cpu().numpy()

    def check(self, pages, q_out, rows=True):
        c = self.cfg
        pe, rkv = c.s_rope_groups * c.rope_dim, c.kv_rank
        plain = np.zeros((len(pages), self.ps, rkv + pe))
        want, ref = PO.append(plain * np.nan, self.table, self.rows, self.q, self.offsets, self.start, self.inv,
                              kv_rank=rkv, nope_dim=c.nope_dim)
        codes, positional, power = EO.unpack(pages, self.ps, rkv, pe)
        old = EO.unpack(self.before, self.ps, rkv, pe)
        written = np.zeros(power.shape, dtype=bool)
        for b in range(len(self.start)):
            for i in range(self.offsets[b], self.offsets[b + 1]):
                p = self.start[b] + i - self.offsets[b]
                at = self.table[b, p // self.ps], p % self.ps
                if not rows:
                    continue
                written[at] = True
                k, e = EO.quantise(self.rows[i, :rkv])
                assert power[at] == e and (codes[at] & np.where(k == 127, 127, 255) == k).all(), (b, i)
                x, y = self.rows[i, rkv:], want[at][rkv:]
                size = np.abs(x.reshape(c.s_rope_groups, 2, -1)).sum(1, keepdims=True).repeat(2, 1).ravel()
                assert (np.abs(positional[at] - y) <= 2.0 ** -8 * np.abs(y) + 2e-6 * size).all(), (b, i)
        for a, b in zip((codes, positional, power), old):    # every other row as it was
            assert np.array_equal(a[~written], b[~written], equal_nan=True)
        tail = self.ps * (rkv + 2 * pe + 4)
        assert (pages[:, tail:] == self.before[:, tail:]).all()
        if q_out is not None:
            have = ~np.isnan(ref)
            size = np.abs(self.q).max()
            assert (np.abs(q_out - ref)[have] <= 2.0 ** -8 * np.abs(ref)[have] + 4e-6 * size).all()
            assert (q_out[~have] == 9.0).all()


@pytest.mark.parametrize("name,new,start,ps", [
    ("tiny", [1], [0], 1), ("tiny", [5, 1, 0, 33], [3, 0, 9, 64], 5), ("05b", [1, 17], [300, 15], 16),
    ("1b", [40, 0, 7], [0, 5, 100], 24), ("8b", [65, 3], [63, 200], 64)])
def test_append(name, new, start, ps):
    print(f"[e4m3] append {name} {new} at {start} page {ps}", flush=True)
    a = Append(shape(name), new, start, ps, seed=ps, lo=2, hi=3)
    a.check(*a())


def test_append_positional_keys_of_many_heads_and_a_wide_latent():
    """Config 4: 32 positional keys of 16 values, 1024 latents (two pieces a lane)."""
    from paper_2607_27269_amd import configs
    a = Append(configs.get(4), [9, 2], [5, 31], 8, seed=4)
    a.check(*a())


def test_append_narrow_latents():
    """40 latents: fewer than a piece for each lane, rows that are no multiple of 16 bytes."""
    a = Append(shape("tiny", kv_rank=40, rope_dim=24, nope_dim=40), [7, 1], [2, 12], 3, seed=5)
    a.check(*a())


def test_append_at_the_ends_of_the_range():
    """Rows of zeros, subnormal ones, the largest values, infinities and NaN among finite ones, halves
    between codes, and the borders between powers."""
    def latents(rows, rng):
        half = 2.0 ** np.arange(-8, 8)
        kinds = [0 * rows[0, :128], rows[0, :128] * 2.0 ** -126, rows[0, :128] * 1e37, rows[0, :128] * 2.0 ** -75]
        for k, v in enumerate(kinds):
            rows[k, :128] = bf16(v)
        rows[4, 3], rows[4, 5], rows[4, 77] = np.inf, -np.inf, np.nan
        rows[5, :128] = np.inf
        rows[6, :128] = np.resize(np.concatenate([448 * half, -17 * half, 1.0625 * half, 1.1875 * half]), 128)
        rows[7, :128], rows[7, 0] = 1.0, 448.0
        rows[8, :128], rows[8, 0] = 1.0, 450.0
        rows[9, :128], rows[9, 0] = 2.0 ** -9, 448.0
        rows[10, :128], rows[10, 0] = 1.5 * 2.0 ** -9, 448.0
        rows[11, :128] = 3.3895313892515355e38       # bf16's largest
        rows[12, :128] = -0.0
    a = Append(shape("tiny"), [13], [0], 4, seed=6, latents=latents)
    a.check(*a())


def test_append_of_rows_alone_queries_alone_and_in_place():
    a = Append(shape("1b"), [6, 4], [30, 1], 16, seed=7)
    pages, _ = a(q=False)
    a.check(pages, None)
    a.d_pool.copy_(up(a.before * 0.0, "fp32").to(a.d_pool.dtype))
    a.before[:] = 0
    pages, q = a(rows=False)
    assert not pages.any()
    a.check(pages, q, rows=False)
    first = a.d_out.clone()
    a(in_place=True)
    import torch
    assert torch.equal(a.d_q, first)


def test_append_outside_the_table_or_on_no_page_is_dropped():
    a = Append(shape("05b"), [20, 20], [0, 0], 8, seed=8)
    a.table[0, 1], a.table[1, 2] = -1, len(a.d_pool)
    a.d_table = ints(a.table[:, :2])
    a.table = a.table[:, :2]
    pages, q = a()
    codes, _, power = EO.unpack(pages, 8, 256, 32)
    old = EO.unpack(a.before, 8, 256, 32)
    for b, page, n in ((0, a.table[0, 0], 8), (1, a.table[1, 0], 8), (1, a.table[1, 1], 8)):
        assert (power[page] >= 2.0 ** -80).all()
    kept = [p for p in range(len(pages)) if p not in (a.table[0, 0], a.table[1, 0], a.table[1, 1])]
    assert (codes[kept] == old[0][kept]).all() and np.array_equal(power[kept], old[2][kept], equal_nan=True)
    assert np.isfinite(q).all() and not (q == 9.0).all(-1).any()


# ---- read ------------------------------------------------------------------------------------
def read(layer, fmt, start, count, lo=0, hi=0, dtype=None):
    import torch
    from paper_2607_27269_amd import _lib as L
    cfg, cache = layer.handle()
    n = lo + sum(count) + hi
    out = torch.full((n, layer.W), 5.0, dtype=dtype or torch.bfloat16, device="cuda")
    offsets, d_start = ints(np.concatenate([[0], np.cumsum(count)]) + lo), ints(start)
    L.mla_recon_cache_read(cfg, cache, fmt, out.data_ptr(), n, offsets.data_ptr(), d_start.data_ptr(),
                           torch.cuda.current_stream().cuda_stream)
    return out.double().cpu().numpy()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("name,ps", [("tiny", 1), ("05b", 7), ("1b", 16), ("8b", 64)])
def test_read(name, ps, e4m3):
    print(f"[e4m3] read {name} page {ps}", flush=True)
    lens = [100, 1, 0, 65, 33]
    lay = (E4m3Layer if e4m3 else Layer)(shape(name), lens, ps, seed=ps)
    start, count = [3, 0, 0, 64, 0], [97, 1, 0, 1, 20]
    got = read(lay, int(e4m3), start, count, lo=3, hi=5)
    assert (got[:3] == 5).all() and (got[-5:] == 5).all()
    at = 3
    for b in range(5):
        want = PO.cached_rows(lay.pool, lay.table, b, lens[b])[start[b]:start[b] + count[b]]
        assert np.array_equal(got[at:at + count[b]], want), b
        at += count[b]


def test_read_of_fp32_rows():
    import torch
    from paper_2607_27269_amd import _lib as L
    lay = Layer(shape("tiny"), [37, 5], 8, seed=1)
    lay.cfg = lay.cfg.replace(dtype="fp32")
    lay.pool = np.random.default_rng(2).standard_normal(lay.pool.shape).astype(np.float32).astype(np.float64)
    lay.d_pool = up(lay.pool, "fp32")
    got = read(lay, L.MLA_CACHE_STORAGE, [1, 0], [36, 5], dtype=torch.float32)
    want = np.concatenate([PO.cached_rows(lay.pool, lay.table, 0, 37)[1:], PO.cached_rows(lay.pool, lay.table, 1, 5)])
    assert np.array_equal(got, want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_read_outside_the_table_or_on_no_page_is_nan(e4m3):
    lay = (E4m3Layer if e4m3 else Layer)(shape("05b"), [40, 40], 16, seed=3)
    lay.table[0, 1], lay.table[1, 0] = -3, 10**7
    lay.upload()
    got = read(lay, int(e4m3), [10, -4], [60, 30])
    for b, first, rows in ((0, 10, got[:60]), (1, -4, got[60:])):
        for i, p in enumerate(range(first, first + len(rows))):
            page = lay.table[b, p // 16] if 0 <= p < 16 * lay.table.shape[1] else -1
            want = lay.pool[page, p % 16] if 0 <= page < len(lay.pool) else np.full(lay.W, np.nan)
            assert np.array_equal(rows[i], want, equal_nan=True), (b, p)


def test_read_of_non_finite_and_extreme_latents():
    lay = E4m3Layer(shape("tiny"), [6], 4, seed=4)
    t = lay.table[0]
    x = lay.pool[t[0], 0, :128].copy()
    x[5], x[9] = np.nan, np.inf
    lay.edit(t[0], 0, x)
    lay.edit(t[0], 1, x * 0)
    lay.edit(t[0], 2, bf16(lay.pool[t[0], 2, :128] * 2.0 ** 100))
    lay.edit(t[0], 3, bf16(lay.pool[t[0], 3, :128] * 2.0 ** -100))
    lay.edit(t[1], 0, bf16(lay.pool[t[1], 0, :128] * 2.0 ** -68))
    lay.upload()
    got = read(lay, 1, [0], [6])
    assert np.array_equal(got, PO.cached_rows(lay.pool, lay.table, 0, 6), equal_nan=True)


def test_appended_rows_are_read_back():
    """append, then read: the rows that the oracle says were stored."""
    import torch
    from paper_2607_27269_amd import _lib as L
    a = Append(shape("8b"), [70, 1, 200], [0, 63, 10], 32, seed=9)
    a()
    cfg = L.make_cfg(a.cfg.replace(batch=3, seq=1))
    cache = L.PagedCache(a.d_pool.data_ptr(), a.d_table.data_ptr(), len(a.d_pool), 32, a.table.shape[1])
    out = torch.zeros(271, 576, dtype=torch.bfloat16, device="cuda")
    L.mla_recon_cache_read(cfg, cache, L.MLA_CACHE_E4M3, out.data_ptr(), 271, a.d_off.data_ptr(), a.d_start.data_ptr(),
                           torch.cuda.current_stream().cuda_stream)
    assert np.array_equal(out.double().cpu().numpy()[:, :512], EO.stored(a.rows, 512)[:, :512])


# ---- decode ----------------------------------------------------------------------------------
@pytest.mark.parametrize("name,ps", [("tiny", 1), ("tiny", 64), ("05b", 7), ("05b", 16), ("1b", 16), ("1b", 100),
                                     ("8b", 24), ("8b", 64)])
def test_decode_edges(name, ps):
    print(f"[e4m3] decode {name} page {ps}", flush=True)
    lay = E4m3Layer(shape(name), EDGES, ps, seed=ps)
    q = lay.queries(len(EDGES))
    d = DecodeE4m3(lay, q, EDGES, max(EDGES))
    check_decode(lay, q, EDGES, d())
    d.guard()


@pytest.mark.parametrize("name,lens,ps", [("8b", [2049], 64), ("05b", [4000, 3, 0, 1025], 16),
                                          ("1b", [777] * 9 + [0] * 3, 32), ("tiny", [9000, 8191], 48)])
def test_decode_long(name, lens, ps):
    print(f"[e4m3] decode {name} {lens} page {ps}", flush=True)
    lay = E4m3Layer(shape(name), lens, ps, seed=len(lens))
    q = lay.queries(len(lens))
    d = DecodeE4m3(lay, q, lens, max(lens))
    check_decode(lay, q, lens, d())
    d.guard()


@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (33, 1), (40, 8), (64, 2)])
def test_decode_head_counts(H, G):
    print(f"[e4m3] decode {H} heads in {G} groups", flush=True)
    lens = [150, 0, 64, 1, 333]
    lay = E4m3Layer(shape("05b", n_heads=H, s_kv_groups=G, n_kv_groups=G), lens, 16, seed=H)
    q = lay.queries(len(lens))
    d = DecodeE4m3(lay, q, lens, 333)
    check_decode(lay, q, lens, d())
    d.guard()


def test_decode_without_non_positional_keys():
    lay = E4m3Layer(shape("1b", nope_dim=0), [90, 33], 16, seed=2)
    q = lay.queries(2)
    check_decode(lay, q, [90, 33], DecodeE4m3(lay, q, [90, 33], 90)())


def test_decode_many_sequences():
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 700)
    lens[[5, 699]] = [900, 0]
    lay = E4m3Layer(shape("tiny"), lens, 8, seed=4)
    q = lay.queries(len(lens))
    d = DecodeE4m3(lay, q, lens, 900)
    check_decode(lay, q, lens, d(), only=set(range(0, 700, 13)) | {5, 698, 699})
    d.guard()


def test_decode_lengths_are_clamped():
    lay = E4m3Layer(shape("05b"), [100, 100, 100, 100], 16, seed=9)
    q = lay.queries(4)
    check_decode(lay, q, [64, 64, 0, 64], DecodeE4m3(lay, q, [64, 2**31 - 1, -5, 70], 64)())
    lay.table = lay.table[:, :6]     # 96 positions
    lay.upload()
    check_decode(lay, q, [96, 96, 96, 5], DecodeE4m3(lay, q, [96, 100, 2000, 5], 4000)())


def test_decode_bad_page_is_nan_for_its_sequence_alone():
    lay = E4m3Layer(shape("1b"), [200, 200, 200, 200], 32, seed=11)
    lay.table[1, 3], lay.table[2, 6] = -1, 10**6
    lay.table[3, 6] = -7            # past the rows that are read below
    lay.upload()
    q = lay.queries(4)
    lens = [200, 200, 200, 192]
    got = DecodeE4m3(lay, q, lens, 200)()
    check_decode(lay, q, lens, got, only={0, 3})
    assert np.isnan(got[1:3].float().cpu().numpy()).all()


def test_decode_non_finite_rows_stay_in_their_sequence():
    lay = E4m3Layer(shape("8b"), [130, 130, 130], 16, seed=12)
    x = lay.pool[lay.table[1, 2], 5, :512].copy()
    x[17] = np.inf
    lay.edit(lay.table[1, 2], 5, x)
    lay.upload()
    q = lay.queries(3)
    got = DecodeE4m3(lay, q, [130] * 3, 130)()
    check_decode(lay, q, [130] * 3, got, only={0, 2})
    assert np.isnan(got[1].float().cpu().numpy()).all()


@pytest.mark.parametrize("spread", [4, 30])
def test_decode_rows_of_very_different_sizes(spread):
    """Powers from 2^-spread to 2^spread in one sequence, queries small enough that the logits stay
    moderate: small rows keep their softmax weight beside large ones, and their share of the sum."""
    lay = E4m3Layer(shape("1b"), [161, 70], 16, seed=13)
    q = lay.queries(2)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** -(spread + 2))
    e = lay.rng.integers(-spread, spread + 1, lay.power.shape)
    for b, n in enumerate([161, 70]):
        for p in range(n):
            at = lay.table[b, p // 16], p % 16
            lay.edit(*at, bf16(lay.pool[at][:512] * 2.0 ** e[at]))
    lay.upload()
    check_decode(lay, q, [161, 70], DecodeE4m3(lay, q, [161, 70], 161)())


def test_decode_rows_of_zeros():
    """Zeros among the rows (their power is the smallest), a whole sequence of zeros, and rows never
    written (a power of 0)."""
    lay = E4m3Layer(shape("05b"), [100, 40, 50], 16, seed=14)
    for p in range(0, 100, 3):
        lay.edit(lay.table[0, p // 16], p % 16, np.zeros(256))
    for p in range(40):
        lay.edit(lay.table[1, p // 16], p % 16, np.zeros(256))
    for p in range(0, 50, 2):
        lay.edit(lay.table[2, p // 16], p % 16, np.zeros(256))
        lay.power[lay.table[2, p // 16], p % 16] = 0.0
    lay.upload()
    q = lay.queries(3)
    got = DecodeE4m3(lay, q, [100, 40, 50], 100)()
    check_decode(lay, q, [100, 0, 50], got)


def test_decode_large_logits():
    """One row that takes all the weight, at each place of a tile, logits of about a thousand."""
    lens = [70] * 70
    lay = E4m3Layer(shape("tiny"), lens, 16, seed=15)
    q = np.zeros((70, 4, 96))
    q[..., 64] = 1000.0
    for b in range(70):
        for p in range(70):
            pe = np.zeros(32)
            pe[0] = 8.0 if p == b else 4.0
            lay.edit(lay.table[b, p // 16], p % 16, positional=pe)
    lay.upload()
    check_decode(lay, q, lens, DecodeE4m3(lay, q, lens, 70)())


def test_decode_repeats_its_bits_and_follows_its_lengths_in_a_graph():
    import torch
    lens = [400, 90, 0, 33]
    lay = E4m3Layer(shape("1b"), [500] * 4, 32, seed=16, poison=False)
    q = lay.queries(4)
    d = DecodeE4m3(lay, q, lens, 500)
    first = d().clone()
    d.ws.fill_(0x7B)
    assert torch.equal(d(), first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d()
    for k, now in enumerate(([400, 90, 0, 33], [1, 500, 499, 0], [77, 78, 79, 80], [0, 0, 0, 0])):
        d.lens.copy_(ints(now))
        lay.table = lay.table[[1, 2, 3, 0]]
        lay.d_table.copy_(ints(lay.table))
        d.o.fill_(3.0)
        graph.replay()
        got = d.o.clone()
        torch.cuda.synchronize()
        d.o.fill_(5.0)
        assert torch.equal(d(), got), k
        check_decode(lay, q, now, got)


def test_decode_position_past_32_bits_of_bytes():
    """Pages more than 8 GiB into the pool."""
    import torch
    lay = E4m3Layer(shape("8b"), [70, 65], 64, seed=17)
    size = lay.d_pool.shape[1]
    far = (1 << 33) // size + 3
    pool = torch.empty(far + 8, size, dtype=torch.uint8, device="cuda")
    table = lay.table.copy()
    for b in range(2):
        for k in range(2):
            pool[far + 2 * b + k] = lay.d_pool[lay.table[b, k]]
            table[b, k] = far + 2 * b + k
    q = lay.queries(2)
    lay.d_pool, lay.d_table = pool, ints(table)
    check_decode(lay, q, [70, 65], DecodeE4m3(lay, q, [70, 65], 70)())


# ---- prefill ---------------------------------------------------------------------------------
def prefill(lay, q, new, lens, extra=0):
    import torch
    from paper_2607_27269_amd import _lib as L
    cfg, cache = lay.handle()
    d_q, n_kv = up(q), int(sum(lens))
    q_off, kv_off = ints(np.concatenate([[0], np.cumsum(new)])), ints(np.concatenate([[0], np.cumsum(lens)]))
    o = torch.full((len(q), lay.cfg.n_heads, lay.cfg.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
    size = L.mla_recon_prefill_e4m3_workspace_size(cfg, len(q), n_kv)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    L.mla_recon_prefill_e4m3(cfg, d_q.data_ptr(), len(q), q_off.data_ptr(), cache, n_kv, kv_off.data_ptr(),
                             lay.d_Wuk.data_ptr(), lay.d_Wuv.data_ptr(), o.data_ptr(), ws.data_ptr(), size,
                             torch.cuda.current_stream().cuda_stream)
    return o.double().cpu().numpy()


@pytest.mark.parametrize("name,new,prefix,ps", [
    ("tiny", [1], [0], 1), ("tiny", [33, 1, 64], [0, 100, 5], 8), ("05b", [77], [0], 16), ("05b", [5, 130], [66, 0], 7),
    ("1b", [20, 1, 129], [300, 63, 0], 24), ("8b", [100, 3], [30, 500], 64)])
def test_prefill(name, new, prefix, ps):
    print(f"[e4m3] prefill {name} {new} after {prefix} page {ps}", flush=True)
    lens = [a + b for a, b in zip(new, prefix)]
    lay = E4m3Layer(shape(name), lens, ps, seed=ps)
    q = lay.queries(sum(new) + 2)                  # two rows of no sequence
    got = prefill(lay, q, new, lens)
    at = 0
    for b, t in enumerate(new):
        ref = lay.oracle(q[at:at + t], b, lens[b], prefix[b])
        for i in range(t):
            assert np.linalg.norm(got[at + i] - ref[i]) <= 1e-2 * np.linalg.norm(ref[i]), (b, i)
        at += t
    assert (got[at:] == 7.0).all()


def test_prefill_non_finite_latents_and_bad_pages():
    """NaN for exactly the queries that see the row, zeros and rows of other sizes beside them."""
    lay = E4m3Layer(shape("1b"), [60, 60], 16, seed=5)
    x = lay.pool[lay.table[0, 2], 3, :512].copy()
    x[3] = np.nan
    lay.edit(lay.table[0, 2], 3, x)                # position 35 of sequence 0
    lay.edit(lay.table[0, 0], 4, np.zeros(512))
    lay.table[1, 3] = -1                           # positions 48 .. of sequence 1
    lay.upload()
    q = lay.queries(120)
    got = prefill(lay, q, [60, 60], [60, 60])
    for b, first_bad in ((0, 35), (1, 48)):
        ref = lay.oracle(q[60 * b:60 * b + first_bad], b, first_bad, 0)
        for i in range(first_bad):
            assert np.linalg.norm(got[60 * b + i] - ref[i]) <= 1e-2 * np.linalg.norm(ref[i]), (b, i)
        assert np.isnan(got[60 * b + first_bad:60 * b + 60]).all()
