"""GPU tests of decoding behind shared prefixes, both cache formats, against float64 over each sequence's own
rows.  Tolerance: that of decoding (tests/test_gpu_paged.py)."""
import numpy as np
import pytest

from test_gpu_cache_e4m3 import E4m3Layer
from test_gpu_paged import Layer, bf16, check_decode, ints, shape, up

pytestmark = pytest.mark.gpu

GUARD = 4096


def make(name, fmt, members, shared, tails, ps, seed, lo=0, hi=0, **kw):
    """A layer whose groups' sequences have the pages of their first shared[g] rows in common (whole
    pages; the rest of the shared rows copied), `lo` sequences of no group before and `hi` behind."""
    lens = [50 + 9 * i for i in range(lo)]
    lens += [s + tails[k % len(tails)] for k, s in enumerate(s for m, s in zip(members, shared) for _ in range(m))]
    lens += [20 + 31 * i for i in range(hi)]
    lay = (E4m3Layer if fmt else Layer)(shape(name, **kw), lens, ps, seed=seed)
    b = lo
    for m, s in zip(members, shared):
        for i in range(b, b + m):
            lay.table[i, :s // ps] = lay.table[b, :s // ps]
            for p in range(s // ps * ps, s):
                src, dst = lay.table[b, p // ps], lay.table[i, p // ps]
                lay.pool[dst, p % ps] = lay.pool[src, p % ps]
                if fmt:
                    lay.codes[dst, p % ps], lay.power[dst, p % ps] = lay.codes[src, p % ps], lay.power[src, p % ps]
        b += m
    lay.upload()
    return lay, lens, np.concatenate([[0], np.cumsum(members)]) + lo


class Shared:
    def __init__(self, lay, q, lens, max_len, offsets, shared, fmt):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.lay, self.max_len, self.fmt, self.c = lay, max_len, int(fmt), lay.handle()
        self.n = len(shared)
        self.q, self.lens, self.off, self.shared = up(q), ints(lens), ints(offsets), ints(shared)
        self.o = torch.full((len(q), lay.cfg.n_heads, lay.cfg.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        self.size = L.mla_recon_decode_shared_workspace_size(self.c[0], self.fmt, max_len, self.n)
        assert self.size > 0, L.last_error()
        self.ws = torch.full((self.size + GUARD,), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.ws[self.size:] = 0xA5
        L.mla_recon_decode_shared(self.c[0], self.q.data_ptr(), self.c[1], self.fmt, self.max_len, self.lens.data_ptr(),
                                  self.n, self.off.data_ptr() if self.n else None,
                                  self.shared.data_ptr() if self.n else None, self.lay.d_Wuk.data_ptr(),
                                  self.lay.d_Wuv.data_ptr(), self.o.data_ptr(), self.ws.data_ptr(), self.size,
                                  torch.cuda.current_stream().cuda_stream)
        return self.o

    def guard(self):
        assert bool((self.ws[self.size:] == 0xA5).all()), "written behind the workspace"


FORMATS = pytest.mark.parametrize("fmt", [False, True], ids=["bf16", "e4m3"])


@FORMATS
@pytest.mark.parametrize("name,members,shared,ps", [
    ("tiny", [2], [64], 16), ("tiny", [9], [300], 7), ("05b", [4], [1000], 16), ("05b", [1, 3, 2], [65, 31, 500], 32),
    ("1b", [5, 6], [128, 33], 16), ("8b", [4], [256], 64), ("8b", [3, 1, 13], [700, 90, 95], 24)])
def test_groups(name, members, shared, ps, fmt):
    print(f"[shared] {name} {members} x {shared} page {ps} {'e4m3' if fmt else 'bf16'}", flush=True)
    lay, lens, off = make(name, fmt, members, shared, [1, 40, 3, 70, 32], ps, seed=ps)
    q = lay.queries(len(lens))
    d = Shared(lay, q, lens, max(lens), off, shared, fmt)
    check_decode(lay, q, lens, d())
    d.guard()


@FORMATS
@pytest.mark.parametrize("H,G", [(1, 1), (14, 2), (33, 1), (40, 8), (64, 2), (128, 128)])
def test_head_counts(H, G, fmt):
    print(f"[shared] {H} heads in {G} groups", flush=True)
    lay, lens, off = make("05b", fmt, [5, 2], [200, 64], [7, 33], 16, seed=H, n_heads=H, s_kv_groups=G, n_kv_groups=G)
    q = lay.queries(len(lens))
    d = Shared(lay, q, lens, max(lens), off, [200, 64], fmt)
    check_decode(lay, q, lens, d())
    d.guard()


@FORMATS
def test_sequences_of_no_group(fmt):
    lay, lens, off = make("1b", fmt, [3, 4], [96, 160], [5, 50], 32, seed=3, lo=2, hi=3)
    q = lay.queries(len(lens))
    d = Shared(lay, q, lens, max(lens), off, [96, 160], fmt)
    check_decode(lay, q, lens, d())
    d.guard()


@FORMATS
def test_no_groups_and_empty_groups(fmt):
    lay, lens, off = make("05b", fmt, [4], [100], [9, 64], 16, seed=4)
    q = lay.queries(4)
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), [0], [], fmt)())
    # groups without sequences, with sequences and without rows, and all of them
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), [0, 0, 4, 4], [70, 100, 5], fmt)())
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), [0, 2, 4], [0, 100], fmt)())
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), [2, 2], [100], fmt)())


@FORMATS
def test_lengths_below_the_shared_rows(fmt):
    """Sequences with fewer rows than their group shares, none among them; shared lengths past max_len and
    negative ones."""
    lay, lens, off = make("8b", fmt, [5], [200], [1, 30], 16, seed=5)
    q = lay.queries(5)
    now = [190, 230, 64, 0, 201]
    check_decode(lay, q, now, Shared(lay, q, now, 230, off, [200], fmt)())
    check_decode(lay, q, [0] * 5, Shared(lay, q, [0] * 5, 230, off, [200], fmt)())
    lay.table[0] = 10**6              # (nothing of a sequence without rows is looked at)
    lay.d_table.copy_(ints(lay.table))
    now = [0, 230, 201, 210, 201]
    check_decode(lay, q, now, Shared(lay, q, now, 230, off, [200], fmt)())
    now = [0, 1, 2, 7, 0]
    check_decode(lay, q, now, Shared(lay, q, now, 230, off, [200], fmt)())
    lens[0] = 0
    check_decode(lay, q, lens, Shared(lay, q, lens, 231, off, [-5], fmt)())
    same = [0] + [200] * 4
    check_decode(lay, q, same, Shared(lay, q, [-1, 201, 2**31 - 1, 230, 210], 200, off, [2**31 - 1], fmt)())


@FORMATS
def test_many_sequences_and_groups(fmt):
    """More sequences and groups than workgroups."""
    rng = np.random.default_rng(6)
    members = rng.integers(1, 4, 300)
    shared = [int(s) for s in rng.integers(0, 100, 300)]
    lay, lens, off = make("tiny", fmt, members, shared, [int(t) for t in rng.integers(1, 30, 41)], 8, seed=6)
    q = lay.queries(len(lens))
    d = Shared(lay, q, lens, max(lens), off, shared, fmt)
    check_decode(lay, q, lens, d(), only=set(range(0, len(lens), 17)))
    d.guard()


@FORMATS
def test_one_large_group(fmt):
    """One group of 130 sequences behind 2000 rows."""
    lay, lens, off = make("05b", fmt, [130], [2000], [1, 2, 40], 64, seed=7)
    q = lay.queries(130)
    d = Shared(lay, q, lens, max(lens), off, [2000], fmt)
    check_decode(lay, q, lens, d(), only=set(range(0, 130, 9)) | {129})
    d.guard()


# Groups of 16 blocks of 32 heads and more on the average: the shared rows' tiles are made fp16 by the launch before.
@FORMATS
@pytest.mark.parametrize("name,members,shared,ps", [
    ("tiny", [17], [300], 7), ("05b", [16, 20], [1000, 95], 16), ("05b", [2, 40, 0, 30], [500, 64, 77, 31], 100),
    ("1b", [40], [129], 24), ("8b", [33], [700], 64)])
def test_large_groups(name, members, shared, ps, fmt):
    print(f"[shared] {name} {members} x {shared} page {ps} {'e4m3' if fmt else 'bf16'}", flush=True)
    lay, lens, off = make(name, fmt, members, shared, [1, 40, 3, 70, 32], ps, seed=ps)
    q = lay.queries(len(lens))
    d = Shared(lay, q, lens, max(lens), off, shared, fmt)
    check_decode(lay, q, lens, d())
    d.guard()


@FORMATS
def test_large_groups_of_too_many_rows_for_a_copy(fmt):
    """The same groups where max_len allows more shared rows than the workspace has room for."""
    lay, lens, off = make("tiny", fmt, [17], [300], [1, 40], 64, seed=20)
    lay.table = np.pad(lay.table, ((0, 0), (0, (1 << 20) // 64)), constant_values=-1)
    lay.upload()
    q = lay.queries(17)
    d = Shared(lay, q, lens, 1 << 20, off, [300], fmt)
    check_decode(lay, q, lens, d())
    d.guard()
    check_decode(lay, q, lens, Shared(lay, q, lens, 1 << 15, off, [300], fmt)())


@FORMATS
def test_large_groups_of_many_heads(fmt):
    lay, lens, off = make("05b", fmt, [5, 6], [200, 64], [7, 33], 16, seed=21, n_heads=128, s_kv_groups=8, n_kv_groups=8)
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), off, [200, 64], fmt)())


@FORMATS
def test_large_groups_with_short_members_and_bad_pages(fmt):
    """Sequences with fewer rows than the group shares, without rows (whose table is not looked at), and a shared
    row on no page: NaN for its group alone."""
    lay, lens, off = make("8b", fmt, [20, 20], [200, 128], [1, 30], 16, seed=22)
    q = lay.queries(40)
    now = [0, 190, 201, 64, 201] + lens[5:]                     # (of 201, 230, 201, 230, .. rows that there are)
    lay.table[0] = 10**6
    lay.d_table.copy_(ints(lay.table))
    check_decode(lay, q, now, Shared(lay, q, now, 231, off, [200, 128], fmt)())
    check_decode(lay, q, [0] * 40, Shared(lay, q, [0] * 40, 231, off, [200, 128], fmt)())
    check_decode(lay, q, now, Shared(lay, q, now, 231, off, [-5, 2**31 - 1], fmt)(), only=set(range(20)))
    lay.table[20:, 1] = -1
    lay.d_table.copy_(ints(lay.table))
    got = Shared(lay, q, now, 231, off, [200, 128], fmt)()
    check_decode(lay, q, now, got, only=set(range(20)))
    assert np.isnan(got[20:].float().cpu().numpy()).all()


@FORMATS
def test_large_groups_of_rows_of_very_different_sizes(fmt):
    """Powers from 2^-30 to 2^30, and rows of zeros, among the shared rows; queries small enough that the logits
    stay moderate."""
    lay, lens, off = make("1b", fmt, [18], [160], [5, 40], 16, seed=23)
    q = lay.queries(18)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** -32)
    for p in range(160):
        at = lay.table[0, p // 16], p % 16
        row = bf16(lay.pool[at][:512] * (0.0 if p % 7 == 0 else 2.0 ** lay.rng.integers(-30, 31)))
        if fmt:
            lay.edit(*at, row)
        else:
            lay.pool[at][:512] = row
    lay.upload()
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), off, [160], fmt)())


@FORMATS
def test_large_groups_non_finite_rows_stay_in_their_group(fmt):
    lay, lens, off = make("05b", fmt, [18, 18], [96, 96], [5, 40], 16, seed=24)
    at = lay.table[0, 2], 3
    if fmt:
        lay.edit(*at, np.where(np.arange(256) == 9, np.inf, lay.pool[at][:256]))
    else:
        lay.pool[at][9] = np.inf
    lay.upload()
    q = lay.queries(36)
    got = Shared(lay, q, lens, max(lens), off, [96, 96], fmt)()
    check_decode(lay, q, lens, got, only=set(range(18, 36)))
    assert np.isnan(got[:18].float().cpu().numpy()).any(axis=(1, 2)).all()


@FORMATS
@pytest.mark.parametrize("n", [1, 3])
def test_the_longest_sequences(n, fmt):
    """2^31 - 1 rows, of two pages again and again, all of one weight (zero queries).  A wavefront's sums of the
    weights and of the latents (1, 2 and 3; 2^21 rows) are whole numbers below 2^24, so only the output rounds."""
    import torch
    from paper_2607_27269_amd import _lib as L
    rows, ps = 2**31 - 1, 1 << 16
    lay = (E4m3Layer if fmt else Layer)(shape("tiny"), [2 * ps], ps, seed=n)
    rkv = lay.cfg.kv_rank
    for name in ("codes", "power"):                              # (made again of the rows below)
        if fmt:
            delattr(lay, name)
    lay.pool[..., :rkv] = np.random.default_rng(n).integers(1, 4, lay.pool[..., :rkv].shape)
    lay.upload()
    table = np.tile(lay.table[:1, :2], (n, rows // ps // 2 + 1))[:, :rows // ps + 1]
    first, second = (lay.pool[lay.table[0, k], :, :rkv] for k in (0, 1))
    mean = (2**14 * (first.sum(0) + second.sum(0)) - second[-1]) / rows   # 2^15 pages, of the last all rows but one
    q = torch.zeros(n, lay.cfg.n_heads, lay.cfg.nope_dim + lay.cfg.rope_dim, dtype=torch.bfloat16, device="cuda")
    o = torch.empty(n, lay.cfg.n_heads, lay.cfg.head_dim, dtype=torch.bfloat16, device="cuda")
    d_table, lens, off, shared = ints(table), ints([rows] * n), ints([0, n]), ints([rows])
    cfg, cache = L.make_cfg(lay.cfg.replace(batch=n, seq=1)), L.PagedCache(
        lay.d_pool.data_ptr(), d_table.data_ptr(), len(lay.d_pool), ps, table.shape[1])
    size = L.mla_recon_decode_shared_workspace_size(cfg, int(fmt), rows, 1)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L.mla_recon_decode_shared(cfg, q.data_ptr(), cache, int(fmt), rows, lens.data_ptr(), 1, off.data_ptr(),
                              shared.data_ptr(), lay.d_Wuk.data_ptr(), lay.d_Wuv.data_ptr(), o.data_ptr(), ws.data_ptr(),
                              size, torch.cuda.current_stream().cuda_stream)
    per = lay.cfg.n_heads // lay.cfg.s_kv_groups
    want = (lay.Wuv @ mean).reshape(lay.cfg.s_kv_groups, -1)
    got = o.double().cpu().numpy()
    for h in range(lay.cfg.n_heads):                             # the output's rounding, and the latents' second part's
        ref = want[h // per]
        assert np.linalg.norm(got[:, h] - ref, axis=-1).max() <= (2.0 ** -8 + 2.0 ** -15) * np.linalg.norm(ref), h


@FORMATS
def test_bad_pages(fmt):
    """A shared row on no page: NaN for the group; a row of one sequence's own: for that one."""
    lay, lens, off = make("1b", fmt, [3, 3], [128, 128], [40], 32, seed=8)
    lay.table[0:3, 1] = -1
    lay.table[4, 4] = 10**6
    lay.upload()
    q = lay.queries(6)
    got = Shared(lay, q, lens, max(lens), off, [128, 128], fmt)()
    check_decode(lay, q, lens, got, only={3, 5})
    assert np.isnan(got[[0, 1, 2, 4]].float().cpu().numpy()).all()


@FORMATS
def test_large_logits(fmt):
    """The row with all the weight in the shared part or behind it, logits of about a thousand."""
    lay, lens, off = make("tiny", fmt, [6], [96], [40], 16, seed=9)
    q = np.zeros((6, 4, 96))
    for b, where in enumerate([0, 31, 32, 95, 96, 135]):
        q[b, :, 64 + b] = 1000.0
        for p in range(136):
            lay.pool[lay.table[b, p // 16], p % 16, 128 + b] = 8.0 if p == where else 4.0
    lay.upload()
    check_decode(lay, q, lens, Shared(lay, q, lens, 136, off, [96], fmt)())


@FORMATS
def test_large_groups_repeat_their_bits_and_follow_their_arrays_in_a_graph(fmt):
    import torch
    lay, lens, off = make("05b", fmt, [20, 16], [160, 96], [30, 1, 65], 32, seed=25)
    q = lay.queries(36)
    d = Shared(lay, q, lens, 300, off, [160, 96], fmt)
    first = d().clone()
    d.ws.fill_(0x7B)
    assert torch.equal(d(), first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d()
    for k, (now, o, s) in enumerate(((lens, off, [160, 96]), ([100] * 20 + [90] * 16, off, [100, 90]),
                                     (lens, [0, 2, 20], [160, 160]), ([0] * 36, off, [160, 96]), (lens, [0, 0, 0], [5, 5]))):
        d.lens.copy_(ints(now)), d.off.copy_(ints(o)), d.shared.copy_(ints(s))
        d.o.fill_(3.0)
        graph.replay()
        got = d.o.clone()
        torch.cuda.synchronize()
        d.o.fill_(5.0)
        assert torch.equal(d(), got), k
        check_decode(lay, q, now, got)


@FORMATS
def test_repeats_its_bits_and_follows_its_arrays_in_a_graph(fmt):
    import torch
    lay, lens, off = make("1b", fmt, [4, 3], [160, 96], [30, 1, 65], 32, seed=10)
    q = lay.queries(7)
    d = Shared(lay, q, lens, 300, off, [160, 96], fmt)
    first = d().clone()
    d.ws.fill_(0x7B)
    assert torch.equal(d(), first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d()
    for k, (now, o, s) in enumerate(((lens, off, [160, 96]), ([100] * 4 + [90] * 3, off, [100, 90]),
                                     (lens, [0, 2, 4], [160, 160]), ([0] * 7, off, [160, 96]), (lens, [0, 0, 0], [5, 5]))):
        d.lens.copy_(ints(now)), d.off.copy_(ints(o)), d.shared.copy_(ints(s))
        d.o.fill_(3.0)
        graph.replay()
        got = d.o.clone()
        torch.cuda.synchronize()
        d.o.fill_(5.0)
        assert torch.equal(d(), got), k
        check_decode(lay, q, now, got)


@FORMATS
def test_two_streams_with_their_own_workspaces(fmt):
    import torch
    lay, lens, off = make("8b", fmt, [6], [512], [40, 1, 100], 64, seed=11)
    a = Shared(lay, lay.queries(6), lens, max(lens), off, [512], fmt)
    b = Shared(lay, lay.queries(6), lens, max(lens), [0, 3, 6], [320, 512], fmt)
    want = a().clone(), b().clone()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.o.zero_(), b.o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            a()
        with torch.cuda.stream(s2):
            b()
        torch.cuda.synchronize()
        assert torch.equal(a.o, want[0]) and torch.equal(b.o, want[1])
