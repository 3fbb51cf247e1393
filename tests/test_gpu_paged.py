"""GPU tests of the operators on a paged latent cache against the float64 oracle (oracle/paged_oracle.py).

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value (half a step), rms about 2^-8 / 2.3
= 1.7e-3.  append: one rounding of the result (bf16 2^-8, fp32 2^-24 relative) plus the fp32 rotation: the
turn's fraction rounded to fp32 (2 pi 2^-26 = 1e-7), sine and cosine within 2 ulp (1.2e-7), two products
and a sum (1.8e-7), together below 1e-6 of |lo| + |hi|.  decode: the absorbed query, the probabilities,
the weighted latent and the output are rounded to bf16, the first of them times the logits' spread
(about 1.5): 1.7e-3 sqrt(1.5^2 + 3) = 3.9e-3 of the norm expected, 1e-2 allowed.  prefill: the expanded
keys (times the spread), the expanded values, the probabilities and the output: the same.
"""
import numpy as np
import pytest

from oracle import paged_oracle as PO
from paper_2607_27269_amd import configs

pytestmark = pytest.mark.gpu

REL = 1e-2


def bf16(x):
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) >> 16
    return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def up(x, dtype="bf16"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.to(torch.bfloat16) if dtype == "bf16" else t).cuda()


def ints(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def shape(name, **kw):
    """A bf16 layer: one of the configurations, or the tiny one's widths."""
    if name == "tiny":
        return configs.get(0).replace(dtype="bf16", **kw)
    return configs.get({"05b": 1, "1b": 2, "8b": 3}[name]).replace(**kw)


def scatter(rng, lens, ps, spare=2, extra=0, unused=-1):
    """A page table over scattered pages, unused entries `unused`, and the pool's size in pages."""
    need = [-(-int(n) // ps) for n in lens]
    total = sum(need) + spare
    order = rng.permutation(total)
    table = np.full((len(lens), max(1, max(need)) + extra), unused, dtype=np.int64)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    return table, total


class Layer:
    """Weights and a cache of one layer, on the host in float64 and on the GPU."""

    def __init__(self, cfg, lens, ps, seed, spare=2, extra=0, poison=True):
        rng = self.rng = np.random.default_rng(seed)
        self.cfg, self.lens, self.ps = cfg, [int(n) for n in lens], ps
        self.W = cfg.kv_rank + cfg.rope_dim
        self.table, total = scatter(rng, lens, ps, spare, extra)
        self.pool = bf16(rng.standard_normal((total, ps, self.W)))
        if poison:   # rows that belong to nobody: spare pages, and the ends of last pages
            used = np.zeros((total, ps), dtype=bool)
            for b, n in enumerate(self.lens):
                for p in range(n):
                    used[self.table[b, p // ps], p % ps] = True
            self.pool[~used] = np.nan
        G, dn, dv, rkv = cfg.s_kv_groups, cfg.nope_dim, cfg.head_dim, cfg.kv_rank
        self.Wuk = bf16(rng.standard_normal((G * dn, rkv)) / np.sqrt(rkv))
        self.Wuv = bf16(rng.standard_normal((G * dv, rkv)) / np.sqrt(rkv))
        self.upload()

    def upload(self):
        self.d_pool, self.d_table = up(self.pool), ints(self.table)
        self.d_Wuk, self.d_Wuv = up(self.Wuk), up(self.Wuv)

    def queries(self, n):
        c = self.cfg
        return bf16(self.rng.standard_normal((n, c.n_heads, c.nope_dim + c.rope_dim)))

    def handle(self, batch=None):
        from paper_2607_27269_amd import _lib as L
        c = L.make_cfg(self.cfg.replace(batch=batch or len(self.table), seq=1))
        return c, L.PagedCache(self.d_pool.data_ptr(), self.d_table.data_ptr(), *self.d_pool.shape[:2],
                               self.d_table.shape[1])

    def oracle(self, q, b, n, first):
        c = self.cfg
        return PO.attend(q, PO.cached_rows(self.pool, self.table, b, n), self.Wuk, self.Wuv, nope_dim=c.nope_dim,
                         scale=float(np.float32(c.softmax_scale)), n_groups=c.s_kv_groups, first=first)


class Decode:
    """A decoding call's buffers; ``__call__`` enqueues it."""

    def __init__(self, layer, q, lens, max_len, d_Wuk=None):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.layer, self.max_len, self.c = layer, max_len, layer.handle()
        self.q, self.lens = up(q), ints(lens)
        self.Wuk = layer.d_Wuk if d_Wuk is None else d_Wuk
        self.o = torch.full((len(q), layer.cfg.n_heads, layer.cfg.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        size = L.mla_recon_decode_paged_workspace_size(self.c[0], max_len)
        assert size > 0, L.last_error()
        # what scratch holds must not matter
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        import torch
        from paper_2607_27269_amd import _lib as L
        L.mla_recon_decode_paged(self.c[0], self.q.data_ptr(), self.c[1], self.max_len, self.lens.data_ptr(),
                                 self.Wuk.data_ptr(), self.layer.d_Wuv.data_ptr(), self.o.data_ptr(),
                                 self.ws.data_ptr(), self.ws.numel(), torch.cuda.current_stream().cuda_stream)
        return self.o


def check_decode(layer, q, lens, got, only=None):
    got = got.double().cpu().numpy()
    for b, n in enumerate(lens):
        if only is not None and b not in only:
            continue
        if n <= 0:
            assert not got[b].any(), (b, n)
            continue
        ref = layer.oracle(q[b:b + 1], b, n, n - 1)[0]
        e = np.linalg.norm(got[b] - ref) / np.linalg.norm(ref)
        assert e <= REL, (b, n, e)


EDGES = [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("name,ps", [("tiny", 1), ("tiny", 64), ("05b", 7), ("05b", 16), ("05b", 128), ("1b", 16),
                                     ("1b", 100), ("8b", 24), ("8b", 32), ("8b", 64)])
def test_decode_edges(name, ps):
    print(f"[paged] decode {name} page {ps}", flush=True)
    lay = Layer(shape(name), EDGES, ps, seed=ps)
    q = lay.queries(len(EDGES))
    d = Decode(lay, q, EDGES, max(EDGES))
    check_decode(lay, q, EDGES, d())


@pytest.mark.parametrize("name,lens,ps", [("8b", [3000], 64), ("05b", [1], 16), ("05b", [5000, 3, 0, 2049], 16),
                                          ("1b", [777] * 9 + [0] * 3, 32), ("tiny", [9000, 8191], 48)])
def test_decode_long(name, lens, ps):
    print(f"[paged] decode {name} {lens} page {ps}", flush=True)
    lay = Layer(shape(name), lens, ps, seed=len(lens))
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Decode(lay, q, lens, max(lens))())


@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (33, 1), (40, 8), (64, 2)])
def test_decode_head_counts(H, G):
    print(f"[paged] decode {H} heads in {G} groups", flush=True)
    lens = [150, 0, 64, 1, 333]
    lay = Layer(shape("05b", n_heads=H, s_kv_groups=G, n_kv_groups=G), lens, 16, seed=H)
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Decode(lay, q, lens, 333)())


def test_decode_many_sequences():
    """More sequences than workgroups, most of them short."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 700)
    lens[[5, 699]] = [900, 0]
    print("[paged] decode 700 sequences", flush=True)
    lay = Layer(shape("tiny"), lens, 8, seed=4)
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Decode(lay, q, lens, 900)(), only=set(range(0, 700, 13)) | {5, 698, 699})


def test_decode_lengths_are_clamped():
    """Lengths beyond max_len, beyond the table, and negative ones."""
    lay = Layer(shape("05b"), [100, 100, 100, 100], 16, seed=9)
    q = lay.queries(4)
    d = Decode(lay, q, [64, 2**31 - 1, -5, 70], 64)
    check_decode(lay, q, [64, 64, 0, 64], d())
    lay.table = lay.table[:, :6]     # 96 positions
    lay.upload()
    d = Decode(lay, q, [96, 100, 2000, 5], 4000)
    check_decode(lay, q, [96, 96, 96, 5], d())


def test_decode_shared_pages_and_unaligned_weights():
    """Forked sequences read the same pages; W_UK at an odd address."""
    import torch
    lay = Layer(shape("8b"), [300, 200, 64], 64, seed=10)
    lay.table[1, :3] = lay.table[0, :3]
    lay.table[2, 0] = lay.table[0, 0]
    lay.upload()
    q = lay.queries(3)
    buf = torch.empty(lay.d_Wuk.numel() + 1, dtype=torch.bfloat16, device="cuda")
    buf[1:] = lay.d_Wuk.reshape(-1)
    lens = [300, 150, 64]
    check_decode(lay, q, lens, Decode(lay, q, lens, 300, d_Wuk=buf[1:])())


def test_decode_bad_page_is_nan_for_its_sequence_alone():
    lay = Layer(shape("1b"), [200, 200, 200, 200], 32, seed=11)
    lay.table[1, 3], lay.table[2, 6] = -1, 10**6
    lay.table[3, 6] = -7            # past the rows that are read below
    lay.upload()
    q = lay.queries(4)
    lens = [200, 200, 200, 192]
    got = Decode(lay, q, lens, 200)()
    check_decode(lay, q, lens, got, only={0, 3})
    assert np.isnan(got[1:3].float().cpu().numpy()).all()


def test_decode_non_finite_rows_stay_in_their_sequence():
    lay = Layer(shape("8b"), [130, 130, 130], 16, seed=12)
    lay.pool[lay.table[1, 2], 5, 17] = np.inf
    lay.upload()
    q = lay.queries(3)
    got = Decode(lay, q, [130] * 3, 130)()
    check_decode(lay, q, [130] * 3, got, only={0, 2})
    assert not np.isfinite(got[1].float().cpu().numpy()).all()


def test_decode_large_logits():
    """Logits of several hundred, growing along the cache: the running maximum moves all the time."""
    lens = [513, 65]
    lay = Layer(shape("05b"), lens, 16, seed=13)
    q = lay.queries(2)
    q[1] *= 0
    for b, n in enumerate(lens):
        for p in range(n):
            lay.pool[lay.table[b, p // 16], p % 16] = bf16(lay.pool[lay.table[b, p // 16], p % 16] * (1 + p / 32))
    lay.upload()
    q = bf16(q * 4)
    got = Decode(lay, q, lens, 513)().double().cpu().numpy()
    # logits s ~ 1.5 x 4 x 17 = 100 carry a rounding of 2^-9 relative from the absorbed query: an error
    # of 0.2 in the exponent, so only the dominated rows are certain: compare where one row holds
    # more than 99.9% of the weight, and the sequence of equal logits (q = 0) as usual
    ref = lay.oracle(q[1:2], 1, 65, 64)[0]
    assert np.linalg.norm(got[1] - ref) <= REL * np.linalg.norm(ref)
    assert np.isfinite(got).all()
    c, g = lay.cfg, lay.cfg.n_heads // lay.cfg.s_kv_groups
    rows = PO.cached_rows(lay.pool, lay.table, 0, 513)
    sure = 0
    for h in range(c.n_heads):
        k = np.concatenate([rows[:, :c.kv_rank] @ lay.Wuk[(h // g) * 64:(h // g) * 64 + 64].T, rows[:, c.kv_rank:]], 1)
        s = np.sort(k @ q[0, h] * c.softmax_scale)
        if s[-1] - s[-2] > 14:       # e^-14 512 < 5e-4, and 0.2 of error either way
            sure += 1
            ref = lay.oracle(q[:1, :], 0, 513, 512)[0, h]
            assert np.linalg.norm(got[0, h] - ref) <= REL * np.linalg.norm(ref), h
    assert sure >= 3


def test_decode_repeats_its_bits_and_follows_its_lengths_in_a_graph():
    """A captured call replayed while lengths, tables and queries change between the replays, each
    replay against the eager call; and the same bits from scratch with other contents."""
    import torch
    lens = [400, 90, 0, 33]
    lay = Layer(shape("1b"), [500] * 4, 32, seed=14, poison=False)
    q = lay.queries(4)
    d = Decode(lay, q, lens, 500)
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


def test_decode_on_two_streams_with_their_own_workspaces():
    import torch
    lay = Layer(shape("8b"), [1500, 1200, 700], 64, seed=15)
    q = lay.queries(6)
    a, b = Decode(lay, q[:3], [1500, 1200, 700], 1500), Decode(lay, q[3:], [3, 1200, 699], 1500)
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
    check_decode(lay, q[:3], [1500, 1200, 700], a.o)
    check_decode(lay, q[3:], [3, 1200, 699], b.o)


def test_decode_position_past_32_bits_of_bytes():
    """A page whose rows lie more than 4 GiB (and 2^31 elements) into the pool."""
    import torch
    cfg = shape("8b")
    lay = Layer(cfg, [70, 65], 64, seed=16)
    far = (1 << 32) // (64 * lay.W) + 3          # 2^32 elements, 8 GiB
    pool = torch.empty(far + 8, 64, lay.W, dtype=torch.bfloat16, device="cuda")
    table = lay.table.copy()
    for b in range(2):
        for k in range(2):
            pool[far + 2 * b + k] = lay.d_pool[lay.table[b, k]]
            table[b, k] = far + 2 * b + k
    q = lay.queries(2)
    lay.d_pool, lay.d_table = pool, ints(table)
    check_decode(lay, q, [70, 65], Decode(lay, q, [70, 65], 70)())


def test_decode_longest_length():
    """2^31 - 1 rows, the largest length (one page of 65536 rows again and again): the attention over the
    page's rows, of which one is there 32767 times and the others 32768 times."""
    lay = Layer(shape("tiny"), [65536], 65536, seed=17, spare=0)
    lay.table = np.zeros((1, 32768), dtype=np.int64)
    lay.upload()
    q = lay.queries(1)
    n = 2**31 - 1
    print("[paged] decode 2^31 - 1 rows", flush=True)
    check_decode(lay, q, [65536], Decode(lay, q, [n], n)())


def test_decode_most_sequences():
    """65535 sequences, the largest batch."""
    rng = np.random.default_rng(18)
    lens = rng.integers(0, 4, 65535)
    lens[[0, 40000, 65534]] = [70, 33, 3]
    print("[paged] decode 65535 sequences", flush=True)
    lay = Layer(shape("tiny"), lens, 4, seed=18)
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Decode(lay, q, lens, 70)(), only=set(range(0, 65535, 997)) | {40000, 65533, 65534})


def test_decode_without_non_positional_keys():
    """d_nope = 0: no W_UK, the key is the positional key alone."""
    lens = [40, 0, 95, 1]
    lay = Layer(shape("05b", nope_dim=0, rope_dim=64, kv_rank=512), lens, 16, seed=19)
    q = lay.queries(len(lens))
    check_decode(lay, q, lens, Decode(lay, q, lens, 95)())


# ---- prefill --------------------------------------------------------------------------------
class Prefill:
    def __init__(self, layer, q, q_off, kv_off, n_kv=None):
        import torch
        from paper_2607_27269_amd import _lib as L
        self.layer, self.c = layer, layer.handle(len(q_off) - 1)
        self.q, self.q_off, self.kv_off = up(q), ints(q_off), ints(kv_off)
        self.n_q, self.n_kv = len(q), int(kv_off[-1]) if n_kv is None else n_kv
        self.o = torch.full((max(1, len(q)), layer.cfg.n_heads, layer.cfg.head_dim), 7.0, dtype=torch.bfloat16,
                            device="cuda")
        size = L.mla_recon_prefill_paged_workspace_size(self.c[0], self.n_q, self.n_kv)
        assert size > 0, L.last_error()
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        import torch
        from paper_2607_27269_amd import _lib as L
        L.mla_recon_prefill_paged(self.c[0], self.q.data_ptr(), self.n_q, self.q_off.data_ptr(), self.c[1], self.n_kv,
                                  self.kv_off.data_ptr(), self.layer.d_Wuk.data_ptr(), self.layer.d_Wuv.data_ptr(),
                                  self.o.data_ptr(), self.ws.data_ptr(), self.ws.numel(),
                                  torch.cuda.current_stream().cuda_stream)
        return self.o


def offsets(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int64)


def check_prefill(layer, q, q_off, kv_lens, got, only=None):
    got = got.double().cpu().numpy()
    for b, n in enumerate(kv_lens):
        if only is not None and b not in only:
            continue
        lo, hi = int(q_off[b]), int(q_off[b + 1])
        if lo == hi:
            continue
        ref = layer.oracle(q[lo:hi], b, n, n - (hi - lo))
        for t in range(lo, hi):
            if n - (hi - t) < 0:
                assert not got[t].any(), (b, t)
                continue
            e = np.linalg.norm(got[t] - ref[t - lo]) / np.linalg.norm(ref[t - lo])
            assert e <= REL, (b, n, t - lo, e)


@pytest.mark.parametrize("name,ps", [("tiny", 1), ("tiny", 64), ("05b", 16), ("05b", 7), ("1b", 32), ("8b", 24), ("8b", 64)])
def test_prefill_edges(name, ps):
    """Whole prompts, continued ones, single tokens, none, and more queries than rows."""
    new = [1, 31, 33, 0, 64, 65, 1, 130, 5, 7, 40]
    kv = [1, 31, 33, 20, 64, 65, 99, 200, 0, 3, 300]
    print(f"[paged] prefill {name} page {ps}", flush=True)
    lay = Layer(shape(name), kv, ps, seed=20 + ps)
    q, q_off = lay.queries(sum(new)), offsets(new)
    check_prefill(lay, q, q_off, kv, Prefill(lay, q, q_off, offsets(kv))())


@pytest.mark.parametrize("name,new,kv", [("8b", [257, 1], [257, 600]), ("05b", [300, 77, 512], [300, 77, 512]),
                                         ("1b", [3, 260], [900, 1000]), ("05b", [1], [1])])
def test_prefill_longer(name, new, kv):
    print(f"[paged] prefill {name} {new} of {kv}", flush=True)
    lay = Layer(shape(name), kv, 32, seed=sum(new))
    q, q_off = lay.queries(sum(new)), offsets(new)
    check_prefill(lay, q, q_off, kv, Prefill(lay, q, q_off, offsets(kv))())


@pytest.mark.parametrize("H,G", [(1, 1), (6, 3), (12, 2), (40, 8)])
def test_prefill_head_counts(H, G):
    new, kv = [70, 3], [70, 90]
    print(f"[paged] prefill {H} heads in {G} groups", flush=True)
    lay = Layer(shape("05b", n_heads=H, s_kv_groups=G, n_kv_groups=G), kv, 16, seed=H)
    q, q_off = lay.queries(sum(new)), offsets(new)
    check_prefill(lay, q, q_off, kv, Prefill(lay, q, q_off, offsets(kv))())


def test_prefill_without_non_positional_keys():
    """d_nope = 0: the key is the positional key alone."""
    new, kv = [40, 9], [40, 50]
    lay = Layer(shape("05b", nope_dim=0, rope_dim=64, kv_rank=512), kv, 16, seed=31)
    q, q_off = lay.queries(sum(new)), offsets(new)
    check_prefill(lay, q, q_off, kv, Prefill(lay, q, q_off, offsets(kv))())


def test_prefill_without_non_positional_keys_long():
    new, kv = [60, 1], [2900, 333]
    lay = Layer(shape("1b", nope_dim=0), kv, 64, seed=37)
    q, q_off = lay.queries(sum(new)), offsets(new)
    check_prefill(lay, q, q_off, kv, Prefill(lay, q, q_off, offsets(kv))())


def test_prefill_padded_batch_leaves_rows_of_no_sequence():
    """Rows before the first and behind the last sequence, room for more cached rows than there are."""
    new, kv = [50, 20], [50, 64]
    lay = Layer(shape("8b"), kv, 16, seed=32)
    q, q_off = lay.queries(100), offsets(new, first=5)
    p = Prefill(lay, q, q_off, offsets(kv), n_kv=500)
    got = p()
    check_prefill(lay, q, q_off, kv, got)
    got = got.float().cpu().numpy()
    assert (got[:5] == 7.0).all() and (got[75:] == 7.0).all()


def test_prefill_non_finite_rows_reach_only_the_queries_that_see_them():
    new, kv = [100, 100, 100], [100, 150, 100]
    lay = Layer(shape("1b"), kv, 16, seed=33)
    lay.pool[lay.table[0, 4], 6, 3] = np.inf                 # position 70
    lay.pool[lay.table[1, 6], 4, lay.W - 1] = np.nan         # position 100, a positional key
    lay.table[2, 5] = -3                                     # positions 80 .. 95: no page
    lay.upload()
    q, q_off = lay.queries(300), offsets(new)
    got = Prefill(lay, q, q_off, offsets(kv))().float().cpu().numpy()
    for b, first in enumerate((70, 100 - 50, 80)):
        o = got[100 * b:100 * b + 100]
        assert np.isnan(o[first:]).all(), b
        ref = lay.oracle(q[100 * b:100 * b + first], b, kv[b] - 100 + first, kv[b] - 100)
        for t in range(first):
            assert np.linalg.norm(o[t] - ref[t]) <= REL * np.linalg.norm(ref[t]), (b, t)


def test_prefill_replays_in_a_graph():
    import torch
    new, kv = [60, 1, 30], [60, 99, 200]
    lay = Layer(shape("05b"), [200] * 3, 16, seed=34, poison=False)
    q = lay.queries(120)
    p = Prefill(lay, q, offsets(new), offsets(kv), n_kv=600)
    first = p().clone()
    p.ws.fill_(0x7B)
    assert torch.equal(p(), first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p()
    for new, kv in (([60, 1, 30], [60, 99, 200]), ([1, 1, 1], [1, 200, 7]), ([0, 120, 0], [0, 120, 50]),
                    ([40, 40, 40], [200, 200, 200])):
        p.q_off.copy_(ints(offsets(new)))
        p.kv_off.copy_(ints(offsets(kv)))
        p.o.fill_(3.0)
        graph.replay()
        got = p.o.clone()
        torch.cuda.synchronize()
        p.o.fill_(3.0)
        assert torch.equal(p(), got), new
        check_prefill(lay, q, offsets(new), kv, got)


@pytest.mark.parametrize("name,new,kv,order", [("8b", [130], [300], 1), ("1b", [200], [200], -1), ("05b", [90, 40], [90, 170], 0),
                                               ("05b", [20], [4500], 0)])
def test_prefill_rows_and_weights_of_any_magnitude(name, new, kv, order):
    """Latents from 2^-69 to 2^69 side by side (ascending, descending or mixed) and rows of W_UV from 2^-40
    to 2^40: every output to its own precision.  The non-positional queries are 0, so that the logits stay
    of ordinary size."""
    print(f"[paged] prefill {name} magnitudes {order}", flush=True)
    lay = Layer(shape(name), kv, 16, seed=50 + order, poison=False)
    rkv = lay.cfg.kv_rank
    for b, n in enumerate(kv):
        k = lay.rng.choice([-69, -40, -20, -9, 0, 0, 0, 9, 31, 69], n)
        k = np.sort(k)[::order] if order else k
        for p in range(n):
            lay.pool[lay.table[b, p // 16], p % 16, :rkv] *= 2.0 ** k[p]
    w = 2.0 ** lay.rng.integers(-40, 41, len(lay.Wuv))
    lay.Wuv = lay.Wuv * w[:, None]
    lay.upload()
    q, q_off = lay.queries(sum(new)), offsets(new)
    q[..., :lay.cfg.nope_dim] = 0
    got = Prefill(lay, q, q_off, offsets(kv))().double().cpu().numpy()
    w = np.repeat(w.reshape(lay.cfg.s_kv_groups, -1), lay.cfg.n_heads // lay.cfg.s_kv_groups, axis=0)
    for b, n in enumerate(kv):
        lo, hi = int(q_off[b]), int(q_off[b + 1])
        ref = lay.oracle(q[lo:hi], b, n, n - (hi - lo))
        for t in range(lo, hi):
            e = np.linalg.norm((got[t] - ref[t - lo]) / w) / np.linalg.norm(ref[t - lo] / w)
            assert e <= REL, (b, t, e)


def test_prefill_latents_too_large_are_nan_for_the_queries_that_see_them():
    lay = Layer(shape("05b"), [60], 16, seed=55)
    lay.pool[lay.table[0, 2], 3, 5] = 2.0 ** 73              # position 35
    lay.upload()
    q = lay.queries(60)
    got = Prefill(lay, q, offsets([60]), offsets([60]))().float().cpu().numpy()
    assert np.isnan(got[35:]).all()
    check_prefill(lay, q, offsets([35]), [35], Prefill(lay, q[:35], offsets([35]), offsets([35]))())
    ref = lay.oracle(q[:35], 0, 35, 0)
    for t in range(35):
        assert np.linalg.norm(got[t] - ref[t]) <= REL * np.linalg.norm(ref[t]), t


def test_prefill_without_cached_rows():
    """Sequences without rows (their queries see nothing), no cached rows at all."""
    lay = Layer(shape("8b"), [0, 0], 16, seed=35)
    q = lay.queries(70)
    for n_kv in (0, 300):
        p = Prefill(lay, q, offsets([69, 1]), offsets([0, 0]), n_kv=n_kv)
        assert not p().any()


def test_prefill_on_two_streams_with_their_own_workspaces():
    import torch
    new, kv = [200, 3], [1500, 700]
    lay = Layer(shape("1b"), kv, 64, seed=36)
    q = lay.queries(203)
    a = Prefill(lay, q, offsets(new), offsets(kv))
    b = Prefill(lay, q[::-1], offsets(new), offsets(kv), n_kv=4000)
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
    check_prefill(lay, q, offsets(new), kv, a.o)
    check_prefill(lay, q[::-1], offsets(new), kv, b.o)


# ---- append -----------------------------------------------------------------------------------
class Append:
    def __init__(self, cfg, pool, table, rows, q, q_off, start, inv, dtype, in_place=False):
        from paper_2607_27269_amd import _lib as L
        self.cfg = L.make_cfg(cfg.replace(batch=len(start), seq=1, dtype=dtype))
        self.pool, self.table, self.n = up(pool, dtype), ints(table), len(rows)
        self.rows, self.q = up(rows, dtype), up(q, dtype)
        self.q_out = self.q if in_place else up(np.full(q.shape, 7.0), dtype)
        self.off, self.start, self.inv = ints(q_off), ints(start), up(inv, "fp32")
        self.cache = L.PagedCache(self.pool.data_ptr(), self.table.data_ptr(), *self.pool.shape[:2],
                                  self.table.shape[1])

    def __call__(self, rows=True, q=True):
        import torch
        from paper_2607_27269_amd import _lib as L
        L.mla_recon_cache_append(self.cfg, self.cache, self.rows.data_ptr() if rows else None,
                                 self.q.data_ptr() if q else None, self.q_out.data_ptr() if q else None, self.n,
                                 self.off.data_ptr(), self.start.data_ptr(), self.inv.data_ptr(),
                                 torch.cuda.current_stream().cuda_stream)


def near(got, want, inputs, half, dtype):
    """One rounding of the result, and 1e-6 of |lo| + |hi| for the rotated pairs."""
    got = got.double().cpu().numpy()
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    pair = np.abs(inputs)
    spread = np.zeros_like(pair)
    w = pair[..., -2 * half:]
    both = w[..., :half] + w[..., half:]
    spread[..., -2 * half:] = np.concatenate([both, both], -1)
    assert (np.abs(got - want) <= step * np.abs(want) + 1e-6 * spread).all()


def append_case(name, dtype, new, start, ps, seed, Gr=1, table_cut=None):
    cfg = shape(name)
    if Gr > 1:
        cfg = cfg.replace(s_rope_groups=Gr, s_kv_groups=cfg.n_heads, n_kv_groups=cfg.n_heads)
    rng = np.random.default_rng(seed)
    rnd = (lambda *s: bf16(rng.standard_normal(s))) if dtype == "bf16" else (
        lambda *s: rng.standard_normal(s).astype(np.float32).astype(np.float64))
    W, n = cfg.kv_rank + Gr * cfg.rope_dim, sum(new)
    table, total = scatter(rng, [a + b for a, b in zip(new, start)], ps)
    pool = rnd(total, ps, W)
    rows, q = rnd(n, W), rnd(n, cfg.n_heads, cfg.nope_dim + cfg.rope_dim)
    inv = (1e4 ** (-np.arange(Gr * cfg.rope_dim // 2) / 16.0)).astype(np.float32).reshape(Gr, -1)
    return cfg, pool, table, rows, q, inv


@pytest.mark.parametrize("name,dtype,new,start,ps", [
    ("8b", "bf16", [1] * 17, list(range(0, 17)), 64), ("8b", "bf16", [100, 0, 33, 1], [0, 5, 31, 4000], 16),
    ("05b", "bf16", [65, 64, 63], [0, 100000, 7], 7), ("1b", "bf16", [5], [0], 1),
    ("tiny", "fp32", [50, 1, 2], [0, 250000, 77], 24), ("tiny", "bf16", [200], [13], 128),
    ("8b", "fp32", [3, 9], [1, 60], 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append(name, dtype, new, start, ps, in_place):
    print(f"[paged] append {name} {dtype} {new} at {start} page {ps}", flush=True)
    cfg, pool, table, rows, q, inv = append_case(name, dtype, new, start, ps, seed=40)
    a = Append(cfg, pool, table, rows, q, offsets(new), start, inv, dtype, in_place)
    a()
    want_pool, want_q = PO.append(pool, table, rows, q, offsets(new), start, inv, kv_rank=cfg.kv_rank,
                                  nope_dim=cfg.nope_dim)
    # the pool's inputs: the row that entered, or what was there (compared exactly)
    source = np.zeros_like(pool)
    off = offsets(new)
    touched = np.zeros(pool.shape[:2], dtype=bool)
    for b in range(len(new)):
        for i in range(off[b], off[b + 1]):
            p = start[b] + i - off[b]
            source[table[b, p // ps], p % ps] = rows[i]
            touched[table[b, p // ps], p % ps] = True
    near(a.pool[touched], want_pool[touched], source[touched], cfg.rope_dim // 2, dtype)
    got = a.pool.double().cpu().numpy()
    assert (got[~touched] == pool[~touched]).all()
    assert (got[touched][:, :cfg.kv_rank] == want_pool[touched][:, :cfg.kv_rank]).all()
    near(a.q_out, want_q, q, cfg.rope_dim // 2, dtype)
    assert (a.q_out[..., :cfg.nope_dim].double().cpu().numpy() == q[..., :cfg.nope_dim]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_positional_keys_of_groups(dtype):
    """G_r positional keys with frequencies of their own; head i takes group i / (H / G_r)'s."""
    new, start = [20, 3], [0, 50]
    cfg, pool, table, rows, q, inv = append_case("05b", dtype, new, start, 16, seed=41, Gr=7)
    a = Append(cfg, pool, table, rows, q, offsets(new), start, inv, dtype)
    a()
    want_pool, want_q = PO.append(pool, table, rows, q, offsets(new), start, inv, kv_rank=cfg.kv_rank,
                                  nope_dim=cfg.nope_dim)
    near(a.q_out, want_q, q, cfg.rope_dim // 2, dtype)
    got = a.pool.double().cpu().numpy()
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want_pool) + 1e-6 * 10   # |lo| + |hi| < 10
    assert (np.abs(got - want_pool) <= tol).all()


def test_append_parts_and_padding():
    """Rows alone, queries alone; packed rows of no sequence and rows without a place stay."""
    new, start = [30, 10], [0, 60]
    cfg, pool, table, rows, q, inv = append_case("05b", "bf16", new, start, 16, seed=42)
    pad = np.zeros((5,) + rows.shape[1:]), np.zeros((5,) + q.shape[1:])
    rows, q = np.concatenate([pad[0], rows, pad[0]]), np.concatenate([pad[1], q, pad[1]])
    table[0, 1] = -1                      # positions 16 .. 29 of sequence 0 have no page
    table = table[:, :4]                  # and 64 .. 69 of sequence 1 lie outside the table
    off = offsets(new, first=5)
    kw = dict(kv_rank=cfg.kv_rank, nope_dim=cfg.nope_dim)
    want_pool, want_q = PO.append(pool, table, rows, q, off, start, inv, **kw)
    a = Append(cfg, pool, table, rows, q, off, start, inv, "bf16")
    a(rows=False)
    assert (a.pool.double().cpu().numpy() == pool).all()
    near(a.q_out[5:45], want_q[5:45], q[5:45], cfg.rope_dim // 2, "bf16")
    assert (a.q_out[:5] == 7.0).all() and (a.q_out[45:] == 7.0).all()
    a.q_out.fill_(9.0)
    a(q=False)
    assert (a.q_out == 9.0).all()
    got = a.pool.double().cpu().numpy()
    changed = (got != pool).any(-1)
    assert changed.sum() == (want_pool != pool).any(-1).sum() == 16 + 4
    assert (np.abs(got - want_pool) <= 2.0 ** -8 * np.abs(want_pool) + 1e-6 * 10).all()


def test_append_replays_in_a_graph():
    """A captured call follows offsets, starts, tables and rows as they are at each replay."""
    import torch
    cfg, pool, table, rows, q, inv = append_case("1b", "bf16", [40, 40, 40], [40, 40, 40], 16, seed=43)
    a = Append(cfg, pool, table, rows[:60], q[:60], offsets([20, 20, 20]), [0, 1, 40], inv, "bf16")
    start_pool = a.pool.clone()
    a()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a()
    for new, start in (([20, 20, 20], [0, 1, 40]), ([60, 0, 0], [7, 0, 0]), ([1, 1, 1], [79, 0, 33]), ([0, 18, 42], [0, 62, 5])):
        a.off.copy_(ints(offsets(new)))
        a.start.copy_(ints(start))
        a.table.copy_(a.table.roll(1, 0))
        a.rows.copy_(a.rows.roll(1, 0))
        both = []
        for run in (graph.replay, a, graph.replay):
            a.pool.copy_(start_pool)
            a.q_out.fill_(3.0)
            run()
            both.append((a.pool.clone(), a.q_out.clone()))
            torch.cuda.synchronize()
        for x in both[1:]:
            assert torch.equal(x[0], both[0][0]) and torch.equal(x[1], both[0][1]), new
        want_pool, want_q = PO.append(pool, a.table.cpu().numpy(), a.rows.double().cpu().numpy(), q[:60],
                                      offsets(new), start, inv, kv_rank=cfg.kv_rank, nope_dim=cfg.nope_dim)
        got = both[0][0].double().cpu().numpy()
        assert (np.abs(got - want_pool) <= 2.0 ** -8 * np.abs(want_pool) + 1e-6 * 10).all(), new
        k = sum(new)
        near(both[0][1][:k], want_q[:k], q[:k], cfg.rope_dim // 2, "bf16")
        assert (both[0][1][k:] == 3.0).all()


# ---- page copies ------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,pages,page_bytes,n", [(1, 7, 16, 3), (3, 20, 4096 + 16, 9), (16, 9, 64 * 1152, 1),
                                                       (2, 2200, 240, 1000), (1, 3, 3 * 4096, 1)])
def test_copy_pages(layers, pages, page_bytes, n):
    import torch
    from paper_2607_27269_amd import _lib as L
    print(f"[paged] copy {n} of {pages} pages of {page_bytes} bytes in {layers} layers", flush=True)
    g = torch.Generator(device="cuda").manual_seed(n)
    gap = 48                                                  # bytes between the layers that stay as they are
    flat = torch.randint(0, 256, (layers, pages * page_bytes + gap), dtype=torch.uint8, device="cuda", generator=g)
    rng = np.random.default_rng(n)
    order = rng.permutation(pages)
    # sources may repeat (a page forked many times), destinations may not
    pairs = np.stack([order[rng.integers(0, max(1, pages - n), n)], order[pages - n:]], 1).astype(np.int32)
    want = flat.clone()
    view = want[:, :pages * page_bytes].view(layers, pages, page_bytes)
    view[:, pairs[:, 1].tolist()] = view[:, pairs[:, 0].tolist()].clone()
    import ctypes
    arr = np.ascontiguousarray(pairs)
    L.mla_recon_cache_copy_pages(flat.data_ptr(), layers, flat.stride(0), pages, page_bytes,
                                 arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), n,
                                 torch.cuda.current_stream().cuda_stream)
    arr[:] = 0                                                # read during the call only
    torch.cuda.synchronize()
    assert torch.equal(flat, want)


# ---- a run of them together ---------------------------------------------------------------------
def test_append_prefill_decode_fork_and_compact_together():
    """Prompts enter the cache and are attended to, tokens are decoded, one sequence is forked (its
    partial page copied) and both go their own ways, then the pool is compacted: the outputs follow
    the oracle on a cache kept in float64 on the host."""
    import ctypes

    import torch
    from paper_2607_27269_amd import _lib as L
    cfg, ps = shape("1b"), 16
    rng = np.random.default_rng(50)
    prompts = [37, 1, 64]
    W, H, dq = cfg.kv_rank + cfg.rope_dim, cfg.n_heads, cfg.nope_dim + cfg.rope_dim
    inv = (5e5 ** (-np.arange(cfg.rope_dim // 2) / 32.0)).astype(np.float32).reshape(1, -1)
    lay = Layer(cfg, [1], ps, seed=51)
    n_pages = 40
    free = list(rng.permutation(n_pages))
    lay.pool = np.full((n_pages, ps, W), np.nan)
    lay.table = np.full((4, 8), -1, dtype=np.int64)
    lay.upload()
    lens = [0, 0, 0, 0]
    kw = dict(kv_rank=cfg.kv_rank, nope_dim=cfg.nope_dim)

    def enter(seqs, new):
        """Append `new` tokens of each of `seqs` (all sequences are in the call's batch)."""
        counts = [0] * 4
        for b, n in zip(seqs, new):
            counts[b] = n
            for k in range(-(-lens[b] // ps), -(-(lens[b] + n) // ps)):
                lay.table[b, k] = free.pop()
        lay.d_table.copy_(ints(lay.table))
        n = sum(counts)
        rows, q = bf16(rng.standard_normal((n, W))), bf16(rng.standard_normal((n, H, dq)))
        a = Append(cfg, np.zeros((1, ps, W)), lay.table, rows, q, offsets(counts), lens, inv, "bf16")
        a.pool, a.table = lay.d_pool, lay.d_table
        a.cache = L.PagedCache(lay.d_pool.data_ptr(), lay.d_table.data_ptr(), n_pages, ps, 8)
        a()
        lay.pool, q = PO.append(lay.pool, lay.table, rows, q, offsets(counts), lens, inv, **kw)
        # the oracle's cache holds what the kernel wrote (rounded once), so that errors do not add up
        lay.pool = bf16(lay.pool)
        for b in range(4):
            lens[b] += counts[b]
        return bf16(q), a.q_out, counts

    q, d_q, counts = enter([0, 1, 2], prompts)
    p = Prefill(lay, q, offsets(counts), offsets(lens))
    p.q = d_q
    check_prefill(lay, q, offsets(counts), lens, p())

    def copy(pairs):
        arr = np.ascontiguousarray(pairs, dtype=np.int32)
        L.mla_recon_cache_copy_pages(lay.d_pool.data_ptr(), 1, 0, n_pages, ps * W * 2,
                                     arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), len(arr),
                                     torch.cuda.current_stream().cuda_stream)
        for s, t in pairs:
            lay.pool[t] = lay.pool[s]

    def decode(seqs):
        q, d_q, counts = enter(seqs, [1] * len(seqs))
        full = np.zeros((4, H, dq))
        full[seqs] = q
        now = [lens[b] if b in seqs else 0 for b in range(4)]
        d = Decode(lay, full, now, 8 * ps)
        d.q = torch.zeros_like(d.q)
        d.q[seqs] = d_q
        check_decode(lay, full, now, d())

    for _ in range(3):
        decode([0, 1, 2])
    # sequence 3 is forked from 0: whole pages shared, the partial one copied
    whole = lens[0] // ps
    lay.table[3, :whole] = lay.table[0, :whole]
    lay.table[3, whole] = free.pop()
    copy([(lay.table[0, whole], lay.table[3, whole])])
    lens[3] = lens[0]
    for _ in range(2):
        decode([0, 3])
    decode([0, 1, 2, 3])
    # compaction: the pages in use move to the front of the pool
    used = sorted({int(v) for v in lay.table.ravel() if v >= 0})
    holes = [v for v in range(len(used)) if v not in used]
    moves = dict(zip([v for v in used if v >= len(used)], holes))
    copy(list(moves.items()))
    lay.table = np.vectorize(lambda v: moves.get(int(v), int(v)))(lay.table)
    free[:] = list(range(len(used), n_pages))
    for v in range(len(used), n_pages):
        lay.pool[v] = np.nan
        lay.d_pool[v] = float("nan")
    decode([0, 1, 2, 3])
