"""The paged cache in both formats as a program uses it (paper_2607_27269_amd/paged.py), with steps that share the
pages of forks: each step's outputs against the float64 oracle on the rows that the sequences hold, in
eight bits as the oracle quantises them (tolerance: tests/test_gpu_paged.py)."""
import numpy as np
import pytest

from oracle import cache_e4m3_oracle as EO
from oracle import paged_oracle as PO
from paper_2607_27269_amd import configs, paged
from test_gpu_paged import REL, bf16, up

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, name, fmt, n_pages, ps, seed):
        from paper_2607_27269_amd.paged import PagedLatentCache
        self.cfg, self.fmt = configs.get({"05b": 1, "1b": 2, "8b": 3}[name]), fmt
        self.layers, self.rng = 2, np.random.default_rng(seed)
        self.cache = PagedLatentCache(self.cfg, self.layers, n_pages, ps, format=fmt)
        c = self.cfg
        self.inv = (1e4 ** (-np.arange(c.rope_dim // 2) / (c.rope_dim // 2))).astype(np.float32).reshape(1, -1)
        self.W = [(bf16(self.rng.standard_normal((c.s_kv_groups * c.nope_dim, c.kv_rank)) / np.sqrt(c.kv_rank)),
                   bf16(self.rng.standard_normal((c.s_kv_groups * c.head_dim, c.kv_rank)) / np.sqrt(c.kv_rank)))
                  for _ in range(self.layers)]
        self.d_W = [(up(a), up(b)) for a, b in self.W]
        self.rows = {}                       # sequence -> per layer the cached rows

    def add(self):
        s = self.cache.add()
        self.rows[s] = [np.zeros((0, self.cache.width)) for _ in range(self.layers)]
        return s

    def fork(self, s):
        t = self.cache.fork(s)
        self.rows[t] = [x.copy() for x in self.rows[s]]
        return t

    def step(self, seqs, counts, share=False, check=True):
        c, rng = self.cfg, self.rng
        batch = self.cache.batch(seqs, counts, share=share)
        n = sum(counts)
        for layer in range(self.layers):
            rows = bf16(rng.standard_normal((n, self.cache.width)))
            q = bf16(rng.standard_normal((n, c.n_heads, c.nope_dim + c.rope_dim)))
            d_q = batch.append(layer, up(rows), up(q), up(self.inv, "fp32"))
            got = batch.attend(layer, d_q, *self.d_W[layer]).double().cpu().numpy()
            turned_q, at = d_q.double().cpu().numpy(), 0
            for s, k in zip(seqs, counts):
                first = len(self.rows[s][layer])
                new = rows[at:at + k].copy()
                for t in range(k):
                    new[t, c.kv_rank:] = PO.rotate(new[t, c.kv_rank:], first + t, self.inv[0])
                    turn = PO.rotate(q[at + t, :, c.nope_dim:], first + t, self.inv[0])
                    assert np.abs(turned_q[at + t, :, c.nope_dim:] - turn).max() <= 2.0 ** -8 * np.abs(turn).max() + 1e-4
                new = bf16(new)
                if self.fmt == "e4m3":
                    new = EO.stored(new, c.kv_rank)
                held = self.rows[s][layer] = np.concatenate([self.rows[s][layer], new])
                if check:
                    ref = PO.attend(turned_q[at:at + k], held, *self.W[layer], nope_dim=c.nope_dim,
                                    scale=float(np.float32(c.softmax_scale)), n_groups=c.s_kv_groups, first=first)
                    for t in range(k):
                        e = np.linalg.norm(got[at + t] - ref[t]) / np.linalg.norm(ref[t])
                        assert e <= REL, (s, layer, t, first, e)
                at += k
        batch.commit()
        return batch


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("name,ps", [("05b", 16), ("1b", 7), ("8b", 32)])
def test_samples_of_prompts(name, ps, fmt, monkeypatch):
    """Two prompts, samples of each side by side in steps that share their pages, a sequence of its own
    between them; sequences that end, compaction, drafts of several tokens."""
    print(f"[serving] {name} {fmt}, pages of {ps}", flush=True)
    monkeypatch.setattr(paged, "worth_sharing", lambda groups, cfg, format: groups)   # (short prompts)
    m = Model(name, fmt, n_pages=150, ps=ps, seed=ps)
    a, alone, b = m.add(), m.add(), m.add()
    m.step([a, alone, b], [200, 3, 150])
    more = [m.fork(a) for _ in range(4)] + [m.fork(b)]
    order = [a] + more[:4] + [alone, b, more[4]]
    for k in range(3):
        step = m.step(order, [1] * 8, share=True)
        assert [g[:2] for g in step.groups] == [(0, 5), (6, 2)] and step.n_groups == 3
    m.cache.free(a)
    m.cache.compact()
    assert [g[:2] for g in m.step(order[1:], [1] * 7, share=True).groups] == [(0, 4), (5, 2)]
    m.step(order[1:], [1, 4, 1, 1, 2, 1, 1], share=True)      # not single tokens: a prefill
    m.step(order[1:], [1] * 7)                                # not shared
    assert m.step(order[1:], [1] * 7, share=True).groups


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_read_gives_back_what_is_stored(fmt):
    m = Model("1b", fmt, n_pages=40, ps=16, seed=5)
    a = m.add()
    m.step([a], [70], check=False)
    m.step([a], [1], check=False)
    b = m.fork(a)
    m.step([b], [5], check=False)
    for s in (a, b):
        for layer in range(2):
            held = m.rows[s][layer]
            got = m.cache.read(layer, s).double().cpu().numpy()
            assert np.array_equal(got[:, :512], held[:, :512])
            assert np.abs(got[:, 512:] - held[:, 512:]).max() <= 2.0 ** -7 * np.abs(held[:, 512:]).max()
            part = m.cache.read(layer, s, 30, 33).double().cpu().numpy()
            assert np.array_equal(part, got[30:63])
    assert m.cache.read(0, a, 71).shape == (0, 576)
    for bad in ((-1, 3), (0, 72), (70, 2), (0, -1)):
        with pytest.raises(ValueError):
            m.cache.read(0, a, *bad)


def test_a_cache_is_moved_into_eight_bits():
    """Rows read from a bf16 cache and appended to one in eight bits: positions come rotated, so they
    are appended at angle 0 and read back as the oracle stores them."""
    import torch
    m = Model("05b", "bf16", n_pages=20, ps=16, seed=6)
    a = m.add()
    m.step([a], [50], check=False)
    small = Model("05b", "e4m3", n_pages=20, ps=16, seed=7)
    s = small.add()
    batch = small.cache.batch([s], [50])
    q = torch.zeros(50, 14, 96, dtype=torch.bfloat16, device="cuda")
    still = torch.zeros(1, 16, device="cuda")
    for layer in range(2):
        batch.append(layer, m.cache.read(layer, a), q, still)
    batch.commit()
    for layer in range(2):
        want = EO.stored(m.cache.read(layer, a).double().cpu().numpy(), 256)
        assert np.array_equal(small.cache.read(layer, s).double().cpu().numpy(), want)
