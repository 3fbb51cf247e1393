"""The paged cache as a program uses it (paper_2607_27269_amd/paged.py): prompts, decoding, forks,
rejected drafts, sequences that end, and compaction, over two layers, each step's outputs against the
float64 oracle on the rows that the sequences hold (tolerance: tests/test_gpu_paged.py)."""
import numpy as np
import pytest

from oracle import paged_oracle as PO
from paper_2607_27269_amd import configs
from test_gpu_paged import REL, bf16, up

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, name, n_pages, ps, seed):
        from paper_2607_27269_amd.paged import PagedLatentCache
        self.cfg = configs.get({"05b": 1, "1b": 2}[name])
        self.layers, self.rng = 2, np.random.default_rng(seed)
        self.cache = PagedLatentCache(self.cfg, self.layers, n_pages, ps)
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

    def step(self, seqs, counts, keep=True):
        c, rng = self.cfg, self.rng
        batch = self.cache.batch(seqs, counts)
        n, grown = sum(counts), {}
        for layer in range(self.layers):
            rows = bf16(rng.standard_normal((n, self.cache.width)))
            q = bf16(rng.standard_normal((n, c.n_heads, c.nope_dim + c.rope_dim)))
            d_q = batch.append(layer, up(rows), up(q), up(self.inv, "fp32"))
            got = batch.attend(layer, d_q, *self.d_W[layer]).double().cpu().numpy()
            at = 0
            for s, k in zip(seqs, counts):
                first = len(self.rows[s][layer])
                new = rows[at:at + k].copy()
                turned = q[at:at + k].copy()
                for t in range(k):
                    new[t, c.kv_rank:] = PO.rotate(new[t, c.kv_rank:], first + t, self.inv[0])
                    turned[t, :, c.nope_dim:] = PO.rotate(turned[t, :, c.nope_dim:], first + t, self.inv[0])
                held = np.concatenate([self.rows[s][layer], bf16(new)])
                grown[s, layer] = held
                ref = PO.attend(bf16(turned), held, *self.W[layer], nope_dim=c.nope_dim,
                                scale=float(np.float32(c.softmax_scale)), n_groups=c.s_kv_groups, first=first)
                for t in range(k):
                    e = np.linalg.norm(got[at + t] - ref[t]) / np.linalg.norm(ref[t])
                    assert e <= REL, (s, layer, t, first, e)
                at += k
        if not keep:
            batch.abandon()
            return
        batch.commit()
        for (s, layer), held in grown.items():
            self.rows[s][layer] = held
        for s in seqs:
            assert self.cache.length(s) == len(self.rows[s][0])

    def truncate(self, s, n):
        self.cache.truncate(s, n)
        self.rows[s] = [x[:n] for x in self.rows[s]]


@pytest.mark.parametrize("name,ps", [("05b", 16), ("1b", 7)])
def test_serving_run(name, ps):
    print(f"[paged] serving {name}, pages of {ps}", flush=True)
    m = Model(name, n_pages=60, ps=ps, seed=ps)
    a, b = m.add(), m.add()
    m.step([a, b], [37, 1])
    m.step([a, b], [1, 1])
    c = m.fork(a)                            # shares a's pages, the last of them partly filled
    d = m.fork(a)
    m.step([c, a], [1, 1])                   # both grow: one of them gets a copy
    m.step([d, b], [5, 9])                   # a draft of five tokens ...
    m.truncate(d, 38 + 2)                    # ... of which two stay
    m.step([a, b, c, d], [1, 1, 1, 1])
    m.step([b], [20], keep=False)            # a step that is given up
    m.cache.free(a)
    assert m.cache.compact() > 0 or m.cache.alloc.free_pages
    m.step([d, c, b], [1, 1, 1])
    m.step([b, c], [3, 30])


def test_refusals():
    import torch
    from paper_2607_27269_amd.paged import OutOfPages
    m = Model("05b", n_pages=4, ps=16, seed=1)
    s = m.add()
    with pytest.raises(ValueError):
        m.cache.batch([s], [0])
    with pytest.raises(ValueError):
        m.cache.batch([], [])
    with pytest.raises(OutOfPages):
        m.cache.batch([s], [65])
    batch = m.cache.batch([s], [2])
    with pytest.raises(RuntimeError):
        m.cache.batch([s], [1])              # one batch at a time
    with pytest.raises(RuntimeError):
        m.cache.fork(s)
    c = m.cfg
    rows = torch.zeros(2, m.cache.width, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, c.n_heads, c.nope_dim + c.rope_dim, dtype=torch.bfloat16, device="cuda")
    inv = up(m.inv, "fp32")
    for bad in ((rows.float(), q, inv), (rows[:1], q, inv), (rows.cpu(), q, inv), (rows, q[:, 1:], inv),
                (rows, q.transpose(0, 1).contiguous().transpose(0, 1), inv), (rows, q, inv.double())):
        with pytest.raises(ValueError):
            batch.append(0, *bad)
    with pytest.raises(ValueError):
        batch.attend(0, q, m.d_W[0][1][:1], m.d_W[0][1])
    batch.append(0, rows, q, inv)
    batch.commit()
    with pytest.raises(RuntimeError):
        batch.commit()
    assert m.cache.length(s) == 2
