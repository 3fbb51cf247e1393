"""The packed prefill at the largest number of cached rows (1048576): key and value arrays, their products and
the copies past 2^31 bytes.  One page of 16384 rows stands in every place of the table, so that the
attention of a query over all rows is that over the page's rows (each as often as the others; the last page is seen up
to the query's own row)."""
import numpy as np
import pytest

from test_gpu_paged import REL, Layer, Prefill, shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["8b", "tiny"])
def test_prefill_of_the_most_rows(name):
    ps, most = 16384, 1 << 20
    print(f"[paged] prefill {name} over {most} rows", flush=True)
    lay = Layer(shape(name), [ps], ps, seed=81, spare=0)
    lay.table = np.zeros((2, most // ps), dtype=np.int64)
    lay.upload()
    kv = np.array([0, 5000, most])           # a short sequence, then the rest
    q = lay.queries(3)
    got = Prefill(lay, q, np.array([0, 1, 3]), kv)().double().cpu().numpy()
    n = most - 5000
    ref = [lay.oracle(q[:1], 0, 5000, 4999)[0]]
    rows = lay.pool[0]
    c = lay.cfg
    for t, seen in ((1, n - 1), (2, n)):
        weight = np.full(ps, seen // ps, dtype=np.float64)
        weight[:seen % ps] += 1
        o = np.zeros((c.n_heads, c.head_dim))
        for h in range(c.n_heads):
            g = h // (c.n_heads // c.s_kv_groups)
            k = np.concatenate([rows[:, :c.kv_rank] @ lay.Wuk[g * c.nope_dim:(g + 1) * c.nope_dim].T, rows[:, c.kv_rank:]], 1)
            s = k @ q[t, h] * float(np.float32(c.softmax_scale))
            p = np.exp(s - s.max()) * weight
            o[h] = p / p.sum() @ rows[:, :c.kv_rank] @ lay.Wuv[g * c.head_dim:(g + 1) * c.head_dim].T
        ref.append(o)
    for t in range(3):
        e = np.linalg.norm(got[t] - ref[t]) / np.linalg.norm(ref[t])
        print(f"[paged] token {t}: {e:.2e}", flush=True)
        assert e <= REL, (t, e)
