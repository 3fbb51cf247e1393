"""GPU tests of the packed prefill where its 16-bit operands' scales span their whole range: rows of latents
near 2^-66 and near 2^66 in one sequence, in either order, with the keys in one part and in several.

The latents' part of the keys gets queries of 0, so that the logits come from the positional keys alone:
their bf16 operands are exact, and the outputs carry the roundings named in tests/test_gpu_paged.py (bound
REL there)."""
import numpy as np
import pytest

from test_gpu_paged import REL, Layer, Prefill, bf16, offsets, shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spread", [0.0, 8.0])
@pytest.mark.parametrize("large", [[0], [-1], [37], [0, -1]])
@pytest.mark.parametrize("name,n", [("05b", 65), ("1b", 200), ("05b", 1500), ("1b", 2900)])
def test_prefill_weights_of_rows_of_the_smallest_and_the_largest_scale(name, n, large, spread):
    """Every row counts in the softmax with its own weight, whatever its latents' scale: the output is
    the large rows' values times their share, which the small rows' number decides.  spread: the
    standard deviation of the logits is about spread / 2 (0: all alike)."""
    print(f"[paged] prefill {name} {n} rows, large at {large}, spread {spread}", flush=True)
    lay = Layer(shape(name), [n], 16, seed=n, poison=False)
    rkv = lay.cfg.kv_rank
    k = np.full(n, -66)
    k[large] = 66
    for p in range(n):
        lay.pool[lay.table[0, p // 16], p % 16, :rkv] *= 2.0 ** k[p]
    lay.upload()
    q = bf16(lay.queries(2) * spread)
    q[..., :lay.cfg.nope_dim] = 0
    if spread:   # the logits do spread
        s = lay.pool[lay.table[0, :n // 16]].reshape(-1, lay.W)[:, rkv:] @ q[0, :, lay.cfg.nope_dim:].T * lay.cfg.softmax_scale
        assert (s.max(0) - s.min(0)).min() > 10
    got = Prefill(lay, q, offsets([2]), offsets([n]))().double().cpu().numpy()
    ref = lay.oracle(q, 0, n, n - 2)
    for t in range(2):
        for h in range(lay.cfg.n_heads):
            e = np.linalg.norm(got[t, h] - ref[t, h]) / np.linalg.norm(ref[t, h])
            assert e <= REL, (t, h, e)
