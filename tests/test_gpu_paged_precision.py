"""How much precision the paged attention may lose between its inputs and its output's rounding.

The latents' part of the queries is 0, so the logits come from the positional keys alone, whose bf16 operands
are exact (so are the absorbed queries and the expanded keys, which are multiplied by 0).  What is left is
the rounding of the output to bf16, e0 = ||bf16(ref) - ref|| / ||ref|| (about 1.6e-3, computed here), and:

* decoding: probabilities and weighted latents as the sum of two bf16 values, off by at most 2^-17 each, and
  fp32 arithmetic (exponents of size 20 and sums of 1000 terms: below 2^-18 and 2^-14 in the worst case):
  e <= e0 + 2e-4.  A probability of one bf16 value (rms 2^-8 / 2.5 = 1.5e-3) gives sqrt(1.6^2 + 1.5^2) = 2.2e-3.
* prefill: values and probabilities rounded to fp16, at most 2^-11 / sqrt(3) = 2.8e-4 of the norm each,
  4e-4 together; added to e0 in quadrature 5e-5, and fp32 arithmetic: e <= e0 + 2e-4.  bf16 values or probabilities
  give 2.2e-3, both 2.7e-3.
"""
import numpy as np
import pytest

from test_gpu_paged import Decode, Layer, Prefill, bf16, offsets, shape

pytestmark = pytest.mark.gpu

MORE = 2e-4


def check(name, got, ref):
    got, norm = got.double().cpu().numpy(), np.linalg.norm(ref)
    e0, e = np.linalg.norm(bf16(ref) - ref) / norm, np.linalg.norm(got - ref) / norm
    print(f"[precision] {name}: rounding {e0:.3e}, error {e:.3e}", flush=True)
    assert e <= e0 + MORE


@pytest.mark.parametrize("name", ["tiny", "05b", "1b", "8b"])
def test_decode(name):
    lens = [1000, 64, 333, 17, 90, 200]
    lay = Layer(shape(name), lens, 16, seed=71)
    q = lay.queries(len(lens))
    q[..., :lay.cfg.nope_dim] = 0
    ref = np.concatenate([lay.oracle(q[b:b + 1], b, n, n - 1) for b, n in enumerate(lens)])
    check("decode " + name, Decode(lay, q, lens, 1000)(), ref)


@pytest.mark.parametrize("name,new,kv", [("tiny", [40, 3], [200, 1000]), ("05b", [70, 3], [70, 500]), ("1b", [40, 3], [300, 1000]),
                                         ("8b", [40, 3], [40, 600]), ("8b", [4], [4000])])
def test_prefill(name, new, kv):
    lay = Layer(shape(name), kv, 16, seed=72)
    q, q_off = lay.queries(sum(new)), offsets(new)
    q[..., :lay.cfg.nope_dim] = 0
    ref = np.concatenate([lay.oracle(q[q_off[b]:q_off[b + 1]], b, n, n - new[b]) for b, n in enumerate(kv)])
    check("prefill " + name, Prefill(lay, q, q_off, offsets(kv))(), ref)
