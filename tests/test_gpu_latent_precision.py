"""How much precision decoding over either cache format may lose between its inputs and its output's rounding
(latent_decode_kernel; tests/test_gpu_paged_precision.py has the other kernels), and W_UK at an odd address.

Beside the rounding of the output to bf16, e0 = ||bf16(ref) - ref|| / ||ref|| (about 1.65e-3, computed here), in quadrature:

* weights: as two bf16 values off by 2^-17 at most; in fp16 (an e4m3 cache, or shared rows of large groups) by 2^-11,
  2.8e-4 rms, which adds 2.4e-5;
* absorbed queries in fp16, 2^-11 / 2.3 = 2.1e-4 rms of each times the logits' spread (below 1.5): 3.2e-4, which adds 3.1e-5
  (in bf16 eight times as much: sqrt(1.65^2 + 2.5^2) = 3.0e-3 in all; so those are tested with queries whose latents'
  part is 0);
* fp32 arithmetic: exponents of size 20 and sums of 1000 terms, below 2^-18 and 2^-14 in the worst case: 6.5e-5.

Together below e0 + 2e-4; a weight of one bf16 value, or bf16 queries where there should be fp16, give 2.2e-3 and more."""
import numpy as np
import pytest

from test_gpu_cache_e4m3 import DecodeE4m3, E4m3Layer
from test_gpu_decode_shared import FORMATS, Shared, make
from test_gpu_paged import Layer, shape
from test_gpu_paged_precision import check

pytestmark = pytest.mark.gpu

NAMES = pytest.mark.parametrize("name", ["tiny", "05b", "1b", "8b"])


def reference(lay, q, lens, only):
    return np.concatenate([lay.oracle(q[b:b + 1], b, lens[b], lens[b] - 1) for b in only])


@pytest.mark.parametrize("absorbed", [False, True])
@NAMES
def test_own_rows_e4m3(name, absorbed):
    lens = [1000, 64, 333, 17, 90, 200]
    lay = E4m3Layer(shape(name), lens, 16, seed=91)
    q = lay.queries(len(lens))
    if not absorbed:
        q[..., :lay.cfg.nope_dim] = 0
    check(f"own e4m3 {name}", DecodeE4m3(lay, q, lens, 1000)(), reference(lay, q, lens, range(len(lens))))


@NAMES
def test_own_rows_bf16(name):
    lens = [1000, 64, 333, 17, 90, 200]
    lay = Layer(shape(name), lens, 16, seed=92)
    q = lay.queries(len(lens))
    q[..., :lay.cfg.nope_dim] = 0
    check(f"own bf16 {name}", Shared(lay, q, lens, 1000, [0], [], False)(), reference(lay, q, lens, range(len(lens))))


@FORMATS
@NAMES
def test_shared_rows(name, fmt):
    """Groups of a few sequences: e4m3 rows, and bf16 ones without the latents' part."""
    lay, lens, off = make(name, fmt, [5, 4], [700, 330], [1, 40], 32, seed=93)
    q = lay.queries(len(lens))
    if not fmt:
        q[..., :lay.cfg.nope_dim] = 0
    got = Shared(lay, q, lens, max(lens), off, [700, 330], fmt)()
    check(f"shared {name}", got, reference(lay, q, lens, range(len(lens))))


@FORMATS
@NAMES
def test_shared_rows_of_large_groups(name, fmt):
    """Nearly all rows are shared: the own ones of a bf16 cache have bf16 queries."""
    lay, lens, off = make(name, fmt, [20], [640], [1, 2], 64, seed=94)
    q, only = lay.queries(len(lens)), [0, 3, 11, 19]
    got = Shared(lay, q, lens, max(lens), off, [640], fmt)()
    check(f"large group {name}", got[only], reference(lay, q, lens, only))


@pytest.mark.parametrize("members,fmt", [(None, True), ([20], False), ([20], True), ([5], False)],
                         ids=["own e4m3", "large bf16", "large e4m3", "small bf16"])
def test_an_unaligned_key_weight(members, fmt):
    import torch
    if members:
        lay, lens, off = make("1b", fmt, members, [96], [5, 40], 16, seed=95)
        q = lay.queries(len(lens))
        call = Shared(lay, q, lens, max(lens), off, [96], fmt)
    else:
        lens = [100, 7, 0, 65]
        lay = E4m3Layer(shape("1b"), lens, 16, seed=95)
        q = lay.queries(len(lens))
        call = DecodeE4m3(lay, q, lens, 100)
    want = call().clone()
    buf = torch.empty(lay.d_Wuk.numel() + 1, dtype=torch.bfloat16, device="cuda")
    buf[1:] = lay.d_Wuk.reshape(-1)
    lay.d_Wuk = call.Wuk = buf[1:]
    call.o.fill_(3.0)
    assert lay.d_Wuk.data_ptr() % 16 == 2 and torch.equal(call(), want)
