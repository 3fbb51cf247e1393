"""GPU tests of the decoding whose rows' powers of two lie far apart (an e4m3 cache, and large groups' shared rows in
either format): rows of zeros, whose power is the smallest, beside rows of 2^60, 2^78 and 2^110, in tiles before and
after one another; and absorbed queries near both ends of their exponents.

The latents' part of the queries is 0 in the first tests and positional values are bf16 operands, so that logits
are exact up to fp32 and every row has a weight of its own, whatever its size: the output is the large rows' part of
the sum.  Tolerance: that of decoding (tests/test_gpu_paged.py)."""
import numpy as np
import pytest

from test_gpu_cache_e4m3 import DecodeE4m3, E4m3Layer
from test_gpu_decode_shared import FORMATS, Shared, make
from test_gpu_paged import bf16, check_decode, shape

pytestmark = pytest.mark.gpu


def change_rows(lay, fmt, b, n, change):
    """Give rows 0 .. n - 1 of sequence b the latents change(positions, latents [n, r_kv])."""
    rkv, p = lay.cfg.kv_rank, np.arange(n)
    at = lay.table[b, p // lay.ps], p % lay.ps
    rows = bf16(change(p[:, None], lay.pool[at][:, :rkv]))
    if fmt:
        lay.edit(*at, rows)
    else:
        lay.pool[(*at, slice(0, rkv))] = rows


def scale_tiles(lay, fmt, b, n, size, period, zeros_first):
    """Rows 0 .. n - 1 of sequence b in runs of `period` tiles of 32: zeros and rows of 2^size in turn."""
    change_rows(lay, fmt, b, n, lambda p, x: x * np.where((p // 32 // period % 2 == 0) == zeros_first, 0.0, 2.0 ** size))


def flat(lay, n):
    """Queries whose logits come from the positional values alone."""
    q = lay.queries(n)
    q[..., :lay.cfg.nope_dim] = 0
    return q


@pytest.mark.parametrize("zeros_first", [True, False])
@pytest.mark.parametrize("name,B,size", [("tiny", 40, 60), ("tiny", 40, 78), ("tiny", 40, 110), ("1b", 36, 78)])
def test_own_rows(name, B, size, zeros_first):
    """32 tiles of each sequence: two a wavefront, eight a workgroup, several workgroups a sequence; in runs of 1, 2, 4,
    8 and 16, so that the border is in a wavefront, between two, and between workgroups."""
    print(f"[extremes] own rows {name} 2^{size}, zeros first {zeros_first}", flush=True)
    lens = [1024 - 7 * (b % 3) for b in range(B)]
    lay = E4m3Layer(shape(name), lens, 64, seed=size, poison=False)
    for b, n in enumerate(lens):
        scale_tiles(lay, True, b, n, size, 1 << b % 5, zeros_first)
    lay.upload()
    q = flat(lay, B)
    check_decode(lay, q, lens, DecodeE4m3(lay, q, lens, 1024)())


@FORMATS
@pytest.mark.parametrize("zeros_first", [True, False])
@pytest.mark.parametrize("name,members,size", [("tiny", [130], 60), ("tiny", [130], 78), ("tiny", [130], 110),
                                               ("tiny", [4] * 33, 60), ("tiny", [4] * 33, 110), ("1b", [34], 78)])
def test_shared_rows(name, members, size, zeros_first, fmt):
    """A large group (rows made fp16 by the launch before) and small ones, four or five tiles a piece in the tiny
    layer's and a tile or two in the other's; the sequences' own rows are of the other kind than the first shared."""
    print(f"[extremes] shared rows {name} {len(members)} groups 2^{size}, zeros first {zeros_first}", flush=True)
    lay, lens, off = make(name, fmt, members, [1024] * len(members), [33, 1, 70], 64, seed=size)
    for g, b in enumerate(off[:-1]):
        scale_tiles(lay, fmt, b, 1024, size, 1 << g % 5 if len(members) > 1 else 3, zeros_first)
    lay.upload()
    q = flat(lay, len(lens))
    d = Shared(lay, q, lens, max(lens), off, [1024] * len(members), fmt)
    check_decode(lay, q, lens, d(), only=set(range(0, len(lens), 7)))


def opposite_rows(lay, fmt, b, n):
    """Rows of zeros but for two of one direction and its opposite: one of them takes a head's whole weight."""
    change_rows(lay, fmt, b, n, lambda p, x: x[5] * (1.0 * (p == 5) - (p == 40)))


@pytest.mark.parametrize("name", ["tiny", "05b", "8b"])
def test_large_absorbed_queries(name):
    """Up to about 2^118."""
    lens = [70, 64, 200]
    lay = E4m3Layer(shape(name), lens, 16, seed=31, poison=False)
    for b, n in enumerate(lens):
        opposite_rows(lay, True, b, n)
    lay.upload()
    q = lay.queries(3)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** 116)
    check_decode(lay, q, lens, DecodeE4m3(lay, q, lens, 200)())


@FORMATS
def test_large_absorbed_queries_over_shared_rows(fmt):
    lay, lens, off = make("tiny", fmt, [20], [96], [1, 20], 16, seed=32)
    opposite_rows(lay, fmt, 0, 96)
    lay.upload()
    q = lay.queries(20)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** 116)
    check_decode(lay, q, [96] * 20, Shared(lay, q, [96] * 20, 96, off, [96], fmt)())


@pytest.mark.parametrize("size", [60, 90, 98])
def test_small_absorbed_queries(size):
    """Rows of 2^size and queries of 2^-size: logits of an ordinary size."""
    lens = [161, 70]
    lay = E4m3Layer(shape("1b"), lens, 16, seed=33, poison=False)
    for b, n in enumerate(lens):
        change_rows(lay, True, b, n, lambda p, x: x * 2.0 ** size)
    lay.upload()
    q = lay.queries(2)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** -size)
    check_decode(lay, q, lens, DecodeE4m3(lay, q, lens, 161)())


@FORMATS
@pytest.mark.parametrize("size", [60, 98])
def test_small_absorbed_queries_over_shared_rows(size, fmt):
    lay, lens, off = make("1b", fmt, [18], [160], [5, 40], 16, seed=34)
    change_rows(lay, fmt, 0, 160, lambda p, x: x * 2.0 ** size)
    lay.upload()
    q = lay.queries(18)
    q[..., :lay.cfg.nope_dim] = bf16(q[..., :lay.cfg.nope_dim] * 2.0 ** -size)
    check_decode(lay, q, lens, Shared(lay, q, lens, max(lens), off, [160], fmt)())


def test_large_positional_logits_without_others():
    """Absorbed queries of zeros: positional logits of about 2^40, whose products are not exact in fp32."""
    lens = [70] * 6
    lay = E4m3Layer(shape("tiny"), lens, 16, seed=35, poison=False)
    q = np.zeros((6, 4, 96))
    for b, where in enumerate([0, 31, 32, 63, 64, 69]):
        q[b, :, 64] = 2.0 ** 20
        for p in range(70):
            pe = np.zeros(32)
            pe[0] = bf16(np.array([1.3 if p == where else 1.1]))[0] * 2.0 ** 20
            lay.edit(lay.table[b, p // 16], p % 16, positional=pe)
    lay.upload()
    check_decode(lay, q, lens, DecodeE4m3(lay, q, lens, 70)())
