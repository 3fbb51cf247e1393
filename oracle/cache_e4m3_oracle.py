"""Plain CPU reference of the eight-bit cache format: rows of latents in e4m3 times a power of two for
the row, positional values in bf16; a page is its rows, then their powers (fp32), padded to 16 bytes.

TEST INFRASTRUCTURE ONLY: only the test-suite may import it.  It shares no code with the GPU path and
imports nothing from it.
"""
from __future__ import annotations

import numpy as np

# the values of codes 0 .. 126 (e4m3: bias 7, the smallest exponent for subnormals, 127 is NaN)
MAGNITUDES = np.array([f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10) for e in range(16) for f in range(8)][:127])


def value(codes):
    """What e4m3 codes stand for."""
    codes = np.asarray(codes, dtype=np.int64)
    m = np.append(MAGNITUDES, np.nan)[codes & 127]
    return np.where(codes & 128, -m, m)


def code(x):
    """The e4m3 codes nearest to x (|x| <= 448), halves to the even code; NaN where x is not finite."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 126)
    below, above = a - MAGNITUDES[hi - 1], MAGNITUDES[hi] - a
    k = np.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)
    return np.where(fine, k + 128 * np.signbit(x), 127).astype(np.uint8)


def exponent(latents):
    """The exponents of the rows' powers: the least e in [-80, 120] with max |x| <= 448 2^e."""
    a = np.where(np.isfinite(latents), np.abs(latents), 0.0).max(-1)
    e = np.full(a.shape, -80)
    for k in range(-80, 120):
        e = np.where(a > 448 * 2.0 ** k, k + 1, e)
    return e


def quantise(latents):
    """(codes, powers) of rows of latents."""
    power = 2.0 ** exponent(latents)
    with np.errstate(invalid="ignore"):
        return code(latents / power[..., None]), power


def stored(rows, kv_rank):
    """Rows [..., width] as the cache gives them back."""
    codes, power = quantise(rows[..., :kv_rank])
    return np.concatenate([value(codes) * power[..., None], rows[..., kv_rank:]], axis=-1)


def pack(codes, positional, power):
    """Pages [n, bytes] uint8 of codes [n, page, kv_rank], bf16 positional values and powers."""
    n, page, _ = codes.shape
    pe = (np.ascontiguousarray(positional, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16).view(np.uint8)
    rows = np.concatenate([codes, pe], axis=-1).reshape(n, -1)
    tail = np.ascontiguousarray(power, dtype=np.float32).view(np.uint8).reshape(n, -1)
    out = np.concatenate([rows, tail], axis=1)
    return np.pad(out, ((0, 0), (0, -out.shape[1] % 16)))


def unpack(pages, page, kv_rank, pe):
    """(codes, positional values, powers) of pages [n, bytes]."""
    n, size = len(pages), kv_rank + 2 * pe
    rows = pages[:, :page * size].reshape(n, page, size)
    bits = np.ascontiguousarray(rows[..., kv_rank:]).view(np.uint16).astype(np.uint32) << 16
    power = np.ascontiguousarray(pages[:, page * size:page * (size + 4)]).view(np.float32)
    return rows[..., :kv_rank], bits.view(np.float32).astype(np.float64), power.astype(np.float64)
