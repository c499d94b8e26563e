"""Plain definition of the 8-bit caches: codes, scales, layouts (numpy, float64).

A row x (one token, one KV head, K or V) has one power-of-two scale:
  E = the least integer >= -100 with max |x_d| <= c 2^E   (c = 448 for e4m3, 127 for int8),
  code_d = x_d 2^-E to the nearest code, ties to the even one;  value_d = code_d 2^E;  scale byte E + 127;
a row with a NaN, an infinity or a magnitude >= 2^127 has byte 255 and codes 0, which stand for NaN.

This is not in the paper (it keeps its caches in bf16): parity unpinned; pinned by the number formats' own definitions
in tests/test_oracle_q8.py.
"""
import numpy as np

from .cache_model import PAGE, ring_slot, split_heads

E4M3, I8 = "e4m3", "i8"


def code_values(fmt):
    """Value of each of the 256 codes."""
    c = np.arange(256)
    if fmt == I8:
        return np.where(c < 128, c, c - 256).astype(np.float64)
    sign, exp, frac = c >> 7, (c >> 3) & 15, c & 7
    mag = np.where(exp == 0, frac / 8.0 * 2.0 ** -6, (1 + frac / 8.0) * 2.0 ** (exp - 7.0))
    mag = np.where((exp == 15) & (frac == 7), np.nan, mag)
    return np.where(sign == 1, -mag, mag)


def largest(fmt):
    return 448.0 if fmt == E4M3 else 127.0


def quantise(x, fmt):
    """Codes uint8 [..., D] and scale bytes uint8 [...] of rows x [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    amax = np.abs(x).max(axis=-1)
    bad = ~(amax < 2.0 ** 127)
    e = np.frexp(np.where(bad | (amax == 0), 1.0, amax))[1] - (9 if fmt == E4M3 else 7)
    e = np.where(np.where(bad, 0.0, amax) > largest(fmt) * np.exp2(e), e + 1, e)
    e = np.where(amax == 0, -100, np.maximum(e, -100))
    y = np.where(bad[..., None], 0.0, x) * np.exp2(-e.astype(np.float64))[..., None]
    if fmt == I8:
        codes = np.rint(y).astype(np.int64) & 255
    else:
        table = code_values(E4M3)[:127]  # ascending; neighbours differ in the last bit
        hi = np.clip(np.searchsorted(table, np.abs(y)), 1, 126)
        below, above = np.abs(y) - table[hi - 1], table[hi] - np.abs(y)
        pick = np.where(below < above, hi - 1, np.where(below > above, hi, np.where(hi % 2 == 0, hi, hi - 1)))
        codes = pick | np.where(np.signbit(y), 128, 0)
    return codes.astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, fmt):
    """The values that codes [..., D] with scale bytes [...] stand for."""
    with np.errstate(invalid="ignore"):
        scale = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
        return code_values(fmt)[codes] * scale[..., None]


def stored(x, fmt):
    """What rows x read back as."""
    return values(*quantise(x, fmt), fmt)


def v_rows(unit):
    """V codes [..., D/4, 4, 4, 4] (dim // 4, row // 4, dim % 4, row % 4) -> [..., 16, D]."""
    n = unit.ndim - 4
    rows = unit.transpose(*range(n), n + 1, n + 3, n, n + 2)
    return rows.reshape(*unit.shape[:n], PAGE, unit.shape[n] * 4)


def v_unit(rows):
    """The inverse of v_rows."""
    n, d = rows.ndim - 2, rows.shape[-1]
    x = rows.reshape(*rows.shape[:n], 4, 4, d // 4, 4)
    return x.transpose(*range(n), n + 2, n, n + 3, n + 1)


def append(full, ring, table, k, v, labels, starts, counts, n_sink, window, fmt):
    """Appends counts[b] tokens of k, v [B][n][Hkv][D] at positions starts[b] on, one after the other, to caches given
    as (K codes, V codes, scale bytes), in place."""
    ret, strm = split_heads(labels)
    kc, ks = quantise(k, fmt)
    vc, vs = quantise(v, fmt)
    for b, (start, count) in enumerate(zip(starts, counts)):
        if not 0 <= start < 1 << 30:
            continue
        for t in range(count):
            p = start + t
            for rank, g in enumerate(ret):
                if p // PAGE >= table.shape[1] or not 0 <= table[b, p // PAGE] < full[0].shape[0]:
                    continue
                _put(full, (table[b, p // PAGE], rank), p % PAGE, kc[b, t, g], vc[b, t, g], ks[b, t, g], vs[b, t, g])
            for rank, g in enumerate(strm):
                c = ring_slot(p, n_sink, window)
                _put(ring, (b, rank, c // PAGE), c % PAGE, kc[b, t, g], vc[b, t, g], ks[b, t, g], vs[b, t, g])


def _put(cache, unit, row, kc, vc, ks, vs):
    k, v, s = cache
    k[unit][row] = kc
    d = np.arange(len(vc))
    v[unit][d // 4, row // 4, d % 4, row % 4] = vc
    s[unit][row] = ks, vs
