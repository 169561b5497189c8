"""The microscaled formats from their definition, in numpy and 64 bits (test infrastructure: shares no
code with the library).  Every element is found by search among all elements of its type."""
from __future__ import annotations

import collections

import numpy as np

Format = collections.namedtuple("Format", "levels emax")
_SMALL = [i * 2.0 ** -9 for i in range(8)]
FORMATS = {
    "int8": Format([float(q) for q in range(128)], 6),
    "e4m3": Format((_SMALL + [(8 + i) * 2.0 ** (e - 3) for e in range(-6, 9) for i in range(8)])[:127], 8),
    "e2m1": Format([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], 2),
}


def _blocks(x):
    rows, cols = x.shape
    return np.pad(x, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)


def _scales(v, fmt):
    """Shared bytes: the smallest power of two for which the largest magnitude does not round past the
    largest element (halfway rounds past it: the element beyond is even)."""
    lv, emax = FORMATS[fmt]
    last = lv[-1] + (lv[-1] - lv[-2]) / 2
    a = np.abs(v).max(2)
    s = np.zeros(a.shape, dtype=np.int64)
    ok = np.isfinite(a) & (a > 0)
    k = np.floor(np.log2(np.where(ok, a, 1.0))).astype(np.int64)
    k += np.ldexp(1.0, k + 1) <= np.where(ok, a, 1.0)           # log2 may be off at a power of two
    k -= np.ldexp(1.0, k) > np.where(ok, a, 1.0)
    k += np.where(ok, a, 1.0) / np.ldexp(1.0, k - emax) >= last
    s[ok] = np.clip(k - emax + 127, 0, 254)[ok]
    s[~np.isfinite(a)] = 255
    return s


def _indices(v, s, fmt):
    """Index of the nearest level for every magnitude, ties to the even index."""
    lv = np.array(FORMATS[fmt].levels)
    a = np.where((s == 255)[..., None], 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)) * np.ldexp(1.0, 127 - s)[..., None])
    mid = (lv[1:] + lv[:-1]) / 2
    i = np.searchsorted(mid, a, side="left")                    # a tie lands on the lower level
    tie = (i < len(mid)) & (a == mid[np.minimum(i, len(mid) - 1)])
    return i + (tie & (i % 2 == 1))


def pack(x, fmt):
    """(codes, scales) of a [rows, cols] float64 array in the documented layout."""
    x = np.asarray(x, dtype=np.float64)
    v = _blocks(x)
    s = _scales(v, fmt)
    i = _indices(v, s, fmt)
    neg = np.signbit(v) & (s != 255)[..., None]
    if fmt == "int8":
        codes = np.where(neg, -i, i).astype(np.int8).view(np.uint8)
    else:
        codes = (i | np.where(neg, 128 if fmt == "e4m3" else 8, 0)).astype(np.uint8)
    codes = codes.reshape(len(x), -1)
    if fmt == "e2m1":
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return codes, np.pad(s.astype(np.uint8), ((0, 0), (0, -s.shape[1] % 4)))


def unpack(codes, scales, cols, fmt):
    """What codes and scales stand for, [rows, cols] float64."""
    lv = np.array(FORMATS[fmt].levels)
    if fmt == "e2m1":
        codes = np.stack([codes & 15, codes >> 4], -1).reshape(len(codes), -1)
        el = np.where(codes & 8, -lv[codes & 7], lv[codes & 7])
    elif fmt == "e4m3":
        el = np.where(codes & 128, -1.0, 1.0) * lv[np.minimum(codes & 127, 126)]
    else:
        el = codes.view(np.int8).astype(np.float64)
    s = np.repeat(scales, 32, axis=1)[:, :cols].astype(np.int64)
    return np.where(s == 255, np.nan, el[:, :cols] * np.ldexp(1.0, s - 127))


def values(x, fmt):
    """What the codes of x stand for."""
    return unpack(*pack(x, fmt), np.asarray(x).shape[1], fmt)


def product_bound(a, w):
    """K 2^-24 sum |a w|: how far a float sum of K exact products, in any order, can be off."""
    return a.shape[1] * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)
