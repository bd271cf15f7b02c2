"""Plain float64 forms of a cache held in 8 bits (test infrastructure).

  codes    the 127 sizes that e4m3 has, listed from its definition; a number's code is the
           nearest of them, of two equally near ones the even code.
  scale    the least power of two, at least 2^-126, that takes the largest finite size to at
           most 448; byte b is 2^(b - 127), 0 is left to blocks of zeros.
  order    values: token 4 g + t, element 64 x + 4 c + d at [x][g][c][d][t].
  fill     new rows into blocks, with what happens to the tokens a block held before.

Written out element by element where that is quick enough, with no bit tricks.
"""
from __future__ import annotations


import numpy as np

from .attention import _ints, to_f64

# code 8 e + m is m 2^-9 for e = 0, else (8 + m) 2^(e - 10); code 127 is NaN
SIZES = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


def encode(x) -> np.ndarray:
    """Bytes of the codes nearest to x (|x| <= 448 where finite)."""
    x = np.asarray(x, dtype=np.float64)
    size = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(SIZES, size), 1, 126)
    lo = hi - 1
    below, above = size - SIZES[lo], SIZES[hi] - size
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = code + 128 * np.signbit(x)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def decode(codes) -> np.ndarray:
    c = np.asarray(codes).astype(np.int64)
    size = np.append(SIZES, np.nan)[c % 128]
    return np.where(c >= 128, -size, size)


def need(values, axis) -> np.ndarray:
    """Scale bytes of finite sizes."""
    most = np.max(np.where(np.isfinite(values), np.abs(values), 0.0), axis=axis)
    out = np.zeros(most.shape, dtype=np.int64)
    for at in np.ndindex(most.shape):
        if most[at] > 0:
            power = -126
            while most[at] > 448 * 2.0 ** power:
                power += 1
            out[at] = power + 127
    return out


def scale(byte) -> np.ndarray:
    return 2.0 ** (np.asarray(byte, dtype=np.float64) - 127)


def value_order(codes) -> np.ndarray:
    """Codes [.., 16, D] as value blocks hold them."""
    codes = np.asarray(codes)
    D = codes.shape[-1]
    out = np.empty(codes.shape[:-2] + (D // 64, 4, 16, 4, 4), dtype=codes.dtype)
    for token in range(16):
        for e in range(D):
            out[..., e // 64, token // 4, e % 64 // 4, e % 4, token % 4] = codes[..., token, e]
    return out


def token_order(codes) -> np.ndarray:
    """Value blocks' codes as [.., 16, D]."""
    codes = np.asarray(codes)
    D = 64 * codes.shape[-5]
    out = np.empty(codes.shape[:-5] + (16, D), dtype=codes.dtype)
    for token in range(16):
        for e in range(D):
            out[..., token, e] = codes[..., e // 64, token // 4, e % 64 // 4, e % 4, token % 4]
    return out


def pack(dense):
    """(codes, bytes) of blocks [n, H, 16, D]."""
    x = to_f64(dense)
    byte = need(x, (2, 3))
    return encode(x / scale(byte)[..., None, None]), byte.astype(np.uint8)


def values(codes, byte) -> np.ndarray:
    """What codes [n, H, 16, D] (token order) and bytes [n, H] stand for."""
    return decode(codes) * scale(byte)[..., None, None]


def fill(new, codes, byte, query_offsets, suffix_tables, suffix_lens):
    """The pool after new rows [T, H, D] (float64) went to their slots: codes [n, H, 16, D]
    in token order, bytes [n, H]."""
    off, lens, tab = _ints(query_offsets), _ints(suffix_lens), _ints(suffix_tables)
    codes, byte = np.array(codes), np.array(byte).astype(np.int64)
    for r in range(len(lens)):
        n = int(off[r + 1] - off[r])
        p, row = int(lens[r]) - n, int(off[r])
        while p < int(lens[r]):
            m = min(int(lens[r]) - p, 16 - p % 16)
            at, first = int(tab[r, p // 16]), p % 16
            x = np.asarray(new[row:row + m]).transpose(1, 0, 2)                   # [H, m, D]
            want = need(x, (1, 2))
            now = want if first == 0 else np.maximum(want, byte[at])
            for h in range(len(now)):
                if first > 0 and now[h] > byte[at, h]:
                    was = codes[at, h, :first]
                    again = encode(decode(was) * 2.0 ** float(byte[at, h] - now[h]))
                    codes[at, h, :first] = np.where(was % 128 == 127, was, again)
                codes[at, h, first:first + m] = encode(x[h] / scale(now[h]))
            byte[at] = now
            p, row = p + m, row + m
    return codes, byte.astype(np.uint8)


def copy_blocks(pools, src, dst):
    """Every pool with block dst[i] equal to what block src[i] was."""
    out = []
    for pool in pools:
        after = np.array(pool)
        for a, b in zip(src, dst):
            if 0 <= a < len(pool) and 0 <= b < len(pool):
                after[b] = pool[a]
        out.append(after)
    return out


__all__ = ["SIZES", "encode", "decode", "need", "scale", "value_order", "token_order", "pack", "values", "fill",
           "copy_blocks"]
