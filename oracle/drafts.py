"""Plain float64 forms of a drafting step (test infrastructure).

  fill     per head x of a row: y = x / sqrt(mean(x^2) + eps) * w, then each pair
           (a, b) of the first RD elements turns by position * f_i:
           (a cos - b sin, b cos + a sin) times the amplitude.
  tree     row j of a request attends to its chain's prefixes, the request's own
           tokens before the drafted ones, and the drafted tokens on the path from
           the root to j; query head i reads cache head i // (HQ / H).
  accept   from the cached context, again and again the lowest row whose parent is
           the row reached last and whose token is the one chosen there.
  commit   the slots the accepted rows move between.

Written out row by row, with no blocking or bit sets.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import _ints, group_chain, request_kv, to_f64


def tree_path(parents, j: int) -> list:
    """Rows from the root to j (parents of one request; None: a chain)."""
    path = [j]
    while (path[-1] - 1 if parents is None else int(parents[path[-1]])) >= 0:
        path.append(path[-1] - 1 if parents is None else int(parents[path[-1]]))
    return path[::-1]


def shared_prefix_tree(q, query_offsets, tree_parents, prefix_k, prefix_v, suffix_k, suffix_v, prefix_tables,
                       prefix_lens, suffix_tables, suffix_lens, group_ids, sm_scale, prefix_parents=None, unit=0.0):
    """(out [T, HQ, D], lse [T, HQ], spread [T, HQ, D], noise [T, HQ]) in float64, NaN
    in rows that no request holds.  spread is sum_j w_j |v_j - out|, by which a
    relative error of each weight enters the output, plus `unit` times |out|; noise is
    the largest sum_d |q_d k_d| of a visible key, scaled as the logits are."""
    qf, off, lens = to_f64(q), _ints(query_offsets), _ints(suffix_lens)
    T, HQ, D = qf.shape
    out, lse = np.full((T, HQ, D), np.nan), np.full((T, HQ), np.nan)
    spread, noise = np.full((T, HQ, D), np.nan), np.full((T, HQ), np.nan)
    for r in range(len(lens)):
        first, n = int(off[r]), int(off[r + 1] - off[r])
        if n == 0:
            continue
        K, V = request_kv(r, prefix_k=prefix_k, prefix_v=prefix_v, suffix_k=suffix_k, suffix_v=suffix_v,
                          prefix_tables=prefix_tables, prefix_lens=prefix_lens, suffix_tables=suffix_tables,
                          suffix_lens=suffix_lens, group_ids=group_ids, prefix_parents=prefix_parents)
        before = K.shape[0] - n
        parents = None if tree_parents is None else _ints(tree_parents)[first:first + n]
        ratio = HQ // K.shape[1]
        for j in range(n):
            seen = list(range(before)) + [before + a for a in tree_path(parents, j)]
            for i in range(HQ):
                k, v = K[seen, i // ratio], V[seen, i // ratio]
                s = sm_scale * (k @ qf[first + j, i])
                m = s.max()
                total = m + math.log(np.exp(s - m).sum())
                w = np.exp(s - total)
                o = w @ v
                out[first + j, i], lse[first + j, i] = o, total
                spread[first + j, i] = w @ np.abs(v - o) + unit * np.abs(o)
                noise[first + j, i] = abs(sm_scale) * (np.abs(k) @ np.abs(qf[first + j, i])).max()
    return out, lse, spread, noise


def rotary_frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0, original_length=0.0, low=None, high=None):
    """(angle per position of every pair, amplitude)."""
    out, amplitude = [], 1.0
    for i in range(rotary_dim // 2):
        b = base * factor ** (rotary_dim / (rotary_dim - 2)) if scaling == "ntk" else base
        f = b ** (-2 * i / rotary_dim)
        if scaling == "linear":
            f = f / factor
        if scaling == "wavelength":
            lo, hi = low or 1.0, high or 4.0
            wavelength = 2 * math.pi / f
            if wavelength > original_length / lo:
                f = f / factor
            elif wavelength >= original_length / hi:
                keep = (original_length / wavelength - lo) / (hi - lo)
                f = keep * f + (1 - keep) * f / factor
        if scaling == "yarn":
            lo, hi = low or 1.0, high or 32.0
            place = lambda t: rotary_dim * math.log(original_length / (2 * math.pi * t)) / (2 * math.log(base))
            a, z = max(0, math.floor(place(hi))), min(rotary_dim - 1, math.ceil(place(lo)))
            ramp = min(1.0, max(0.0, (i - a) / max(z - a, 1e-3)))
            f = f * (1 - ramp) + f / factor * ramp
            amplitude = 0.1 * math.log(factor) + 1
        out.append(f)
    return out, amplitude


def rotate(x, positions, radians, interleaved, amplitude, weight=None, eps=0.0):
    """(y, size) of heads x [T, heads, D] (float64): size is |a| + |b| of each element's
    pair after the norm and times the amplitude (|x| outside the pairs), by which the
    errors of sine and cosine enter y."""
    x = to_f64(x)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * to_f64(weight)
    y, size = x.copy(), np.abs(x)
    half = len(radians)
    for i, f in enumerate(radians):
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * f
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        a, b = x[..., one], x[..., two]
        y[..., one], y[..., two] = a * c - b * s, b * c + a * s
        size[..., one] = size[..., two] = amplitude * (np.abs(a) + np.abs(b))
    return y, size


def fill_slots(query_offsets, suffix_tables, suffix_lens, block=16):
    """(row, block, offset) of every row that a request holds."""
    off, lens, tab = _ints(query_offsets), _ints(suffix_lens), _ints(suffix_tables)
    rows = []
    for r in range(len(lens)):
        n = int(off[r + 1] - off[r])
        for j in range(n):
            p = int(lens[r]) - n + j
            rows.append((int(off[r]) + j, int(tab[r, p // block]), p % block))
    return rows


def tree_accept(query_offsets, tree_parents, draft, target, root):
    """(accept_rows [T] with -1 behind a request's, accept_lens, next_tokens)."""
    off = _ints(query_offsets)
    rows = np.full(len(draft), -1, dtype=np.int64)
    lens, follow = [], []
    for r in range(len(off) - 1):
        at, want, n = -1, int(root[r]), 0
        while True:
            fits = [j for j in range(int(off[r + 1] - off[r]))
                    if (j - 1 if tree_parents is None else int(tree_parents[off[r] + j])) == at
                    and int(draft[off[r] + j]) == want]
            if not fits:
                break
            at = min(fits)
            want = int(target[off[r] + at])
            rows[off[r] + n] = at
            n += 1
        lens.append(n)
        follow.append(want)
    return rows, np.array(lens), np.array(follow)


def tree_commit(query_offsets, accept_rows, accept_lens, suffix_tables, suffix_lens, block=16):
    """(moves [((block, offset) from, (block, offset) to)], committed lengths)."""
    off, lens, tab = _ints(query_offsets), _ints(suffix_lens), _ints(suffix_tables)
    moves, after = [], []
    slot = lambda r, p: (int(tab[r, p // block]), p % block)
    for r in range(len(lens)):
        cached = int(lens[r] - (off[r + 1] - off[r]))
        for i in range(int(accept_lens[r])):
            moves.append((slot(r, cached + int(accept_rows[off[r] + i])), slot(r, cached + i)))
        after.append(cached + int(accept_lens[r]))
    return moves, np.array(after)
