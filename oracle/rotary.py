"""Oracle for rotary positions with several axes and for the cache append.

Test infrastructure only (see the package docstring).

``rope_axes`` turns the pairs (i, i + P) of every head's first 2P channels by
pos[a] * theta^(-i / P), or theta^(-(i - i0) / n_a) with the frequencies
restarted in every axis; axis a owns the next sections[a] pairs.  Angles are
formed in extended precision, so that far positions keep their fraction.

``kv_append`` writes rotated keys, and values, to the last positions of each
sequence: row row_start[b] + j of n_b rows takes position kv_len[b] - n_b + j.
"""

import numpy as np


def rope_angles(pos, sections, theta, per_axis=False):
    """[T, P] angles (extended precision) of pos [axes, T]."""
    pos = np.asarray(pos)
    cols = []
    first, pairs = 0, sum(sections)
    for a, n in enumerate(sections):
        for i in range(n):
            e = np.longdouble(i) / n if per_axis else np.longdouble(first + i) / pairs
            cols.append(pos[a].astype(np.longdouble) * np.longdouble(theta) ** -e)
        first += n
    return np.stack(cols, axis=1)


def rope_axes(x, pos, sections, theta, per_axis=False, inverse=False):
    """x [T, H, D] -> float64 [T, H, D]."""
    x = np.asarray(x, np.float64)
    ang = rope_angles(pos, sections, theta, per_axis)
    c = np.cos(ang).astype(np.float64)[:, None]
    s = np.sin(ang).astype(np.float64)[:, None] * (-1.0 if inverse else 1.0)
    P = ang.shape[1]
    y = x.copy()
    y[..., :P] = x[..., :P] * c - x[..., P:2 * P] * s
    y[..., P:2 * P] = x[..., :P] * s + x[..., P:2 * P] * c
    return y


def append_places(row_start, kv_len, T):
    """(sequence, cache position) of every row; sequence -1 for rows of none."""
    seq = np.full(T, -1, np.int64)
    place = np.zeros(T, np.int64)
    for b in range(len(kv_len)):
        n = int(row_start[b + 1]) - int(row_start[b])
        for j in range(n):
            seq[int(row_start[b]) + j] = b
            place[int(row_start[b]) + j] = int(kv_len[b]) - n + j
    return seq, place


def kv_append(q, k, v, k_cache, v_cache, kv_len, row_start, sections, theta, pos=None, per_axis=False,
              page_table=None, page_size=16):
    """Returns (q, k_cache, v_cache) in float64; rows of no sequence leave q at NaN."""
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    T = k.shape[0]
    seq, place = append_places(row_start, kv_len, T)
    if sections:
        p = np.asarray(pos) if pos is not None else np.stack([place] * len(sections))
        k = rope_axes(k, p, sections, theta, per_axis)
        qo = rope_axes(q, p, sections, theta, per_axis) if q is not None else None
    else:
        qo = np.array(q, np.float64) if q is not None else None
    kc, vc = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    for t in range(T):
        b, at = seq[t], place[t]
        if b < 0:
            if qo is not None:
                qo[t] = np.nan
            continue
        if page_table is None:
            if 0 <= at < kc.shape[1]:
                kc[b, at], vc[b, at] = k[t], v[t]
        elif 0 <= at < page_size * page_table.shape[1]:
            page = page_table[b, at // page_size]
            if 0 <= page < kc.shape[0]:
                kc[page, :, at % page_size], vc[page, :, at % page_size] = k[t], v[t]
    return qo, kc, vc
