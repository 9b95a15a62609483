"""Plain CPU form of the 8-bit paged KV cache (include/pagedattn_q8.h), from the
format's definition in float64: the scale rule, rounding, the tiles' byte layout,
the append with its pages' growing scales, and the read.  Test infrastructure;
loops over what the kernels do at once.
"""
from __future__ import annotations

import numpy as np

from oracle.q4 import rows_of

PAGE = 16
E_LOW, E_HIGH = -110, 119


def _e4m3_values():
    v = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return v


VALUES = _e4m3_values()
_MAGS = VALUES[:127]  # 0 .. 448, increasing with the code


def exponent(x):
    """The scale's exponent that the finite values x need."""
    x = np.asarray(x, np.float64).ravel()
    x = np.abs(x[np.isfinite(x)])
    a = x.max() if x.size else 0.0
    if a == 0:
        return E_LOW
    m, k = np.frexp(a)  # 1/2 <= m < 1: a = (2 m) 2^(k - 1)
    return int(np.clip(k - 1 - 8 if 2 * m <= 1.75 else k - 1 - 7, E_LOW, E_HIGH))


def codes(x, e):
    """Code of the e4m3 nearest to each x / 2^e, ties to the even code; NaN's for what
    is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    y = np.minimum(np.abs(np.where(fine, x, 0.0)) * 2.0 ** -e, 448.0)
    hi = np.clip(np.searchsorted(_MAGS, y), 0, 126)  # the first magnitude not below y
    lo = np.maximum(hi - 1, 0)
    d_hi, d_lo = _MAGS[hi] - y, y - _MAGS[lo]
    c = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return np.where(fine, c | 128 * np.signbit(x), 127).astype(np.uint8)


def byte_of(which, token, d):
    """Byte of a tile that holds dim d of a token."""
    if which == "k":
        return (d // 16 * 16 + token) * 16 + d % 16
    return d // 64 * 1024 + (token // 4 * 16 + d % 32 // 2) * 16 + d // 32 % 2 * 8 + d % 2 * 4 + token % 4


def places(which, D):
    """[16][D]: byte_of."""
    return np.array([[byte_of(which, t, d) for d in range(D)] for t in range(PAGE)])


def unpack(which, tiles, scales, D):
    """float64 [..., 16, D] of tiles [..., 16 D] with scale bytes [...]."""
    return VALUES[tiles[..., places(which, D)]] * np.ldexp(1.0, scales.astype(np.int64) - 127)[..., None, None]


def pack(which, x):
    """(tiles [..., 16 D], scale bytes [...]) of x [..., 16, D]."""
    D, flat = x.shape[-1], x.reshape(-1, *x.shape[-2:])
    tiles, scales = np.zeros((len(flat), PAGE * D), np.uint8), np.zeros(len(flat), np.uint8)
    for i, page in enumerate(flat):
        e = exponent(page)
        tiles[i, places(which, D)] = codes(page, e)
        scales[i] = e + 127
    return tiles.reshape(*x.shape[:-2], -1), scales.reshape(x.shape[:-2])


def append(k_new, v_new, block_table, context_lens, k_pages, v_pages, scales, query_start_loc=None, keep=None):
    """(k_pages, v_pages, scales) after the append (copies).  keep: rows that are
    written (None: all)."""
    pools, scales = [k_pages.copy(), v_pages.copy()], scales.copy()
    D = k_new.shape[-1]
    written = {}  # (sequence, page of it) -> rows with their slots
    for r, b, pos in rows_of(context_lens, query_start_loc):
        if keep is None or keep[r]:
            written.setdefault((b, pos // PAGE), []).append((r, pos % PAGE))
    for (b, p), rows in written.items():
        page, first = block_table[b, p], rows[0][1]
        for which, (name, new) in enumerate((("k", k_new), ("v", v_new))):
            at = places(name, D)
            for g in range(new.shape[1]):
                tile, e = pools[which][page, g], exponent(new[[r for r, _ in rows], g])
                if first > 0:
                    held = int(scales[page, g, which]) - 127
                    e = max(e, held)
                    if e > held:
                        tile[at[:first]] = codes(VALUES[tile[at[:first]]] * 2.0 ** (held - e), 0)
                for r, t in rows:
                    tile[at[t]] = codes(new[r, g], e)
                scales[page, g, which] = e + 127
    return pools[0], pools[1], scales


def dense(which, pool, scales, block_table, b, C, D):
    """float64 [H_kv][C][D]: sequence b's first C tokens."""
    pages = block_table[b, :(C + PAGE - 1) // PAGE]
    x = unpack(which, pool[pages], scales[pages][..., 0 if which == "k" else 1], D)
    return x.transpose(1, 0, 2, 3).reshape(pool.shape[1], -1, D)[:, :C]


def read(k_pages, v_pages, scales, block_table, context_lens, D, query_start_loc=None, keep=None):
    """float64 [2][rows][H_kv][D], NaN where keep is false or no sequence has the row."""
    rows = rows_of(context_lens, query_start_loc)
    T = len(context_lens) if query_start_loc is None else int(query_start_loc[-1])
    out = np.full((2, T, k_pages.shape[1], D), np.nan)
    for r, b, pos in rows:
        if keep is None or keep[r]:
            page = block_table[b, pos // PAGE]
            for which, (name, pool) in enumerate((("k", k_pages), ("v", v_pages))):
                x = unpack(name, pool[page], scales[page, :, which], D)
                out[which, r] = x[:, pos % PAGE]
    return out
