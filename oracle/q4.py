"""Plain CPU form of the 4-bit paged KV cache (include/pagedattn_q4.h), from
the format's definition in float64: quantising, the tiles' byte layout, the
append, the read and attention.  Test infrastructure; loops over what the
kernels do at once.
"""
from __future__ import annotations

import numpy as np

PAGE, BLOCK = 16, 32
MAGS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def tile_bytes(D):
    return PAGE * (D // 2 + D // BLOCK)


def quantise(x):
    """(codes [..., D] 0..15, scale bytes [..., D / 32]) of x [..., D]."""
    x = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    fine = np.isfinite(x).all(-1)
    x = np.where(fine[..., None], x, 0.0)
    a = np.abs(x).max(-1)
    m, k = np.frexp(a)  # a = m 2^k with 1/2 <= m < 1: (2 m) 2^(k - 1)
    e = np.where(2 * m <= 1.75, k - 1 - 2, k - 1 - 1)
    e = np.where(a == 0, 0, np.clip(e, -125, 125))
    y = np.abs(x) / np.ldexp(1.0, e)[..., None]
    # nearest magnitude; on a tie the even code
    d = np.abs(y[..., None] - MAGS)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = (code + 8 * np.signbit(x)) * fine[..., None]
    return code.reshape(*code.shape[:-2], -1).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    """float64 values of codes [..., D] with scale bytes [..., D / 32]."""
    c = codes.reshape(*codes.shape[:-1], codes.shape[-1] // BLOCK, BLOCK)
    x = np.where(c >= 8, -1.0, 1.0) * MAGS[c & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (x * s[..., None]).reshape(codes.shape)


def byte_of(which, D, token, pair):
    """Byte of a tile that holds dims 2 pair, 2 pair + 1 of a token."""
    w = D // 8
    if which == "k":
        return (pair // w * 16 + token) * w + pair % w
    return (token // 4 * 16 + pair % 16) * w + 4 * (pair // 16) + token % 4


def scale_byte_of(D, token, block):
    return 8 * D + token * (D // BLOCK) + block


def put(which, pool, page, g, token, x):
    """Quantise the vector x [D] into a pool [N][H_kv][tile]."""
    D = x.shape[-1]
    codes, scales = quantise(x)
    for m in range(D // 2):
        pool[page, g, byte_of(which, D, token, m)] = codes[2 * m] | codes[2 * m + 1] << 4
    for j in range(D // BLOCK):
        pool[page, g, scale_byte_of(D, token, j)] = scales[j]


def unpack(which, tiles, D):
    """float64 [..., 16, D] of tiles [..., tile]."""
    at = np.array([[byte_of(which, D, t, m) for m in range(D // 2)] for t in range(PAGE)])
    sc = np.array([[scale_byte_of(D, t, j) for j in range(D // BLOCK)] for t in range(PAGE)])
    b = tiles[..., at]
    codes = np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], D)
    return values(codes, tiles[..., sc])


def pack(which, x):
    """Pool tiles [..., tile] of x [..., 16, D]."""
    D = x.shape[-1]
    codes, scales = quantise(x)
    out = np.zeros(x.shape[:-2] + (tile_bytes(D),), np.uint8)
    at = np.array([[byte_of(which, D, t, m) for m in range(D // 2)] for t in range(PAGE)])
    sc = np.array([[scale_byte_of(D, t, j) for j in range(D // BLOCK)] for t in range(PAGE)])
    out[..., at] = codes[..., 0::2] | codes[..., 1::2] << 4
    out[..., sc] = scales
    return out


def rows_of(context_lens, query_start_loc):
    """(row, sequence, position) of every row of a call."""
    if query_start_loc is None:
        return [(b, b, int(c) - 1) for b, c in enumerate(context_lens) if c > 0]
    return [(r, b, int(context_lens[b]) - (int(query_start_loc[b + 1]) - r)) for b in range(len(context_lens))
            for r in range(int(query_start_loc[b]), int(query_start_loc[b + 1]))]


def append(k_new, v_new, block_table, context_lens, k_pages, v_pages, query_start_loc=None):
    """The pools after the append (copies)."""
    k_pages, v_pages = k_pages.copy(), v_pages.copy()
    for r, b, pos in rows_of(context_lens, query_start_loc):
        for g in range(k_new.shape[1]):
            put("k", k_pages, block_table[b, pos // PAGE], g, pos % PAGE, k_new[r, g])
            put("v", v_pages, block_table[b, pos // PAGE], g, pos % PAGE, v_new[r, g])
    return k_pages, v_pages


def dense(which, pool, block_table, b, C, D):
    """float64 [H_kv][C][D]: sequence b's first C tokens."""
    tiles = pool[block_table[b, :(C + PAGE - 1) // PAGE]]
    x = unpack(which, tiles, D)
    return x.transpose(1, 0, 2, 3).reshape(pool.shape[1], -1, D)[:, :C]


def attention(q, k_pages, v_pages, block_table, context_lens, scale, query_start_loc=None):
    """(out, spread, mass, size, reach) in float64: the attention [rows][H_q][D],
    sum_t w_t |v_t|, sum_t |v_t|, and per (row, head) the largest scale * sum_d |q_d k_d| and scale *
    max_d |q_d| * sum_d |k_d| of its keys.  Rows of no sequence are NaN; of an empty
    decode context 0."""
    rows, H_q, D = q.shape
    H_kv = k_pages.shape[1]
    s = H_q // H_kv
    out, spread, size = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.zeros((rows, H_q))
    mass, reach = np.zeros(q.shape), np.zeros((rows, H_q))
    for b, C in enumerate(int(c) for c in context_lens):
        r0, r1 = (b, b + 1) if query_start_loc is None else (int(query_start_loc[b]), int(query_start_loc[b + 1]))
        if C == 0:
            out[r0:r1] = spread[r0:r1] = 0.0
            continue
        if r0 == r1:
            continue
        k, v = dense("k", k_pages, block_table, b, C, D), dense("v", v_pages, block_table, b, C, D)
        for r in range(r0, r1):
            n = C - (r1 - r0) + (r - r0) + 1
            for h in range(H_q):
                g = h // s
                qk = q[r, h].astype(np.float64) * k[g, :n]
                x = scale * qk.sum(-1)
                with np.errstate(all="ignore"):
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    out[r, h], spread[r, h] = w @ v[g, :n], w @ np.abs(v[g, :n])
                mass[r, h] = np.abs(v[g, :n]).sum(0)
                size[r, h] = scale * np.abs(qk).sum(-1).max()
                reach[r, h] = scale * np.abs(q[r, h]).max() * np.abs(k[g, :n]).sum(-1).max()
    return out, spread, mass, size, reach
