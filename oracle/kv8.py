"""Reference of the 8-bit paged KV cache: codes, records and reads in fp64 and integers.

TEST INFRASTRUCTURE: see the package docstring. A pool is uint8 [num_pages, Hkv, 4224]; a record
holds K codes [16][128], V codes [4][128][4], K scales fp32 [16] and V scales fp32 [16].
"""
from __future__ import annotations

import numpy as np

INT8, E4M3 = 0, 1
D, PAGE = 128, 16
RECORD = 2 * PAGE * D + 2 * PAGE * 4
TOP = {INT8: 127.0, E4M3: 448.0}


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 e4m3 codes (bias 7, no infinities, 0x7F and 0xFF NaN)."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (c & 127) == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v[c] = -x if c & 128 else x
    return v


VALUES = {INT8: np.arange(256).astype(np.uint8).view(np.int8).astype(np.float64), E4M3: e4m3_values()}


def quantise(x: np.ndarray, fmt: int):
    """x fp16 [..., D] -> (codes uint8 [..., D], scales fp32 [...]); exact: x * top / m is formed as a
    ratio of integers, so a tie is a tie."""
    x = np.asarray(x, dtype=np.float16)
    bad = ~np.isfinite(x).all(-1)
    xi = np.rint(np.where(bad[..., None], 0, x).astype(np.float64) * 2.0 ** 24).astype(np.int64)   # exact integers
    m = np.abs(xi).max(-1, keepdims=True)
    top = int(TOP[fmt])
    num, den = np.abs(xi) * top, np.maximum(m, 1)
    if fmt == INT8:
        q, r = num // den, num % den
        q = q + ((2 * r > den) | ((2 * r == den) & (q % 2 == 1)))
        codes = np.where(xi < 0, -q, q).astype(np.int8).view(np.uint8)
    else:
        # the grid of magnitudes in steps of 2^-9 and the borders between neighbours in 2^-10
        grid = np.rint(VALUES[E4M3][:127] * 2 ** 9).astype(np.int64)
        border = grid[:-1] + grid[1:]
        scaled = num << 10
        q = np.zeros(num.shape, dtype=np.int64)
        for c, b in enumerate(border):  # past the border, or on it and the upper code is the even one
            q += (scaled > b * den) | ((scaled == b * den) & (c % 2 == 1))
        codes = (q + np.where(np.signbit(x), 128, 0)).astype(np.uint8)
    codes = np.where(bad[..., None] | (m == 0), 0, codes).astype(np.uint8)
    with np.errstate(invalid="ignore"):
        scale = np.abs(np.where(bad[..., None], 0, x).astype(np.float64)).max(-1) / TOP[fmt]
    return codes, np.where(bad, np.nan, scale).astype(np.float32)


def views(pool: np.ndarray):
    """K codes [pages, Hkv, 16, D], V codes [pages, Hkv, 4, D, 4], K and V scales [pages, Hkv, 16]."""
    n, h, _ = pool.shape
    k = pool[:, :, :PAGE * D].reshape(n, h, PAGE, D)
    v = pool[:, :, PAGE * D:2 * PAGE * D].reshape(n, h, 4, D, 4)
    s = pool[:, :, 2 * PAGE * D:].view(np.float32)
    return k, v, s[:, :, :PAGE], s[:, :, PAGE:]


def ref_append(pool, k, v, block_table, seq_lens, fmt, offsets=None) -> np.ndarray:
    """The pool after the write."""
    pool = pool.copy()
    kc, vc, ks, vs = views(pool)
    assert all(np.shares_memory(x, pool) for x in (kc, vc, ks, vs))
    (kq, ksc), (vq, vsc) = quantise(k, fmt), quantise(v, fmt)
    for i, n in enumerate(np.asarray(seq_lens).tolist()):
        b, e = (i, i + (n > 0)) if offsets is None else (int(offsets[i]), int(offsets[i + 1]))
        pos = np.arange(n - (e - b), n)
        page, s = np.asarray(block_table[i])[pos // PAGE], pos % PAGE
        kc[page, :, s] = kq[b:e]
        vc[page, :, s // 4, :, s % 4] = vq[b:e]
        ks[page, :, s] = ksc[b:e]
        vs[page, :, s] = vsc[b:e]
    return pool


def stored(pool, block_table_row, n: int, fmt: int):
    """(K, V) fp64 [n, Hkv, D]: the row's first n tokens as the pool holds them."""
    k, v, ks, vs = views(pool[np.asarray(block_table_row[:-(-n // PAGE)], dtype=np.int64)])
    val = VALUES[fmt]
    K = (val[k] * ks[..., None].astype(np.float64)).transpose(0, 2, 1, 3)
    V = (val[v].transpose(0, 1, 2, 4, 3).reshape(k.shape) * vs[..., None].astype(np.float64)).transpose(0, 2, 1, 3)
    return tuple(x.reshape(-1, *x.shape[2:])[:n] for x in (K, V))


def ref_decode8(q, pool, block_table, seq_lens, fmt, sm_scale: float = 1.0) -> np.ndarray:
    """Eq. (1) over the stored values, fp64 [B, Hq, D]; rows of length 0 give 0."""
    B, hq, _ = q.shape
    hkv = pool.shape[1]
    out = np.zeros((B, hq, D))
    for i, n in enumerate(np.asarray(seq_lens).tolist()):
        if n == 0:
            continue
        K, V = stored(pool, block_table[i], n, fmt)
        for h in range(hq):
            s = sm_scale * (K[:, h // (hq // hkv)] @ q[i, h].astype(np.float64))
            w = np.exp(s - s.max())
            out[i, h] = (w @ V[:, h // (hq // hkv)]) / w.sum()
    return out
