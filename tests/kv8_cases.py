"""Shared by the CPU and GPU tests of the 8-bit cache: how far an attention output may be off."""
import numpy as np

from oracle import kv8


def decode_bound(q, pool, bt, lens, fmt, sm_scale):
    """(reference, bound) [B, Hq, 128]. The output rounds to fp16: half a step, 2^-11 of the value
    (2^-25 where it is subnormal). The weights of the second product carry 16 bits: 2^-16 of the
    mean of |v| under them. A score is an fp32 sum of 128 exact products: 128 * 2^-24 of the sum of
    their magnitudes, and an error e of a score moves the output by at most 2 e mean|v|; the scale, exp2
    and their products add 2^-20. Sums over n tokens in fp32: n * 2^-24 / 4 (four lanes share them)."""
    ref = kv8.ref_decode8(q, pool, bt, lens, fmt, sm_scale)
    tol = np.abs(ref) * 2.0 ** -11 + 2.0 ** -25
    hq, hkv = q.shape[1], pool.shape[1]
    for i, n in enumerate(np.asarray(lens).tolist()):
        if n == 0:
            continue
        K, V = kv8.stored(pool, bt[i], n, fmt)
        for h in range(hq):
            k, v, x = K[:, h // (hq // hkv)], np.abs(V[:, h // (hq // hkv)]), q[i, h].astype(np.float64)
            s = sm_scale * (k @ x)
            w = np.exp(s - s.max())
            size = abs(sm_scale) * (np.abs(k) @ np.abs(x)).max()
            tol[i, h] += (w @ v) / w.sum() * (2.0 ** -16 + 2.0 ** -20 * (1 + np.abs(s).max()) + 2 * 2.0 ** -17 * size + n * 2.0 ** -26)
    return ref, tol


def assert_decode(out, q, pool, bt, lens, fmt, sm_scale, what=""):
    ref, tol = decode_bound(q, pool, bt, lens, fmt, sm_scale)
    err = np.abs(np.asarray(out, dtype=np.float64) - ref)
    assert np.all(err <= tol), (what, float((err / tol).max()), float(np.nanmax(err)))


def fine_bound(q, pool, bt, lens, fmt, sm_scale):
    """(reference, bound) [B, Hq, 128] for rows of at most 32 tokens, whose weights are formed under one
    maximum, with no factor that real errors cannot reach (decode_bound, for rows of any length, grants the weights
    8 bits less than they have, and scores the worst order of sums). With S = |scale| sum|q k| of a token:
    - a score s: the scale to fp32 and times log2(e), that times the query's unit and the K scale, and the sum
      times that, and the sum of its two halves: five roundings, 2^-24 each. The halves themselves: in int8 the query
      x = 2^24 d3 + 2^16 d2 + 2^8 d1 + d0 is taken as d3, d1 and d2, d0, whose exact sums are joined in one rounding each,
      and in one more where there are digits beyond, and |2^24 d3 + 2^8 d1| + |2^16 d2 + d0| <= 3.01 |x| (the second
      sum is at most 2^23 + 2^7, and d3 = 0 unless |x| >= 2^23 - 2^15 - 2^7): 6.1 S of 2^-24. In e4m3 each of 129
      additions is off by at most 2^-23 of S.
    - a weight, relatively: the error of s; s - max rounded, 2^-24 of it; exp2 2^-23.
    - a weight's error d moves the output by p d |v - o| (p: the weight over the weights' sum, o: the output).
    - weight times V scale 2^-24 and its parts 2^-24; a dim's sum has three parts of n products, each addition off by
      at most 2^-23 of mean|v|; the sum of weights n + 4 roundings, its reciprocal and product 2^-22, of o.
    - the output's rounding: 2^-11 of the value, 2^-25 where it is subnormal."""
    ref = kv8.ref_decode8(q, pool, bt, lens, fmt, sm_scale)
    tol = np.abs(ref) * 2.0 ** -11 + 2.0 ** -25
    hq, hkv = q.shape[1], pool.shape[1]
    for i, n in enumerate(np.asarray(lens).tolist()):
        assert n <= 32
        if n == 0:
            continue
        K, V = kv8.stored(pool, bt[i], n, fmt)
        for h in range(hq):
            k, v, x = K[:, h // (hq // hkv)], V[:, h // (hq // hkv)], q[i, h].astype(np.float64)
            s, size = sm_scale * (k @ x), abs(sm_scale) * (np.abs(k) @ np.abs(x))
            p = np.exp(s - s.max())
            p /= p.sum()
            d = 2.0 ** -24 * (5 * np.abs(s) + (6.1 if fmt == kv8.INT8 else 2 * 129) * size + np.abs(s - s.max())) + 2.0 ** -23
            tol[i, h] += (p * d) @ np.abs(v - ref[i, h]) + (p @ np.abs(v)) * (2.0 ** -23 + 3 * n * 2.0 ** -23)
            tol[i, h] += np.abs(ref[i, h]) * ((n + 4) * 2.0 ** -24 + 2.0 ** -22)
    return ref, tol


def assert_fine(out, q, pool, bt, lens, fmt, sm_scale):
    ref, tol = fine_bound(q, pool, bt, lens, fmt, sm_scale)
    err = np.abs(np.asarray(out, dtype=np.float64) - ref)
    assert np.all(err <= tol), (float((err / tol).max()), float(np.nanmax(err)))


def outlier_queries(cache, hq, large, small, seed=3):
    """Queries with one large channel whose K codes are all 0: the scores are those of the small ones."""
    r = np.random.default_rng(seed)
    kv8.views(cache.pool)[0][..., 5] = 0
    q = (r.standard_normal((cache.B, hq, 128)) * small).astype(np.float16)
    q[..., 5] = large
    return q


def shared_prefix(fmt, seed=9):
    """Rows whose tables name the same pages: a prefix of 37 pages, then pages of their own; the last row is the
    prefix alone, cut inside a page, and names its first page twice."""
    from tests.cpu_kv8 import Cache
    c = Cache([700, 640, 593, 37 * 16, 400], 2, fmt, seed=seed)
    c.bt[1:4, :37] = c.bt[0, :37]
    c.bt[4, :25] = c.bt[0, :25]
    c.bt[4, 20] = c.bt[4, 0]
    return c


def opposed_values(rows, hq, fmt, seed=6):
    """Rows of two tokens with nearly equal scores and opposed V: outputs are a small part of the values."""
    from tests.cpu_kv8 import Cache
    c, r = Cache([2] * rows, 2, fmt, seed=seed), np.random.default_rng(seed)
    _, v, _, vs = kv8.views(c.pool)
    first = c.bt[:, 0]
    v[first, :, 0, :, 1] = -v[first, :, 0, :, 0].view(np.int8).astype(np.int16) if fmt == kv8.INT8 else v[first, :, 0, :, 0] ^ 128
    vs[first, :, 1] = vs[first, :, 0]
    return c, (r.standard_normal((rows, hq, 128)) * 0.002).astype(np.float16)


def gathered(pool, bt_row, begin, end, fmt):
    """The row's tokens [begin, end) as the read-back gives them: fp16 of the fp32 product."""
    k, v, ks, vs = kv8.views(pool[np.asarray(bt_row[begin // 16:-(-end // 16)], dtype=np.int64)])
    val = kv8.VALUES[fmt].astype(np.float32)
    K = (val[k] * ks[..., None]).transpose(0, 2, 1, 3)
    V = (val[v].transpose(0, 1, 2, 4, 3).reshape(k.shape) * vs[..., None]).transpose(0, 2, 1, 3)
    cut = slice(begin % 16, begin % 16 + end - begin)
    return tuple(x.reshape(-1, *x.shape[2:])[cut].astype(np.float16) for x in (K, V))
