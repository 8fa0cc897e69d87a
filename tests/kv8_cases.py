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


def gathered(pool, bt_row, begin, end, fmt):
    """The row's tokens [begin, end) as the read-back gives them: fp16 of the fp32 product."""
    k, v, ks, vs = kv8.views(pool[np.asarray(bt_row[begin // 16:-(-end // 16)], dtype=np.int64)])
    val = kv8.VALUES[fmt].astype(np.float32)
    K = (val[k] * ks[..., None]).transpose(0, 2, 1, 3)
    V = (val[v].transpose(0, 1, 2, 4, 3).reshape(k.shape) * vs[..., None]).transpose(0, 2, 1, 3)
    cut = slice(begin % 16, begin % 16 + end - begin)
    return tuple(x.reshape(-1, *x.shape[2:])[cut].astype(np.float16) for x in (K, V))
