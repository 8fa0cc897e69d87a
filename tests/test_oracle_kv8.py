"""Pins of the 8-bit cache's oracle: codes by hand, ties, the record's layout, and its read."""
import numpy as np

from oracle import kv8


def vec(*x):
    v = np.zeros(kv8.D, dtype=np.float16)
    v[:len(x)] = x
    return v


def test_e4m3_values():
    v = kv8.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[0x38] == 1 and v[0x39] == 1.125 and v[126] == 448 and v[128 | 126] == -448 and np.isnan(v[127])


def test_int8_codes_and_ties():
    codes, s = kv8.quantise(vec(127, -127, 0.5, 1.5, 2.5, -0.5, -1.5), kv8.INT8)
    assert codes[:7].view(np.int8).tolist() == [127, -127, 0, 2, 2, 0, -2] and s == 1
    # 63.5 of 127: a tie that real arithmetic has and fp32's 127 / 3 does not
    codes, s = kv8.quantise(vec(3, 1.5, -1.5), kv8.INT8)
    assert codes[:3].view(np.int8).tolist() == [127, 64, -64] and s == np.float32(3 / 127)


def test_e4m3_codes_and_ties():
    codes, s = kv8.quantise(vec(448, 17, 18, 19, -19, 2.0 ** -10, 3 * 2.0 ** -10), kv8.E4M3)
    assert s == 1
    assert kv8.VALUES[kv8.E4M3][codes[:7]].tolist() == [448, 16, 18, 20, -20, 0, 2 * 2.0 ** -9]


def test_zero_and_non_finite_vectors():
    for fmt in (kv8.INT8, kv8.E4M3):
        codes, s = kv8.quantise(vec(), fmt)
        assert s == 0 and not codes.any()
        for bad in (np.inf, -np.inf, np.nan):
            codes, s = kv8.quantise(vec(1, bad), fmt)
            assert np.isnan(s) and not codes.any()
        codes, s = kv8.quantise(vec(2.0 ** -24), fmt)  # the smallest subnormal is the largest value
        assert kv8.VALUES[fmt][codes[0]] == kv8.TOP[fmt] and s > 0


def test_record_layout_and_round_trip():
    r = np.random.default_rng(1)
    for fmt, step in ((kv8.INT8, 0.5 / 127), (kv8.E4M3, 2.0 ** -4)):
        pool = np.zeros((3, 2, kv8.RECORD), dtype=np.uint8)
        k, v = (r.standard_normal((21, 2, kv8.D)).astype(np.float16) for _ in "kv")
        bt = np.array([[2, 0]])
        pool = kv8.ref_append(pool, k, v, bt, [21], fmt, [0, 21])
        kc, vc, ks, vs = kv8.views(pool)
        codes, s = kv8.quantise(v[6, 1], fmt)
        assert np.array_equal(vc[2, 1, 1, :, 2], codes) and vs[2, 1, 6] == s
        assert pool[2, 1, 2048 + 512 + 4 * 9 + 2] == codes[9]
        codes, s = kv8.quantise(k[20, 0], fmt)
        assert np.array_equal(kc[0, 0, 4], codes) and ks[0, 0, 4] == s
        K, V = kv8.stored(pool, bt[0], 21, fmt)
        for x, y in ((K, k), (V, v)):
            top = np.abs(y.astype(np.float64)).max(-1, keepdims=True)
            assert np.all(np.abs(x - y) <= step * np.maximum(top if fmt == kv8.INT8 else np.abs(y), top * 2.0 ** -14) * 1.0001)
        assert not pool[1].any()


def test_attention_of_the_stored_values():
    from oracle import ref_decode
    r = np.random.default_rng(2)
    pool = np.zeros((4, 2, kv8.RECORD), dtype=np.uint8)
    bt, lens = np.array([[3, 1], [0, 0]]), [30, 0]
    k, v = (r.integers(-127, 128, (30, 2, kv8.D)).astype(np.float16) for _ in "kv")
    k[:, :, 0] = v[:, :, 0] = 127  # scale 1: the stored values are the values
    pool = kv8.ref_append(pool, k, v, bt, lens, kv8.INT8, [0, 30, 30])
    q = (r.standard_normal((2, 4, kv8.D)) / 100).astype(np.float16)
    k16, v16 = np.zeros((4, 16, 2, kv8.D), dtype=np.float16), np.zeros((4, 16, 2, kv8.D), dtype=np.float16)
    for t in range(30):
        k16[bt[0, t // 16], t % 16], v16[bt[0, t // 16], t % 16] = k[t], v[t]
    a, b = kv8.ref_decode8(q, pool, bt, lens, kv8.INT8, 0.3), ref_decode(q, k16, v16, bt, lens, 0.3)
    assert np.abs(a - b).max() < 1e-12 * np.abs(b).max()


def test_error_of_a_value():
    """At most half a step of its code: m / 254 in int8, the larger of 2^-4 |x| and 2^-10 m / 448 in e4m3, plus the
    scale's rounding. Every fp16 magnitude up to m, for several m; each bound is reached to within 5%."""
    every = np.arange(0x7C00, dtype=np.uint16).view(np.float16)
    for m in (65504.0, 1.0, 3.0, 1.7, 0.0101, 2.0 ** -14):
        m = float(np.float16(m))
        x = every[every <= m]
        x = np.concatenate([x, np.zeros(-len(x) % 127, dtype=np.float16)]).reshape(-1, 127)
        x = np.concatenate([np.full((len(x), 1), m, dtype=np.float16), x], 1)
        v = x.astype(np.float64)
        for fmt, half in ((kv8.INT8, np.full_like(v, m / 254)), (kv8.E4M3, np.maximum(2.0 ** -4 * v, 2.0 ** -10 * m / 448))):
            codes, s = kv8.quantise(x, fmt)
            err = np.abs(kv8.VALUES[fmt][codes] * s[:, None].astype(np.float64) - v)
            assert np.all(err <= half + 2.0 ** -24 * v), (m, fmt)
            if m >= 1:
                assert (err / half).max() > 0.95
