"""Numerics of the 8-bit cache's kernels at their borders, their own sources on the CPU: zeros of both
signs, queries of many sizes and values that cancel."""
import numpy as np
import pytest

from oracle import kv8
from tests import cpu_kv8
from tests.cpu_cases import compiler
from tests.cpu_kv8 import Cache, call
from tests.kv8_cases import assert_decode, assert_fine, gathered, opposed_values, outlier_queries, shared_prefix

FORMATS = [kv8.INT8, kv8.E4M3]

pytestmark = pytest.mark.skipif(compiler() is None, reason="needs clang")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return cpu_kv8.build(str(tmp_path_factory.mktemp("cpu_kv8")))


def signed_zeros():
    """[8, 2, 128]: vectors of zeros of both signs, and such zeros beside one value."""
    x = np.zeros((8, 2, 128), dtype=np.float16)
    x[1] = -0.0
    x[2, :, ::3] = -0.0
    x[3, 1, 127] = -0.0
    x[4:] = x[:4]
    x[4:, :, 64] = [[3], [-3], [2.0 ** -24], [-65504]]
    return x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("offsets", [[0, 8], None])
def test_zeros_of_both_signs(exe, fmt, offsets):
    """A vector without a value has codes 0; beside a value a zero keeps its sign where the format has one."""
    x = signed_zeros()
    c = Cache([8] if offsets else [3] * 8, 2, fmt, filled=False)
    (st, bits, _, pool), = call(exe, "append", c, k=x.reshape(8, 256), v=x[::-1].reshape(8, 256).copy(), tokens=8,
                                offsets=None if offsets is None else np.array(offsets))
    assert (st, bits) == (0, 0)
    assert np.array_equal(pool, kv8.ref_append(c.pool, x, x[::-1], c.bt, c.lens, fmt, offsets))


# The large channel, the size of the others (2: multiples of 1/64) and of K. Below 64 the int8 scores' four digits reach
# to the last bit of fp16; 30 bits from a larger value down to 2^-14 (60000, 65504), 2^-16 (16000) or 2^-21 (300).
OUTLIERS = [(60000, 2.0, 1), (16000, 2.0, 1), (40, 1.0, 1), (63.97, 1.0, 1), (64, 1.0, 1), (60000, 0.01, 100), (300, 1e-4, 2000),
            (-65504, 1.0, 1), (6e-5, 3e-7, 30000), (60000, 0, 1)]


def outlier_case(fmt, large, small, k_size):
    c = Cache([31, 1, 0, 32, 17], 2, fmt, seed=14)
    q = outlier_queries(c, 8, large, small)
    kv8.views(c.pool)[2][:] *= k_size
    if small == 2.0:  # no values that end below the unit of the digits
        q[..., 6:] = np.rint(q[..., 6:].astype(np.float64) * 64) / 64
        q[..., :5] = np.rint(q[..., :5].astype(np.float64) * 64) / 64
    return c, q


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("large,small,k_size", OUTLIERS)
def test_one_large_query_channel(exe, fmt, large, small, k_size):
    c, q = outlier_case(fmt, large, small, k_size)
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=8, sm_scale=0.09)
    assert (st, bits) == (0, 0)
    assert_fine(out, q, c.pool, c.bt, c.lens, fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq", range(2, 17, 2))
def test_values_that_cancel(exe, fmt, hq):
    """Weights keep fp32's bits on their way to the values."""
    c, q = opposed_values(40, hq, fmt)
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=hq, sm_scale=0.09)
    assert (st, bits) == (0, 0)
    assert_fine(out, q, c.pool, c.bt, c.lens, fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("units", [1, 3, 40])
def test_rows_that_share_pages(exe, fmt, units):
    """Attention and read-back over a shared prefix; each row's new token goes to a page of its own."""
    c, r = shared_prefix(fmt), np.random.default_rng(2)
    k, v = (r.standard_normal((5, 256)).astype(np.float16) for _ in "kv")
    write = np.array([700, 640, 593, 0, 0])
    (st, bits, _, pool), = call(exe, "append", c, lens=write, k=k, v=v, tokens=5, compute_units=units)
    assert (st, bits) == (0, 0)
    assert np.array_equal(pool, kv8.ref_append(c.pool, k.reshape(5, 2, 128), v.reshape(5, 2, 128), c.bt, write, fmt))
    c.pool = pool
    q = r.standard_normal((5, 8, 128)).astype(np.float16)
    (st, bits, left, out), = call(exe, "decode", c, q=q, hq=8, sm_scale=0.09, compute_units=units)
    assert (st, bits, left) == (0, 0, 0)
    assert_decode(out, q, c.pool, c.bt, c.lens, fmt, 0.09)
    offs = np.concatenate([[0], np.cumsum(c.lens)])
    n = int(offs[-1])
    (st, bits, _, (ko, _)), = call(exe, "gather", c, k=np.zeros((n, 256), dtype=np.float16), v=np.zeros((n, 256), dtype=np.float16),
                                   offsets=offs, tokens=n, compute_units=units)
    assert (st, bits) == (0, 0)
    for i in range(5):
        assert np.array_equal(ko.reshape(n, 2, 128)[offs[i]:offs[i + 1]], gathered(c.pool, c.bt[i], 0, c.lens[i], fmt)[0])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_query_that_is_not_finite_reaches_its_head_only(exe, fmt, bad):
    c, q = outlier_case(fmt, 300, 1.0, 1)
    q[:, 2, 77] = bad
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=8, sm_scale=0.09)
    live = c.lens > 0
    assert (st, bits) == (0, 0) and np.isnan(out[live, 2]).all() and not out[~live].any()
    keep = [h for h in range(8) if h != 2]
    q[:, 2, 77] = 0
    want = call(exe, "decode", c, q=q, hq=8, sm_scale=0.09)[0][3]
    assert np.array_equal(out[:, keep], want[:, keep])


def some_heads_large(fmt, g):
    """One head with a large channel, one with values just below 64, the others ordinary."""
    c = Cache([31, 1, 0, 32, 17], 2, fmt, seed=15)
    q = outlier_queries(c, 2 * g, 1.0, 1.0)
    q[:, 0, 5] = 1000
    q[:, 0, 9] = 2.0 ** -13 + 2.0 ** -23
    q[:, -1, 5] = 63.96875
    return c, q


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g", range(1, 9))
def test_a_large_channel_of_one_head(exe, fmt, g):
    c, q = some_heads_large(fmt, g)
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=2 * g, sm_scale=0.09)
    assert (st, bits) == (0, 0)
    assert_fine(out, q, c.pool, c.bt, c.lens, fmt, 0.09)
