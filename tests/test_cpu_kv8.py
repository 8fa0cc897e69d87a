"""The 8-bit cache's kernels, their own sources, on the CPU (tests/cpu_device): every access bounds
checked, under schedules that let one wave run ahead of the others as far as the barriers allow."""
import numpy as np
import pytest

from oracle import kv8
from tests import cpu_kv8
from tests.cpu_cases import ASCENDING, DESCENDING, compiler
from tests.cpu_kv8 import Cache, call
from tests.kv8_cases import assert_decode, gathered

SCHEDULES = [ASCENDING, DESCENDING, 12345]
FORMATS = [kv8.INT8, kv8.E4M3]
SEQ_LEN, PAGE_ID = 1, 2

pytestmark = pytest.mark.skipif(compiler() is None, reason="needs clang")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return cpu_kv8.build(str(tmp_path_factory.mktemp("cpu_kv8")))


def queries(cache, hq, seed=1):
    return np.random.default_rng(seed).standard_normal((cache.B, hq, 128)).astype(np.float16)


def attend(exe, cache, hq, **kw):
    q = queries(cache, hq)
    for st, bits, left, out in call(exe, "decode", cache, q=q, hq=hq, calls=2, sm_scale=0.09, **kw):
        assert (st, bits, left) == (0, 0, 0)
        assert_decode(out, q, cache.pool, cache.bt, cache.lens, cache.fmt, 0.09)
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv", [(2, 2), (2, 1), (3, 1), (8, 2), (5, 1), (6, 1), (14, 2), (8, 1)])
def test_heads(exe, hq, hkv, fmt):
    """Rows inside one wave, over waves of one workgroup and over workgroups; empty ones between."""
    attend(exe, Cache([77, 0, 1, 16, 33, 300, 0, 15], hkv, fmt, seed=hq), hq, compute_units=3)


@pytest.mark.parametrize("order", SCHEDULES)
@pytest.mark.parametrize("lens,cus", [([1000], 3), ([1] * 40, 2), ([0, 0, 5, 0], 2), ([2100], 1), ([600, 31, 32, 64, 65, 2], 2),
                                      ([0], 1), ([32] * 9 + [500], 4), ([40, 0, 100, 250, 7, 0, 33, 64] * 3, 2),
                                      ([500, 30, 512, 0, 60] * 4, 1), ([1100, 0, 900], 3), ([1024, 10], 5),
                                      ([500, 0, 33], 3), ([250, 1, 0, 100, 256], 3), ([70, 0, 65, 33, 7], 3), ([300, 100, 0], 2)])
def test_lengths_and_schedules(exe, lens, cus, order):
    attend(exe, Cache(lens, 2, kv8.INT8, seed=5), 8, compute_units=cus, order=order)


def test_more_rows_than_threads(exe):
    lens = np.random.default_rng(3).integers(0, 40, 700)
    attend(exe, Cache(lens, 1, kv8.E4M3, seed=4), 1, compute_units=2)


def test_results_do_not_depend_on_the_schedule(exe):
    c = Cache([300, 900, 17], 2, kv8.E4M3, seed=6)
    outs = [attend(exe, c, 4, compute_units=3, order=o) for o in SCHEDULES]
    assert all(np.array_equal(o.view(np.uint16), outs[0].view(np.uint16)) for o in outs)


def test_strided_queries(exe):
    c, hq = Cache([100, 3, 50], 2, kv8.INT8), 4
    q = np.random.default_rng(2).standard_normal((3, 1024)).astype(np.float16)
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=hq, strides=(1024,), sm_scale=0.09)
    assert (st, bits) == (0, 0)
    assert_decode(out, q[:, :512].reshape(3, hq, 128), c.pool, c.bt, c.lens, c.fmt, 0.09)


@pytest.mark.parametrize("page", [0, 2, 9, 18])
def test_a_page_outside_the_pool_zeroes_its_row_only(exe, page):
    c = Cache([300, 200], 2, kv8.INT8, seed=8)
    for wrong in (-1, c.num_pages, 2 ** 31 - 1):
        bt = c.bt.copy()
        bt[0, page] = wrong
        q = queries(c, 4)
        for st, bits, left, out in call(exe, "decode", c, bt=bt, q=q, hq=4, calls=2, sm_scale=0.09, compute_units=3):
            assert (st, bits, left) == (0, PAGE_ID, 0) and not out[0].any()
            assert_decode(out[1:], q[1:], c.pool, c.bt[1:], c.lens[1:], c.fmt, 0.09)


def test_a_length_outside_the_table_zeroes_its_row_only(exe):
    c = Cache([300, 200, 10], 1, kv8.E4M3, seed=9)
    for wrong in (-1, c.bt.shape[1] * 16 + 1, 2 ** 31 - 1, -2 ** 31):
        lens = c.lens.copy()
        lens[1] = wrong
        q = queries(c, 4)
        (st, bits, left, out), = call(exe, "decode", c, lens=lens, q=q, hq=4, sm_scale=0.09)
        assert (st, bits, left) == (0, SEQ_LEN, 0) and not out[1].any()
        keep = [0, 2]
        assert_decode(out[keep], q[keep], c.pool, c.bt[keep], c.lens[keep], c.fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_scales_reach_their_row_only(exe, fmt):
    c = Cache([300, 200], 2, fmt, seed=10)
    at = c.pool[c.bt[0, 3], 1]
    at[4096 + 64 + 4 * 5:4096 + 64 + 4 * 6] = np.frombuffer(np.float32(np.nan).tobytes(), dtype=np.uint8)
    q = queries(c, 4)
    (st, bits, _, out), = call(exe, "decode", c, q=q, hq=4, sm_scale=0.09)
    assert (st, bits) == (0, 0) and np.isnan(out[0, 2:]).all() and np.isfinite(out[0, :2]).all() and np.isfinite(out[1]).all()


def moved(seed, tokens, hkv, stride):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((tokens, stride)) * 2.0 ** r.integers(-12, 8, (tokens, 1))).astype(np.float16)
    return x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("order", SCHEDULES)
def test_append_and_gather_chunks(exe, fmt, order):
    """Chunks that begin and end inside groups of four and pages; rows without new tokens; tokens
    behind the last row's, which are not touched."""
    lens, new = [40, 5, 17, 64, 3, 0, 33], [30, 0, 17, 1, 3, 0, 6]
    c = Cache(lens, 3, fmt, seed=1)
    offs = np.concatenate([[0], np.cumsum(new)])
    n, extra = int(offs[-1]), 3
    k, v = moved(2, n + extra, 3, 400), moved(3, n + extra, 3, 512)
    k[4, 130] = np.inf
    v[7, 5] = np.nan
    k[9, :128] = 0
    args = dict(offsets=offs, tokens=n + extra, strides=(400, 512), order=order)
    (st, bits, _, pool), = call(exe, "append", c, k=k, v=v, **args)
    assert (st, bits) == (0, 0)
    ref = kv8.ref_append(c.pool, k[:, :384].reshape(-1, 3, 128), v[:, :384].reshape(-1, 3, 128), c.bt, c.lens, fmt, offs)
    assert np.array_equal(pool, ref)
    c.pool = pool
    (st, bits, _, (ko, vo)), = call(exe, "gather", c, k=np.full_like(k, 7), v=np.full_like(v, 7), **args)
    assert (st, bits) == (0, 0)
    for got, stride, which in ((ko, 400, 0), (vo, 512, 1)):
        whole = np.full((n + extra) * stride, 7, dtype=np.float16)
        whole[:got.size] = got
        whole = whole.reshape(n + extra, stride)
        assert np.all(whole[:, 384:] == 7) and np.all(whole[n:] == 7)
        for i in range(len(lens)):
            want = gathered(pool, c.bt[i], lens[i] - new[i], lens[i], fmt)[which] if new[i] else np.zeros((0, 3, 128))
            assert np.array_equal(whole[offs[i]:offs[i + 1], :384].reshape(-1, 3, 128), want, equal_nan=True), i


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_and_gather_one_token_per_row(exe, fmt):
    c = Cache([1, 0, 16, 17, 30, 4], 2, fmt, seed=2)
    k, v = moved(4, 6, 2, 256), moved(5, 6, 2, 256)
    (st, bits, _, pool), = call(exe, "append", c, k=k, v=v, tokens=6)
    assert (st, bits) == (0, 0)
    assert np.array_equal(pool, kv8.ref_append(c.pool, k.reshape(6, 2, 128), v.reshape(6, 2, 128), c.bt, c.lens, fmt))
    c.pool = pool
    (st, bits, _, out), = call(exe, "gather", c, k=np.full_like(k, 7), v=np.full_like(v, 7), tokens=6)
    assert (st, bits) == (0, 0)
    for got, which in zip(out, (0, 1)):
        for i, n in enumerate(c.lens):
            want = gathered(pool, c.bt[i], n - 1, n, fmt)[which][0] if n else np.zeros((2, 128))
            assert np.array_equal(got.reshape(6, 2, 128)[i], want)


@pytest.mark.parametrize("what", ["append", "gather"])
def test_bad_rows_of_a_move_are_flagged_and_left(exe, what):
    c = Cache([40, 20, 30], 2, kv8.INT8, seed=3)
    offs, n = np.array([0, 10, 20, 30]), 30
    k, v = moved(6, n, 2, 256), moved(7, n, 2, 256)
    good = kv8.ref_append(c.pool, k.reshape(n, 2, 128), v.reshape(n, 2, 128), c.bt, c.lens, c.fmt, offs)

    def check(bits_wanted, touched, **kw):
        (st, bits, _, got), = call(exe, what, c, k=k, v=v, **{"offsets": offs, "tokens": n, **kw})
        assert (st, bits) == (0, bits_wanted)
        if what == "append":
            for i in range(3):
                pages = c.bt[i, :3][c.bt[i, :3] >= 0]
                assert np.array_equal(got[pages], (good if i in touched else c.pool)[pages]), i
        else:
            for i in range(3):
                rows = got[0].reshape(n, 2, 128)[10 * i:10 * i + 10]
                want = gathered(c.pool, c.bt[i], c.lens[i] - 10, c.lens[i], c.fmt)[0] if i in touched else 0
                assert np.all(rows == want), i

    check(0, (0, 1, 2))
    for wrong in (9, -1, c.bt.shape[1] * 16 + 1, -2 ** 31):
        check(SEQ_LEN, (0, 2), lens=[40, wrong, 30])
    for wrong in (-1, c.num_pages):
        bt = c.bt.copy()
        bt[1, :2] = wrong
        check(PAGE_ID, (0, 2), bt=bt)


@pytest.mark.parametrize("what", ["append", "gather"])
@pytest.mark.parametrize("offs", [[0, 20, 10, 30], [-5, 0, 0, 30], [0, 2 ** 31 - 1, 5, 30], [30, 20, 10, 0], [0, 0, 0, -1],
                                  [5, 10, 20, 2 ** 31 - 1], [-2 ** 31, -1, 40, 30]])
def test_offsets_that_do_not_ascend_stay_in_bounds(exe, what, offs):
    c = Cache([40, 20, 30], 2, kv8.E4M3, seed=3)
    k, v = moved(6, 30, 2, 256), moved(7, 30, 2, 256)
    (st, _, _, _), = call(exe, what, c, k=k, v=v, offsets=offs, tokens=30)
    assert st == 0


def test_append_then_attend_over_steps(exe):
    """A prompt in two chunks, then single tokens, as a serving loop calls them."""
    fmt = kv8.INT8
    c = Cache([50, 7], 2, fmt, filled=False, spare=2)
    r = np.random.default_rng(11)
    for lens, new in (([20, 7], [20, 7]), ([47, 7], [27, 0]), ([48, 8], None), ([49, 9], None)):
        n = 2 if new is None else sum(new)
        k, v = (r.standard_normal((n, 256)).astype(np.float16) for _ in "kv")
        offs = None if new is None else np.concatenate([[0], np.cumsum(new)])
        c.lens = np.array(lens, dtype=np.int32)
        (st, bits, _, pool), = call(exe, "append", c, k=k, v=v, offsets=offs, tokens=n)
        assert (st, bits) == (0, 0)
        c.pool = pool
        attend(exe, c, 8, compute_units=2)
