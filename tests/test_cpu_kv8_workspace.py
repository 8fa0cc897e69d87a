"""One workspace for batches of several sizes, and merges of many workgroups' states: the 8-bit cache's
attention kernel on the CPU, its workgroups in an order that the test chooses."""
import numpy as np
import pytest

from oracle import kv8
from tests import cpu_kv8
from tests.cpu_cases import compiler
from tests.cpu_kv8 import Cache, call
from tests.kv8_cases import assert_decode

pytestmark = pytest.mark.skipif(compiler() is None, reason="needs clang")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return cpu_kv8.build(str(tmp_path_factory.mktemp("cpu_kv8")))


@pytest.mark.parametrize("hq", [2, 8, 16])
@pytest.mark.parametrize("rows", [3, 33, 200, 4096])
def test_a_workspace_of_more_rows_keeps_its_counters(exe, hq, rows):
    c = Cache([1100, 0, 900], 2, kv8.INT8, seed=5)
    q = np.random.default_rng(1).standard_normal((3, hq, 128)).astype(np.float16)
    for st, bits, left, out in call(exe, "decode", c, q=q, hq=hq, calls=2, sm_scale=0.09, compute_units=3, workspace_rows=rows):
        assert (st, bits, left) == (0, 0, 0)
        assert_decode(out, q, c.pool, c.bt, c.lens, c.fmt, 0.09)


def merged(exe, c, hq, **kw):
    q = np.random.default_rng(1).standard_normal((c.B, hq, 128)).astype(np.float16)
    (st, bits, left, out), = call(exe, "decode", c, q=q, hq=hq, sm_scale=0.09, **kw)
    assert (st, bits, left) == (0, 0, 0)
    return q, out


def boundary(lens, units):
    """The workgroup with both the end of the first row and the start of the second (one KV head)."""
    pairs = [-(-n // 32) + 1 for n in lens]
    waves = min(8 * units, sum(pairs))
    q, r = divmod(sum(pairs), waves)
    begins = [w * q + min(w, r) for w in range(waves)]
    return max(w for w in range(waves) if begins[w] <= pairs[0] - 2) // 8


@pytest.mark.parametrize("fmt", [kv8.INT8, kv8.E4M3])
@pytest.mark.parametrize("hq", range(1, 9))
def test_a_workgroup_that_brings_the_last_state_of_two_rows(exe, hq, fmt):
    """Two rows over 60 workgroups; the one with the end of the first and the start of the second comes last and
    merges both. The sums are formed in the same order as when others merge: the results are the same bits."""
    lens = [9000, 7000]
    c = Cache(lens, 1, fmt, seed=2)
    q, out = merged(exe, c, hq, compute_units=60, last_workgroup=boundary(lens, 60))
    assert_decode(out, q, c.pool, c.bt, c.lens, fmt, 0.09)
    assert np.array_equal(merged(exe, c, hq, compute_units=60)[1], out)


@pytest.mark.parametrize("hq", [1, 4, 7])
def test_a_row_over_more_workgroups_than_a_wave_has_lanes(exe, hq):
    """30000 tokens of one KV head, a pair or two a wave: 118 workgroups' states, the first's brought last."""
    c = Cache([30000], 1, kv8.INT8, seed=2)
    q, out = merged(exe, c, hq, compute_units=256, last_workgroup=0)
    assert_decode(out, q, c.pool, c.bt, c.lens, kv8.INT8, 0.09)
