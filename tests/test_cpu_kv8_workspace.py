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
