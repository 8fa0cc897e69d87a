"""Numerics of the 8-bit cache's kernels at their borders, their own sources on the CPU: zeros of both
signs, queries of many sizes and values that cancel."""
import numpy as np
import pytest

from oracle import kv8
from tests import cpu_kv8
from tests.cpu_cases import compiler
from tests.cpu_kv8 import Cache, call

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
