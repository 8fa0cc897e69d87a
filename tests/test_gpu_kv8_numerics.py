"""Numerics of the 8-bit cache's kernels at their borders, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2606_26666_amd as pkv
from oracle import kv8
from tests.cpu_kv8 import Cache
from tests.kv8_cases import assert_decode, assert_fine, gathered, opposed_values, shared_prefix
from tests.test_cpu_kv8_numerics import FORMATS, OUTLIERS, outlier_case, signed_zeros, some_heads_large

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda")


@pytest.mark.parametrize("fmt", FORMATS)
def test_zeros_of_both_signs(fmt):
    x = signed_zeros()
    for c, offs in ((Cache([8], 2, fmt, filled=False), [0, 8]), (Cache([3] * 8, 2, fmt, filled=False), None)):
        pool, ws = dev(c.pool), pkv.Kv8Buffers(c.B, 2, 2, 128, "cuda").ws
        pkv.pkv_kv8_append(dev(x), dev(x[::-1]), pool, dev(c.bt), dev(c.lens), ws, format=fmt,
                           offsets=None if offs is None else dev(np.array(offs, dtype=np.int32)))
        assert np.array_equal(pool.cpu().numpy(), kv8.ref_append(c.pool, x, x[::-1], c.bt, c.lens, fmt, offs))


def attend(c, q, hq):
    """An attention call over a Cache's arrays: its output on the host."""
    bufs = pkv.Kv8Buffers(c.B, hq, c.hkv, 128, "cuda")
    bufs.partial_region().fill_(0xFF)
    out = torch.full((c.B, hq, 128), float("nan"), dtype=torch.float16, device="cuda")
    pkv.pkv_kv8_decode(dev(q), dev(c.pool), dev(c.bt), dev(c.lens), 0.09, out, bufs.ws, format=c.fmt)
    assert pkv.pkv_check_device_status(bufs.ws) == 0
    return out.cpu().numpy()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("large,small,k_size", OUTLIERS)
def test_one_large_query_channel(fmt, large, small, k_size):
    c, q = outlier_case(fmt, large, small, k_size)
    assert_fine(attend(c, q, 8), q, c.pool, c.bt, c.lens, fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq", [8, 16])
def test_columns_of_a_head_agree(fmt, hq):
    """A weight's parts lie in several columns, each with a score of its own: where two scores differ in the last
    bit, one weight in some 2^15 is off by 2^-8. Here there are 5 weights for each of 4096 rows' heads."""
    c = Cache([5] * 4096, 2, fmt, seed=3)
    q = np.random.default_rng(8).standard_normal((4096, hq, 128)).astype(np.float16)
    assert_decode(attend(c, q, hq), q, c.pool, c.bt, c.lens, fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq", range(2, 17, 2))
def test_values_that_cancel(fmt, hq):
    c, q = opposed_values(400, hq, fmt)
    assert_fine(attend(c, q, hq), q, c.pool, c.bt, c.lens, fmt, 0.09)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq", [2, 8, 16])
def test_rows_that_share_pages(fmt, hq):
    c, r = shared_prefix(fmt), np.random.default_rng(2)
    x = r.standard_normal((5, 4, 128)).astype(np.float16)
    write = np.array([700, 640, 593, 0, 0], dtype=np.int32)
    pool, ws = dev(c.pool), pkv.Kv8Buffers(5, 2, 2, 128, "cuda").ws
    xd = dev(x)
    pkv.pkv_kv8_append(xd[:, :2], xd[:, 2:], pool, dev(c.bt), dev(write), ws, format=fmt)
    c.pool = kv8.ref_append(c.pool, x[:, :2], x[:, 2:], c.bt, write, fmt)
    assert np.array_equal(pool.cpu().numpy(), c.pool)
    q = r.standard_normal((5, hq, 128)).astype(np.float16)
    assert_decode(attend(c, q, hq), q, c.pool, c.bt, c.lens, fmt, 0.09)
    offs = np.concatenate([[0], np.cumsum(c.lens)]).astype(np.int32)
    k, v = (torch.zeros((int(offs[-1]), 2, 128), dtype=torch.float16, device="cuda") for _ in "kv")
    pkv.pkv_kv8_gather(pool, dev(c.bt), dev(c.lens), k, v, ws, format=fmt, offsets=dev(offs))
    for i in range(5):
        for got, want in zip((k, v), gathered(c.pool, c.bt[i], 0, c.lens[i], fmt)):
            assert np.array_equal(got[offs[i]:offs[i + 1]].cpu().numpy(), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_one_token_of_each_row_is_read_back(fmt):
    """Without offsets: each row's last token, and zeros for a row of length 0."""
    c = Cache([1, 0, 16, 17, 30, 4, 700] * 9, 3, fmt, seed=2)
    k, v = (torch.full((c.B, 3, 128), 7.0, dtype=torch.float16, device="cuda") for _ in "kv")
    ws = pkv.Kv8Buffers(c.B, 3, 3, 128, "cuda").ws
    pkv.pkv_kv8_gather(dev(c.pool), dev(c.bt), dev(c.lens), k, v, ws, format=fmt)
    assert pkv.pkv_check_device_status(ws) == 0
    for i, n in enumerate(c.lens.tolist()):
        for got, want in zip((k, v), gathered(c.pool, c.bt[i], n - 1, n, fmt) if n else [np.zeros((1, 3, 128))] * 2):
            assert np.array_equal(got[i].cpu().numpy(), want[0])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_query_that_is_not_finite_reaches_its_head_only(fmt, bad):
    c, q = outlier_case(fmt, 300, 1.0, 1)
    q[:, 2, 77] = bad
    out, live = attend(c, q, 8), c.lens > 0
    assert np.isnan(out[live, 2]).all() and not out[~live].any()
    keep = [h for h in range(8) if h != 2]
    q[:, 2, 77] = 0
    assert np.array_equal(out[:, keep], attend(c, q, 8)[:, keep])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g", range(1, 9))
def test_a_large_channel_of_one_head(fmt, g):
    c, q = some_heads_large(fmt, g)
    assert_fine(attend(c, q, 2 * g), q, c.pool, c.bt, c.lens, fmt, 0.09)
