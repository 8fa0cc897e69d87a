"""One workspace for batches of several sizes, and merges of many workgroups' states, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2606_26666_amd as pkv
from tests.cpu_kv8 import Cache
from tests.test_gpu_kv8 import Device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [pkv.PKV_KV8_INT8, pkv.PKV_KV8_E4M3])
def test_batches_of_several_sizes_share_a_workspace(fmt):
    r = np.random.default_rng(3)
    many = Device(Cache(r.integers(100, 700, 600), 4, fmt, seed=1), 16)
    few = Device(Cache([9000, 0, 400], 4, fmt, seed=2), 16)
    few_heads = Device(Cache([5000], 2, fmt, seed=4), 4)
    want = [d.decode() for d in (many, few, few_heads)]
    for d, w in zip((many, few, few_heads), want):
        d.check(w)
    for _ in range(3):
        for d, w in zip((few, many, few_heads, many), (want[1], want[0], want[2], want[0])):
            out = torch.full_like(w, float("nan"))
            pkv.pkv_kv8_decode(torch.from_numpy(d.q).to("cuda"), d.pool, d.bt, d.lens, 0.09, out, many.bufs.ws, format=fmt)
            assert torch.equal(out, w)
            assert pkv.pkv_check_device_status(many.bufs.ws) == 0
            assert not many.bufs.ws[256:256 + 4 * 600 * 4].any()  # every counter of the largest batch is zero


@pytest.mark.parametrize("hq", [1, 4, 7])
@pytest.mark.parametrize("lens", [[40_000], [70_000], [9_000, 7_000], [33_000, 0, 30_000]])
def test_merges_of_many_workgroups(lens, hq):
    """One KV head: up to 256 workgroups' states for a row."""
    d = Device(Cache(lens, 1, pkv.PKV_KV8_INT8, seed=2), hq)
    out = d.decode()
    d.check(out)
    for _ in range(5):  # whichever workgroup merges
        assert torch.equal(d.decode(), out)
