"""A step over some of the admitted slots, for each way the cache is held: the other slots keep every
byte of their pages and their lengths. The device calls are stand-ins on host tensors."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2606_26666_amd import serving

HKV, MAXP = 2, 3


class Event:
    def __init__(self, enable_timing):
        pass

    def record(self):
        pass

    def elapsed_time(self, other):
        return 0.0


def engine(monkeypatch, kv):
    """Four slots, three pages each; the calls' work is the oracle's."""
    e = object.__new__(serving.Engine)
    e.torch, e.dev, e.B, e.hq, e.hkv, e.d, e.maxp, e.mlp = torch, torch.device("cpu"), 4, 4, HKV, 128, MAXP, None
    e.kv, e.format = kv, serving.KV_FORMATS[kv]
    e.gen = torch.Generator().manual_seed(5)
    e.bt_host = np.zeros((4, MAXP), dtype=np.int32)
    e.bt, e.lens = torch.zeros((4, MAXP), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    e.lens_host = np.zeros(4, dtype=np.int32)
    e.q, e.out = (torch.zeros((4, 4, 128), dtype=torch.float16) for _ in "qo")
    e.fixed_target, e.params = 256, None
    e.bufs = type("Bufs", (), dict.fromkeys(("ws", "tasks", "split_offsets", "num_tasks")))
    r = np.random.default_rng(1)
    if e.format is None:
        e.k, e.v = (torch.from_numpy(r.standard_normal((12, 16, HKV, 128)).astype(np.float16)) for _ in "kv")
    else:
        e.cache = torch.from_numpy(r.integers(0, 100, (12, HKV, kv8.RECORD)).astype(np.uint8))
    e.attended = []

    def append(k, v, cache, block_table, seq_lens, ws, *, format):
        cache.copy_(torch.from_numpy(kv8.ref_append(cache.numpy(), k.numpy(), v.numpy(), block_table.numpy(), seq_lens.numpy(), format)))

    monkeypatch.setattr(serving._b, "pkv_kv8_append", append)
    monkeypatch.setattr(serving._b, "pkv_kv8_decode", lambda q, cache, bt, lens, *a, **kw: e.attended.append(lens.tolist()))
    monkeypatch.setattr(serving._b, "pkv_plan_decode", lambda q, k, v, bt, lens, *a: e.attended.append(lens.tolist()))
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    return e


def slots(e):
    """Bytes of each slot's three pages: [4, 3, ...]."""
    if e.format is None:
        return torch.stack((e.k, e.v), 1).view(4, MAXP, -1).clone()
    return e.cache.view(4, MAXP, -1).clone()


@pytest.mark.parametrize("kv", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("active", [[0], [1, 3], [3], [2, 0], [0, 1, 3], [], [-1]])
def test_a_step_leaves_the_other_slots_as_they_are(monkeypatch, kv, active):
    e = engine(monkeypatch, kv)
    lens = [20, 16, 0, 33]  # slot 2 is free; 16: the next token begins a page
    for s, n in enumerate(lens):
        if n or 2 in active:
            e.admit(s, [3 * s, 3 * s + 1, 3 * s + 2], n)
    before = slots(e)
    e.step(active)
    stepped = [s % 4 for s in active]
    assert e.attended == [[n + (s in stepped) for s, n in enumerate(lens)]]
    after = slots(e)
    for s in range(4):
        changed = [p for p in range(MAXP) if not torch.equal(before[s, p], after[s, p])]
        assert changed == ([lens[s] // 16] if s in stepped else []), s


@pytest.mark.gpu
@pytest.mark.parametrize("kv", ["fp16", "int8", "e4m3"])
def test_a_step_of_some_slots_on_the_gpu(kv):
    e = serving.Engine(4, MAXP, 12, hq=4, hkv=HKV, kv=kv, seed=2)
    lens = [20, 16, 0, 33]
    for s in (0, 1, 3):
        e.admit(s, [3 * s, 3 * s + 1, 3 * s + 2], lens[s])
    for active in ([0], [1, 3], [], [3, 0], [0, 1, 3]):
        before = slots(e)
        e.step(active)
        after = slots(e)
        for s in range(4):
            changed = [p for p in range(MAXP) if not torch.equal(before[s, p], after[s, p])]
            assert changed == ([lens[s] // 16] if s in active else []), (active, s)
            lens[s] += s in active
    assert e.lens.tolist() == lens
