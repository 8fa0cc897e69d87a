"""The 8-bit cache's entry points refuse bad arguments on the host, before anything is enqueued (no
GPU: every call below fails validation), and the binding refuses tensors that do not fit."""
import types

import pytest
import torch

import paper_2606_26666_amd as pkv
from paper_2606_26666_amd import _binding as b

FAKE = 4096  # a non-null, 16-byte-aligned address that is never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = pkv.PKV_ERR_INVALID_ARG, pkv.PKV_ERR_UNSUPPORTED, pkv.PKV_ERR_WORKSPACE


def test_sizes():
    assert pkv.pkv_kv8_record_bytes(128) == 2 * 2048 + 2 * 64
    assert pkv.pkv_kv8_record_bytes(64) == 0
    assert pkv.pkv_kv8_workspace_size(8, 32, 8, 128) == 256 + 256 + 1024 * 2080
    assert pkv.pkv_kv8_workspace_size(1, 5, 1, 128) == 512 + 1024 * (5 * 128 + 12) * 4
    for bad in ((0, 32, 8, 128), (1, 30, 8, 128), (1, 72, 8, 128), (1, 32, 8, 64), (1, 32, 0, 128), (1 << 20, 1 << 12, 1 << 12, 128)):
        assert pkv.pkv_kv8_workspace_size(*bad) == 0, bad


def decode(**kw):
    a = dict(q=FAKE, qs=4096, cache=FAKE, pages=10, bt=FAKE, maxp=10, lens=FAKE, B=2, hq=32, hkv=8, d=128, fmt=0, scale=1.0,
             out=FAKE, ws=FAKE, n=1 << 30)
    a.update(kw)
    return b.lib().pkv_kv8_decode(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(q=FAKE + 8), INVALID), (dict(qs=4088), INVALID), (dict(qs=4100), INVALID),
    (dict(cache=None), INVALID), (dict(cache=FAKE + 8), INVALID), (dict(pages=0), INVALID), (dict(bt=None), INVALID),
    (dict(bt=FAKE + 2), INVALID), (dict(maxp=0), INVALID), (dict(maxp=1 << 28), INVALID), (dict(lens=None), INVALID),
    (dict(B=0), INVALID), (dict(hq=33), INVALID), (dict(hkv=0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(out=None), INVALID), (dict(out=FAKE + 4), INVALID), (dict(ws=None), INVALID),
    (dict(ws=FAKE + 8), INVALID), (dict(d=64), UNSUPPORTED), (dict(fmt=2), UNSUPPORTED), (dict(fmt=-1), UNSUPPORTED),
    (dict(hq=72, qs=9216), UNSUPPORTED), (dict(B=4097), UNSUPPORTED), (dict(B=4096, maxp=1 << 20), UNSUPPORTED),
    (dict(n=1024), WORKSPACE), (dict(n=256 + 256 + 1024 * 2080 - 1), WORKSPACE)])
def test_decode_refusals(kw, status):
    assert decode(**kw) == status


def move(what, **kw):
    a = dict(k=FAKE, v=FAKE, ks=1024, vs=1024, off=FAKE, tokens=5, cache=FAKE, pages=10, bt=FAKE, maxp=10, lens=FAKE, B=2, hkv=8,
             d=128, fmt=1, ws=FAKE, n=1 << 20)
    a.update(kw)
    if what == "append":
        return b.lib().pkv_kv8_append(*a.values(), None)
    order = ("cache", "pages", "bt", "maxp", "lens", "off", "tokens", "B", "hkv", "d", "fmt", "k", "v", "ks", "vs", "ws", "n")
    return b.lib().pkv_kv8_gather(*(a[x] for x in order), None)


@pytest.mark.parametrize("what", ["append", "gather"])
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=FAKE + 2), INVALID), (dict(ks=1016), INVALID),
    (dict(vs=1028), INVALID), (dict(tokens=-1), INVALID), (dict(off=None), INVALID), (dict(off=FAKE + 1), INVALID),
    (dict(cache=None), INVALID), (dict(cache=FAKE + 4), INVALID), (dict(bt=None), INVALID), (dict(lens=None), INVALID),
    (dict(lens=FAKE + 2), INVALID), (dict(B=0), INVALID), (dict(hkv=0), INVALID), (dict(pages=0), INVALID), (dict(maxp=0), INVALID),
    (dict(ws=None), INVALID), (dict(d=96), UNSUPPORTED), (dict(fmt=7), UNSUPPORTED), (dict(n=255), WORKSPACE)])
def test_move_refusals(what, kw, status):
    assert move(what, **kw) == status


def test_no_tokens_is_no_work():
    for what in ("append", "gather"):
        assert move(what, tokens=0) == 0 and move(what, tokens=0, k=None, v=None) == 0


def test_binding_refuses_host_tensors_types_and_shapes():
    cpu = torch.zeros((2, 8, 128), dtype=torch.float16)
    with pytest.raises(TypeError, match="device tensor"):
        b._rows(cpu, "k")

    def dev(shape, dtype=torch.float16, stride=None, device=0):  # a device tensor's looks
        t = torch.empty(shape, dtype=dtype) if stride is None else torch.empty_strided(shape, stride, dtype=dtype)

        class Fake(torch.Tensor):
            is_cuda = True
        return t.as_subclass(Fake)

    with pytest.raises(TypeError, match="float16"):
        b._rows(dev((2, 8, 128), torch.bfloat16), "k")
    with pytest.raises(ValueError, match="contiguous"):
        b._rows(dev((2, 8, 128), stride=(1024, 1, 8)), "k")
    with pytest.raises(ValueError, match="tokens"):
        b._rows(dev((8, 128)), "k")
    assert b._rows(dev((2, 8, 128), stride=(6144, 128, 1)), "k") == 6144
    assert b._rows(dev((1, 8, 128), stride=(8, 128, 1)), "k") == 1024   # one token: its stride says nothing
    assert b._rows(dev((3, 1, 128), stride=(512, 5, 1)), "k") == 512    # one head: likewise
    pool, ws = dev((4, 8, 4224), torch.uint8), dev((512,), torch.uint8)
    table, lens = dev((2, 8), torch.int32), dev((2,), torch.int32)
    b._explain_cache(pool, table, lens, ws, 128, 8)
    for args, match in (((dev((4, 8, 4096), torch.uint8), table, lens, ws, 128), "cache"), ((pool, table, lens, ws, 64), "cache"),
                        ((pool, table, lens, ws, 128, 4), "KV heads"), ((pool, dev((3, 8), torch.int32), lens, ws, 128), "block_table"),
                        ((pool, table, dev((2, 1), torch.int32), ws, 128), "block_table")):
        with pytest.raises(ValueError, match=match):
            b._explain_cache(*args)
    with pytest.raises(TypeError, match="seq_lens"):
        b._explain_cache(pool, table, dev((2,), torch.int64), ws, 128)
    with pytest.raises(ValueError, match="offsets"):
        b._explain_offsets(dev((2,), torch.int32), 2)
    with pytest.raises(ValueError, match="bad sizes"):
        pkv.Kv8Buffers(1, 72, 8, 128, "cpu")
    with pytest.raises(ValueError, match="not supported"):
        pkv.kv8_pool(1, 8, 64, "cpu")


def test_binding_refuses_tensors_of_several_devices(monkeypatch):
    def on(i):
        return types.SimpleNamespace(get_device=lambda: i)
    monkeypatch.setattr(b, "_device_index", lambda: 0)
    b._one_device(None, q=on(0), ws=on(0), offsets=None)
    b._one_device(types.SimpleNamespace(device_index=0), q=on(0))
    b._one_device(12345, q=on(0))                         # a raw handle says nothing
    with pytest.raises(ValueError, match="stream"):
        b._one_device(types.SimpleNamespace(device_index=1), q=on(0))
    with pytest.raises(ValueError, match="current device"):
        b._one_device(object(), q=on(1))
    with pytest.raises(ValueError, match="ws"):
        b._one_device(None, q=on(0), ws=on(1))
    with pytest.raises(ValueError, match="current device"):
        b._one_device(None, q=on(1))


def test_serving_names_its_formats():
    from paper_2606_26666_amd.serving import KV_FORMATS, Engine
    assert KV_FORMATS == {"fp16": None, "int8": pkv.PKV_KV8_INT8, "e4m3": pkv.PKV_KV8_E4M3}
    with pytest.raises(ValueError, match="kv must be"):
        Engine(4, 4, 16, kv="int4")


@pytest.mark.parametrize("slots", [[0, 1, 2], [2, 0], [1, 1], [2, 2, 0], [0, 0, 1], [3], [1, 3], [-2, 0], []])
def test_cached_rows_are_the_slots_asked_for(monkeypatch, slots):
    """`Engine.cached` and `snapshot` give each slot asked for, in that order, also the same one twice, an
    empty one and one counted from the end. The read-back is a stand-in that writes 100 * row + position."""
    import numpy as np
    from paper_2606_26666_amd import serving
    lens = np.array([3, 20, 1, 0], dtype=np.int32)
    tables = np.arange(8, dtype=np.int32).reshape(4, 2)

    def gather(cache, block_table, seq_lens, k, v, ws, *, format, offsets):
        assert offsets[0] == 0 and offsets[-1] == k.shape[0] and int(seq_lens.sum()) == k.shape[0]
        for row in range(4):
            for t in range(int(offsets[row]), int(offsets[row + 1])):
                pos = int(seq_lens[row]) - (int(offsets[row + 1]) - t)
                k[t] = 100 * row + pos
                v[t] = 100 * row + pos + 0.5

    monkeypatch.setattr(serving._b, "pkv_kv8_gather", gather)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    e = object.__new__(serving.Engine)
    e.torch, e.dev, e.B, e.hq, e.hkv, e.d = torch, torch.device("cpu"), 4, 1, 1, 128
    e.kv, e.format, e.lens_host, e.bt_host, e.bt = "int8", 0, lens, tables, torch.from_numpy(tables)
    e.cache, e.bufs = torch.zeros((8, 1, 1)), type("Bufs", (), {"ws": None})
    e.q = torch.zeros((4, 1, 128), dtype=torch.float16)
    want = [100 * (s % 4) + p for s in slots for p in range(lens[s])]
    k, v = e.cached(slots)
    assert k.shape == v.shape == (len(want), 1, 128)
    assert k[:, 0, 0].tolist() == want and v[:, 0, 127].tolist() == [x + 0.5 for x in want]
    _, pool_k, _, bt, n = e.snapshot(slots)
    assert n.tolist() == [lens[s] for s in slots]
    for i, s in enumerate(slots):
        for p in range(n[i]):
            assert (pool_k[bt[i, p // 16], p % 16] == 100 * (s % 4) + p).all()


def test_cached_refuses_a_slot_that_there_is_not():
    import numpy as np
    from paper_2606_26666_amd import serving
    e = object.__new__(serving.Engine)
    e.torch, e.dev, e.B, e.format, e.lens_host = torch, torch.device("cpu"), 4, 0, np.zeros(4, dtype=np.int32)
    for slots in ([4], [0, -5]):
        with pytest.raises(IndexError):
            e.cached(slots)
