"""The binding's checks of the 8-bit cache's calls: each thing that can be wrong with a call's tensors is
refused with an error that names it, and nothing that fails the checks gets past them unnamed."""
import types

import pytest
import torch

import paper_2606_26666_amd as pkv
from paper_2606_26666_amd import _binding as b


class Dev(torch.Tensor):
    """A host tensor with a device tensor's looks."""
    is_cuda = True
    on = 0

    def get_device(self):
        return self.on


def dev(shape, dtype=torch.float16, on=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Dev)
    t.on = on
    return t


def transposed(shape, dtype):
    t = dev(shape[:-2] + (shape[-1], shape[-2]), dtype)
    return t.transpose(-1, -2)


def tensors():
    return dict(q=dev((2, 32, 128)), k=dev((2, 8, 128)), v=dev((2, 8, 128)), out=dev((2, 32, 128)), cache=dev((4, 8, 4224), torch.uint8),
                block_table=dev((2, 6), torch.int32), seq_lens=dev((2,), torch.int32), ws=dev((1 << 23,), torch.uint8),
                offsets=dev((3,), torch.int32), stream=None)


def other_stream():
    return types.SimpleNamespace(device_index=1, cuda_stream=0)


CACHE = [("cache", lambda: dev((4, 8, 4096), torch.uint8)), ("cache", lambda: dev((4, 8 * 4224), torch.uint8)),
         ("cache", lambda: dev((4, 8, 4224), torch.int8)), ("cache", lambda: transposed((4, 8, 4224), torch.uint8)),
         ("cache", lambda: dev((4, 8, 4224), torch.uint8, on=1)), ("block_table", lambda: dev((3, 6), torch.int32)),
         ("block_table", lambda: dev((12,), torch.int32)), ("block_table", lambda: dev((2, 6), torch.int64)),
         ("block_table", lambda: transposed((2, 6), torch.int32)), ("block_table", lambda: dev((2, 6), torch.int32, on=1)),
         ("seq_lens", lambda: dev((2, 1), torch.int32)), ("seq_lens", lambda: dev((3,), torch.int32)),
         ("seq_lens", lambda: dev((2,), torch.int64)), ("seq_lens", lambda: dev((4,), torch.int32)[::2]),
         ("seq_lens", lambda: dev((2,), torch.int32, on=1)), ("ws", lambda: dev((1 << 21,), torch.int32)),
         ("ws", lambda: dev((1 << 24,), torch.uint8)[::2]), ("ws", lambda: dev((1 << 23,), torch.uint8, on=1)), ("stream", other_stream)]
MOVE = CACHE + [("cache", lambda: dev((4, 4, 4224), torch.uint8)), ("v", lambda: dev((2, 8, 128), on=1)), ("v", lambda: dev((3, 8, 128))),
                ("offsets", lambda: dev((2,), torch.int32)), ("offsets", lambda: dev((3,), torch.int64)),
                ("offsets", lambda: dev((6,), torch.int32)[::2]), ("offsets", lambda: dev((3,), torch.int32, on=1))]
DECODE = CACHE + [("out", lambda: dev((2, 32, 128), torch.float32)), ("out", lambda: dev((2, 16, 128))),
                  ("out", lambda: transposed((2, 32, 128), torch.float16)), ("out", lambda: dev((2, 32, 128), on=1))]


def call(what, t):
    if what == "decode":
        return pkv.pkv_kv8_decode(t["q"], t["cache"], t["block_table"], t["seq_lens"], 1.0, t["out"], t["ws"], format=0, stream=t["stream"])
    move = {k: t[k] for k in ("k", "v", "cache", "block_table", "seq_lens", "ws", "offsets", "stream")}
    return getattr(pkv, f"pkv_kv8_{what}")(**move, format=0)


@pytest.fixture
def calls(monkeypatch):
    """The C calls that were made, in place of the library."""
    made = []
    lib = types.SimpleNamespace(**{f"pkv_kv8_{w}": lambda *a, w=w: made.append(w) or 0 for w in ("append", "gather", "decode")},
                                pkv_kv8_record_bytes=lambda d: 4224 if d == 128 else 0)
    monkeypatch.setattr(b, "lib", lambda: lib)
    monkeypatch.setattr(b, "_device_index", lambda: 0)
    monkeypatch.setattr(b, "_stream", lambda s: 0)
    return made


@pytest.mark.parametrize("what", ["append", "gather", "decode"])
def test_a_sound_call_is_made(calls, what):
    call(what, tensors())
    call(what, {**tensors(), "stream": types.SimpleNamespace(device_index=0)})
    if what != "decode":
        call(what, {**tensors(), "offsets": None})
    assert set(calls) == {what}


@pytest.mark.parametrize("what", ["append", "gather", "decode"])
@pytest.mark.parametrize("named", [True, False])
def test_what_does_not_fit_is_refused(calls, monkeypatch, what, named):
    """named: with the errors that say what is wrong; else without them, as for a condition that they lack."""
    if not named:
        for f in ("_explain_cache", "_explain_offsets", "_one_device", "_dev"):
            monkeypatch.setattr(b, f, lambda *a, **kw: None)
    for i, (name, make) in enumerate(DECODE if what == "decode" else MOVE):
        with pytest.raises((TypeError, ValueError)) as e:
            call(what, {**tensors(), name: make()})
        if named:
            assert name in str(e.value) or "device" in str(e.value) or "k and v" in str(e.value), (i, name, str(e.value))
    assert calls == []
