"""The 8-bit cache on the GPU through the binding, against its fp64 oracle: heads, formats, lengths,
strides, long pools, streams and graphs, and the three calls together."""
import numpy as np
import pytest
import torch

import paper_2606_26666_amd as pkv
from oracle import kv8
from tests.cpu_kv8 import Cache
from tests.kv8_cases import assert_decode, gathered

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMATS = [pkv.PKV_KV8_INT8, pkv.PKV_KV8_E4M3]


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


class Device:
    """A Cache's arrays on the device."""

    def __init__(self, c, hq):
        self.c, self.hq = c, hq
        self.pool, self.bt, self.lens = dev(c.pool), dev(c.bt), dev(c.lens)
        self.bufs = pkv.Kv8Buffers(c.B, hq, c.hkv, 128, DEV)
        self.q = np.random.default_rng(c.B).standard_normal((c.B, hq, 128)).astype(np.float16)

    def decode(self, q=None, bits=0, scale=0.09, bufs=None):
        bufs = bufs or self.bufs
        bufs.partial_region().fill_(0xFF)  # every state slot starts as NaN
        q = dev(self.q) if q is None else q
        out = torch.full((self.c.B, self.hq, 128), float("nan"), dtype=torch.float16, device=DEV)
        pkv.pkv_kv8_decode(q, self.pool, self.bt, self.lens, scale, out, bufs.ws, format=self.c.fmt)
        assert pkv.pkv_check_device_status(bufs.ws) == bits
        assert not bufs.ws[256:256 + 4 * self.c.B * self.c.hkv].any()  # counters back at zero
        return out

    def check(self, out, rows=slice(None), scale=0.09):
        c = self.c
        assert_decode(out.cpu().numpy()[rows], self.q[rows], c.pool, c.bt[rows], c.lens[rows], c.fmt, scale)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g", range(1, 9))
def test_heads(g, fmt):
    d = Device(Cache([77, 0, 1, 16, 33, 700, 0, 15, 32, 2049], 2, fmt, seed=g), 2 * g)
    a = d.decode()
    d.check(a)
    assert torch.equal(d.decode(), a)


@pytest.mark.parametrize("lens,hkv,hq", [([20011], 8, 32), ([1], 8, 32), ([0], 1, 4), ([5] * 300, 2, 8), ([9000, 3, 0, 1200], 4, 32),
                                         ([33] * 7 + [4000], 1, 1), ([2047, 2048, 2049], 3, 18),
                                         ([250, 0, 1, 99] * 70, 8, 32), ([500, 512, 0] * 60, 16, 80), ([1024, 1000, 0, 3], 8, 64),
                                         ([500, 0, 77, 512] * 15, 8, 32), ([250, 0, 1, 99] * 30, 8, 32)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_lengths(lens, hkv, hq, fmt):
    d = Device(Cache(lens, hkv, fmt, seed=3), hq)
    d.check(d.decode())


def test_most_rows():
    lens = np.random.default_rng(4).integers(0, 50, 4096)
    d = Device(Cache(lens, 1, pkv.PKV_KV8_INT8, seed=4), 2)
    d.check(d.decode())
    with pytest.raises(pkv.PkvError, match="unsupported"):
        pkv.pkv_kv8_decode(torch.zeros((4097, 2, 128), dtype=torch.float16, device=DEV), d.pool,
                           torch.zeros((4097, 1), dtype=torch.int32, device=DEV), torch.zeros(4097, dtype=torch.int32, device=DEV),
                           1.0, torch.zeros((4097, 2, 128), dtype=torch.float16, device=DEV), d.bufs.ws, format=0)


def test_strided_queries_and_scale():
    d = Device(Cache([100, 3, 50], 2, pkv.PKV_KV8_INT8), 8)
    x = torch.zeros((3, 12, 128), dtype=torch.float16, device=DEV)
    x[:, :8] = dev(d.q)
    x[:, 8:] = float("nan")
    d.check(d.decode(q=x[:, :8], scale=-0.3), scale=-0.3)


def test_large_scores_keep_the_softmax_in_range():
    d = Device(Cache([500, 40], 2, pkv.PKV_KV8_INT8, seed=2), 8)
    d.q = (d.q.astype(np.float32) * 500).astype(np.float16)
    d.check(d.decode(scale=1.0), scale=1.0)


def test_bad_page_and_bad_length_zero_their_rows():
    d = Device(Cache([3000, 200, 900], 2, pkv.PKV_KV8_E4M3, seed=8), 8)
    for page in (0, 100, 187):
        d.bt = dev(d.c.bt)
        d.bt[0, page] = d.c.num_pages
        out = d.decode(bits=pkv.PKV_DEVERR_PAGE_ID)
        assert not out[0].any()
        d.check(out, [1, 2])
    d.bt = dev(d.c.bt)
    d.lens[1] = d.c.bt.shape[1] * 16 + 1
    out = d.decode(bits=pkv.PKV_DEVERR_SEQ_LEN)
    assert not out[1].any()
    d.check(out, [0, 2])
    d.lens[1] = 200
    d.check(d.decode())


def test_pages_past_four_gib():
    """A pool of 5.4 GB of which the last pages are used: record offsets pass 32 bits."""
    pages, hkv = 160_000, 8
    pool = torch.empty((pages, hkv, 4224), dtype=torch.uint8, device=DEV)
    lens = torch.tensor([70, 33], dtype=torch.int32, device=DEV)
    bt = torch.tensor([[pages - 1, 5, pages - 3, 100_000, pages - 2], [pages - 9, pages - 8, 127_200, 0, 0]], dtype=torch.int32, device=DEV)
    r = np.random.default_rng(5)
    k, v = (r.standard_normal((103, hkv, 128)).astype(np.float16) for _ in "kv")
    offs = torch.tensor([0, 70, 103], dtype=torch.int32, device=DEV)
    bufs = pkv.Kv8Buffers(2, 32, hkv, 128, DEV)
    pkv.pkv_kv8_append(dev(k), dev(v), pool, bt, lens, bufs.ws, format=0, offsets=offs)
    q = r.standard_normal((2, 32, 128)).astype(np.float16)
    out = torch.empty((2, 32, 128), dtype=torch.float16, device=DEV)
    pkv.pkv_kv8_decode(dev(q), pool, bt, lens, 0.09, out, bufs.ws, format=0)
    ko, vo = (torch.zeros((103, hkv, 128), dtype=torch.float16, device=DEV) for _ in "kv")
    pkv.pkv_kv8_gather(pool, bt, lens, ko, vo, bufs.ws, format=0, offsets=offs)
    assert pkv.pkv_check_device_status(bufs.ws) == 0
    small = np.zeros((9, hkv, kv8.RECORD), dtype=np.uint8)
    bt9 = np.array([[0, 1, 2, 3, 4], [5, 6, 7, 8, 8]])
    small = kv8.ref_append(small, k, v, bt9, [70, 33], 0, [0, 70, 103])
    assert_decode(out.cpu().numpy(), q, small, bt9, [70, 33], 0, 0.09)
    for i, (b, e) in enumerate(((0, 70), (70, 103))):
        for got, want in zip((ko, vo), gathered(small, bt9[i], 0, e - b, 0)):
            assert np.array_equal(got[b:e].cpu().numpy(), want)


def chunk(seed, tokens, hkv, heads):
    """k and v as slices of one projection [tokens, heads, 128], with magnitudes of many sizes."""
    r = np.random.default_rng(seed)
    x = (r.standard_normal((tokens, heads, 128)) * 2.0 ** r.integers(-14, 10, (tokens, heads, 1))).astype(np.float16)
    return x, dev(x)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens,new,hkv", [([40, 5, 17, 64, 3, 0, 33], [30, 0, 17, 1, 3, 0, 6], 3), ([2000, 300], [1999, 257], 2),
                                          ([1] * 90, [1] * 90, 1), ([70] * 5, [3, 4, 5, 6, 7], 8), ([1000], [1], 5)])
def test_append_and_gather(lens, new, hkv, fmt):
    c = Cache(lens, hkv, fmt, seed=1)
    pool, bt, n = dev(c.pool), dev(c.bt), sum(new)
    x, xd = chunk(2, n + 5, hkv, 2 * hkv + 1)
    x[n // 2, 1, 7] = np.inf
    x[n // 3, hkv, :] = 0
    xd = dev(x)
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    bufs = pkv.Kv8Buffers(c.B, hkv, hkv, 128, DEV)
    pkv.pkv_kv8_append(xd[:, 1:1 + hkv], xd[:, 1 + hkv:], pool, bt, dev(c.lens), bufs.ws, format=fmt, offsets=dev(offs))
    assert pkv.pkv_check_device_status(bufs.ws) == 0
    c.pool = kv8.ref_append(c.pool, x[:, 1:1 + hkv], x[:, 1 + hkv:], c.bt, c.lens, fmt, offs)
    assert np.array_equal(pool.cpu().numpy(), c.pool)
    back = torch.full((n + 5, 2 * hkv + 2, 128), 7.0, dtype=torch.float16, device=DEV)
    pkv.pkv_kv8_gather(pool, bt, dev(c.lens), back[:, :hkv], back[:, hkv:2 * hkv], bufs.ws, format=fmt, offsets=dev(offs))
    assert pkv.pkv_check_device_status(bufs.ws) == 0
    back = back.cpu().numpy()
    assert np.all(back[n:] == 7) and np.all(back[:, 2 * hkv:] == 7)
    for i in range(c.B):
        if new[i]:
            k, v = gathered(c.pool, c.bt[i], lens[i] - new[i], lens[i], fmt)
            assert np.array_equal(back[offs[i]:offs[i + 1], :hkv], k, equal_nan=True)
            assert np.array_equal(back[offs[i]:offs[i + 1], hkv:2 * hkv], v, equal_nan=True)


def test_intervals_of_a_row_are_read_by_their_end():
    c = Cache([333], 2, pkv.PKV_KV8_INT8, seed=7)
    bufs = pkv.Kv8Buffers(1, 2, 2, 128, DEV)
    for b, e in ((0, 1), (0, 333), (13, 30), (331, 333), (16, 48), (7, 8)):
        k, v = (torch.zeros((e - b, 2, 128), dtype=torch.float16, device=DEV) for _ in "kv")
        pkv.pkv_kv8_gather(dev(c.pool), dev(c.bt), dev(np.array([e], dtype=np.int32)), k, v, bufs.ws, format=c.fmt,
                           offsets=dev(np.array([0, e - b], dtype=np.int32)))
        for got, want in zip((k, v), gathered(c.pool, c.bt[0], b, e, c.fmt)):
            assert np.array_equal(got.cpu().numpy(), want), (b, e)
    assert pkv.pkv_check_device_status(bufs.ws) == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_code_and_every_magnitude_is_quantised_as_in_real_arithmetic(fmt):
    """Vectors whose largest value runs over every fp16 magnitude's leading digits, with all fractions
    of it that could lie near a rounding border."""
    r = np.random.default_rng(9)
    n = 2048
    x = r.integers(0, 0x7C00, (n, 4, 128)).astype(np.uint16).view(np.float16)
    x[:, 0] = (r.integers(-2047, 2048, (n, 128)) * 2.0 ** r.integers(-20, 4, (n, 1))).astype(np.float16)   # one binade: ties
    x[:, 1, 0] = (1024 + np.arange(n) % 1024) * 2.0 ** -5
    x[:, 1, 1:] = x[:, 1, :1] * (r.integers(-254, 255, (n, 127)) / 254)                    # halves of int8 steps
    c = Cache([n], 4, fmt, filled=False)
    bufs = pkv.Kv8Buffers(1, 4, 4, 128, DEV)
    pool = dev(c.pool)
    offs = np.array([0, n], dtype=np.int32)
    pkv.pkv_kv8_append(dev(x), dev(-x), pool, dev(c.bt), dev(c.lens), bufs.ws, format=fmt, offsets=dev(offs))
    assert np.array_equal(pool.cpu().numpy(), kv8.ref_append(c.pool, x, -x, c.bt, c.lens, fmt, offs))


@pytest.mark.parametrize("fmt", FORMATS)
def test_the_three_calls_over_a_rows_life(fmt):
    """A prompt in chunks, then single tokens in a captured graph, then a read-back: as serving does."""
    hq, hkv, cap = 8, 2, 40
    c = Cache([400, 30, 0], hkv, fmt, filled=False, spare=4)
    d = Device(c, hq)
    r = np.random.default_rng(12)

    def new_tokens(n):
        return tuple(r.standard_normal((n, hkv, 128)).astype(np.float16) for _ in "kv")

    for lens, new in (([150, 30, 0], [150, 30, 0]), ([400, 30, 0], [250, 0, 0])):
        k, v = new_tokens(sum(new))
        offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        c.lens = np.array(lens, dtype=np.int32)
        d.lens.copy_(dev(c.lens))
        pkv.pkv_kv8_append(dev(k), dev(v), d.pool, d.bt, d.lens, d.bufs.ws, format=fmt, offsets=dev(offs))
        c.pool = kv8.ref_append(c.pool, k, v, c.bt, c.lens, fmt, offs)
        d.check(d.decode())
    kd, vd = (torch.zeros((3, hkv, 128), dtype=torch.float16, device=DEV) for _ in "kv")
    qd, out = dev(d.q), torch.zeros((3, hq, 128), dtype=torch.float16, device=DEV)
    live = torch.tensor([1, 1, 0], dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        d.lens.add_(live)
        pkv.pkv_kv8_append(kd, vd, d.pool, d.bt, d.lens, d.bufs.ws, format=fmt)
        pkv.pkv_kv8_decode(qd, d.pool, d.bt, d.lens, 0.09, out, d.bufs.ws, format=fmt)
    for step in range(20):
        k, v = new_tokens(3)
        kd.copy_(dev(k))
        vd.copy_(dev(v))
        graph.replay()
        torch.cuda.synchronize()
        c.lens = c.lens + np.array([1, 1, 0], dtype=np.int32)
        c.pool = kv8.ref_append(c.pool, k, v, c.bt, c.lens, fmt)
        if step % 5 == 0 or step == 19:
            assert np.array_equal(d.pool.cpu().numpy(), c.pool)
            d.check(out)
            assert torch.equal(out, d.decode())  # eager on the same state, between the replays
    assert pkv.pkv_check_device_status(d.bufs.ws) == 0


def test_two_streams_with_workspaces_of_their_own():
    a, b = (Device(Cache([4000, 50, 900], 4, f, seed=s), 16) for s, f in ((1, 0), (2, 1)))
    want = a.decode(), b.decode()
    a.check(want[0])
    b.check(want[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(w) for w in want]
    qs = [dev(x.q) for x in (a, b)]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, q, o, st in zip((a, b), qs, outs, streams):
            pkv.pkv_kv8_decode(q, x.pool, x.bt, x.lens, 0.09, o, x.bufs.ws, format=x.c.fmt, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_two_graphs_share_a_workspace():
    c = Cache([3000, 50, 900], 4, 0, seed=1)
    d = Device(c, 16)
    q2 = -dev(d.q)
    want = d.decode(), d.decode(q=q2)
    outs = [torch.zeros_like(w) for w in want]
    q1 = dev(d.q)
    graphs = []
    torch.cuda.synchronize()
    for q, o in zip((q1, q2), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pkv.pkv_kv8_decode(q, d.pool, d.bt, d.lens, 0.09, o, d.bufs.ws, format=0)
        graphs.append(g)
    for _ in range(5):
        for g, o, w in zip(graphs, outs, want):
            o.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w)


def test_refusals():
    d = Device(Cache([10], 2, 0), 4)
    q, out = dev(d.q), torch.zeros((1, 4, 128), dtype=torch.float16, device=DEV)
    call = lambda **kw: pkv.pkv_kv8_decode(**{**dict(q=q, cache=d.pool, block_table=d.bt, seq_lens=d.lens, sm_scale=1.0, out=out,  # noqa: E731
                                                     ws=d.bufs.ws, format=0), **kw})
    call()
    for kw, err in ((dict(q=q.float()), TypeError), (dict(q=q.cpu()), TypeError), (dict(q=q.transpose(1, 2)), ValueError),
                    (dict(cache=d.pool[:, :, :4096].contiguous()), ValueError), (dict(out=out[:, :2]), ValueError),
                    (dict(seq_lens=d.lens.long()), TypeError), (dict(block_table=d.bt.expand(2, -1).contiguous()), ValueError),
                    (dict(ws=d.bufs.ws[:1024]), pkv.PkvError), (dict(format=5), pkv.PkvError),
                    (dict(sm_scale=float("nan")), pkv.PkvError)):
        with pytest.raises(err):
            call(**kw)
    k = torch.zeros((1, 2, 128), dtype=torch.float16, device=DEV)
    for kw, err in ((dict(k=k[:, :1]), ValueError), (dict(v=k.bfloat16()), TypeError), (dict(k=k.repeat(2, 1, 1), v=k.repeat(2, 1, 1)), pkv.PkvError),
                    (dict(offsets=torch.zeros(3, dtype=torch.int32, device=DEV)), ValueError)):
        with pytest.raises(err):
            pkv.pkv_kv8_append(**{**dict(k=k, v=k, cache=d.pool, block_table=d.bt, seq_lens=d.lens, ws=d.bufs.ws, format=0), **kw})


@pytest.mark.parametrize("kv", ["int8", "e4m3"])
def test_serving_over_an_8_bit_cache(kv):
    """Requests come and go; each step appends, attends and (here) reads back, checked against the oracle
    over what is read back: off by its fp16 rounding, half a step of K and V."""
    from oracle import ref_decode
    from paper_2606_26666_amd.serving import PAGE, Engine, PagePool, Scheduler
    from tests.gpu_cases import assert_close
    from workloads.requests import Request
    trace = [Request(0, 0, 300, 3), Request(1, 0, 5000, 6), Request(2, 1, 1200, 2), Request(3, 2, 64, 4), Request(4, 4, 900, 2)]
    maxp = max(-(-(q.prompt_len + q.decode_len) // PAGE) for q in trace)
    engine = Engine(4, maxp, 4 * maxp, mlp=True, seed=7, kv=kv)
    checked = []

    def check(rec):
        slots = rec["slots"]
        out = engine.out.cpu()
        if slots:
            q, k, v, bt, lens = engine.snapshot(slots)
            assert_close(out[slots], ref_decode(q, k, v, bt, lens), f"step {rec['step']}")
            back = engine.cached(slots[::-1])[0]
            n = int(lens[-1])
            last = torch.from_numpy(k[bt[-1, (n - 1) // PAGE], (n - 1) % PAGE])
            assert torch.equal(back[n - 1].cpu(), last)
            checked.append(rec["step"])
        assert torch.all(out[[s for s in range(4) if s not in slots]] == 0)
        assert pkv.pkv_check_device_status(engine.bufs.ws) == 0

    sched = Scheduler(trace, engine, PagePool(4 * maxp, seed=7), max_batch=4, observer=check)
    while not sched.finished and sched.step_idx < 30:
        sched.step()
    assert sched.finished and sorted(sched.done) == list(range(5)) and len(checked) >= 6


def test_serving_refuses_an_unknown_format():
    from paper_2606_26666_amd.serving import Engine
    with pytest.raises(ValueError, match="kv must be"):
        Engine(4, 4, 16, kv="int4")
    with pytest.raises(ValueError, match="8 bits"):
        Engine(1, 1, 1, hq=1, hkv=1).cached([0])
