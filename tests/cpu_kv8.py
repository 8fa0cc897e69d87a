"""The 8-bit cache's kernels on the CPU: their sources against tests/cpu_device, and one call through
the C ABI on host arrays (every access bounds checked, the waves' schedule chosen by the test)."""
from __future__ import annotations

import os
import re
import struct
import subprocess
import tempfile

import numpy as np

from oracle import kv8
from tests.cpu_cases import ASCENDING, CSRC, DEVICE, compiler
from workloads import page_table


def build(folder):
    flags = [compiler(), "-std=c++17", "-O2", "-fno-pie", "-ffp-contract=off", "-w", "-I", DEVICE, "-I", CSRC]
    with open("/proc/cpuinfo") as f:
        have = set(re.findall(r"\b(?:fma|f16c)\b", f.read()))
    flags += [f"-m{x}" for x in sorted(have)]
    units = [(os.path.join(CSRC, n), n.split(".")[0]) for n in
             ("pkv_kernels.hip", "pkv_kv8.hip", "pkv_capi.cpp", "pkv_kv8_capi.cpp")]
    units += [(os.path.join(DEVICE, "emu.cpp"), "emu"), (os.path.join(DEVICE, "main_kv8.cpp"), "main")]
    objs, jobs = [], []
    for src, name in units:
        objs.append(os.path.join(folder, name + ".o"))
        jobs.append(subprocess.Popen([*flags, "-x", "c++", "-c", src, "-o", objs[-1]], stderr=subprocess.PIPE, text=True))
    for j in jobs:
        err = j.communicate()[1]
        assert j.returncode == 0, err
    exe = os.path.join(folder, "cpu_kv8")
    subprocess.run([compiler(), "-no-pie", *objs, "-o", exe], check=True)
    return exe


class Cache:
    """Rows of given lengths with a pool of pages in scattered order. Everything that no row holds
    (unowned pages, slots past a row's end) reads as NaN: scales and, in e4m3, codes."""

    def __init__(self, lens, hkv=2, fmt=kv8.INT8, seed=0, filled=True, spare=1):
        r = np.random.Generator(np.random.PCG64(seed))
        self.lens = np.asarray(lens, dtype=np.int32)
        self.B, self.hkv, self.fmt = len(lens), hkv, fmt
        bt, n = page_table(np.maximum(self.lens, 1) + 16 * (spare - 1), 16, 0.3, r)
        self.bt, self.num_pages = np.ascontiguousarray(bt, dtype=np.int32), int(n)
        self.pool = np.full((self.num_pages, hkv, kv8.RECORD), 0xFF, dtype=np.uint8)
        if filled:  # codes and scales as values near N(0, 1) leave them
            row = np.repeat(np.arange(self.B), self.lens)
            pos = np.concatenate([np.arange(n) for n in self.lens] + [np.zeros(0, dtype=np.int64)]).astype(np.int64)
            page, slot = self.bt[row, pos // 16], pos % 16
            k, v, ks, vs = kv8.views(self.pool)
            for codes, scales in ((k, ks), (v, vs)):
                x = r.standard_normal((len(pos), hkv, kv8.D), dtype=np.float32)
                if fmt == kv8.INT8:
                    c = np.clip(np.rint(x * 40), -127, 127).astype(np.int8).view(np.uint8)
                else:
                    c = (np.searchsorted(kv8.VALUES[fmt][:127], np.abs(x) * 100) + 128 * (x < 0)).clip(0, 254).astype(np.uint8)
                    c[c == 127] = 126
                if codes.ndim == 4:
                    codes[page, :, slot] = c
                else:
                    codes[page, :, slot // 4, :, slot % 4] = c
                scales[page, :, slot] = (r.random((len(pos), hkv)) * 0.4 + 0.8) / (40 if fmt == kv8.INT8 else 100)


def call(exe, what, cache, *, lens=None, bt=None, q=None, k=None, v=None, offsets=None, tokens=0, strides=None, hq=None,
         order=ASCENDING, compute_units=2, calls=1, sm_scale=1.0, num_pages=None, workspace_rows=0,
         last_workgroup=-1):
    """[(status, error bits, counters left, array or pair)] of each call; k and v are [tokens, stride]
    flat arrays for append, strides (k, v) for append and gather, (q,) for decode. workspace_rows: the batch
    that the workspace was made for (0: this one). last_workgroup: the one that runs behind all others (-1: in order)."""
    B, hkv = cache.B, cache.hkv
    hq = hq or hkv
    lens = cache.lens if lens is None else np.asarray(lens, dtype=np.int32)
    bt = cache.bt if bt is None else np.ascontiguousarray(bt, dtype=np.int32)
    strides = strides or ((hkv * 128,) * 2 if what != "decode" else (hq * 128,))
    ks, vs = strides if what != "decode" else (0, 0)
    head = struct.pack("<17if", ("append", "gather", "decode").index(what), order, compute_units, calls, B, hq, hkv,
                       cache.num_pages if num_pages is None else num_pages, bt.shape[1], cache.fmt, tokens,
                       offsets is not None, ks, vs, strides[0] if what == "decode" else 0, workspace_rows,
                       last_workgroup, sm_scale)
    parts = [cache.pool, bt, lens]
    if what == "decode":
        parts.append(q.reshape(-1)[:(B - 1) * strides[0] + hq * 128])
    elif tokens:
        parts += [x.reshape(-1)[:(tokens - 1) * s + hkv * 128] for x, s in ((k, ks), (v, vs))]
    if offsets is not None:
        parts.append(np.asarray(offsets, dtype=np.int32))
    with tempfile.TemporaryDirectory() as d:
        req, ans = os.path.join(d, "req"), os.path.join(d, "ans")
        with open(req, "wb") as f:
            f.write(head)
            for p in parts:
                f.write(np.ascontiguousarray(p).tobytes())
        p = subprocess.run([exe, req, ans], capture_output=True, text=True, timeout=300)
        assert p.returncode == 0, (p.returncode, p.stderr)
        raw = open(ans, "rb").read()
    got, at = [], 0

    def take(dtype, n):
        nonlocal at
        a = np.frombuffer(raw, dtype=dtype, count=n, offset=at)
        at += a.nbytes
        return a

    for _ in range(calls):
        st = take(np.int32, 3).tolist()
        if what == "append":
            got.append((*st, take(np.uint8, cache.pool.size).reshape(cache.pool.shape)))
        elif what == "decode":
            got.append((*st, take(np.float16, B * hq * 128).reshape(B, hq, 128)))
        else:
            got.append((*st, tuple(take(np.float16, (tokens - 1) * s + hkv * 128) for s in (ks, vs))))
    return got
