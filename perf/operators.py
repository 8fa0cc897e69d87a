"""The 8-bit paged KV cache: writing it, reading it back, and attending one new token over it,
as a serving program calls them, with plain forms of the same mathematics.

A pool is uint8 [num_pages, Hkv, RECORD]: for each page of 16 tokens and each KV head one record of
  K codes [16][128], V codes [4][128][4] (token 4a + b, dim c at [a][c][b]), K scales fp32 [16],
  V scales fp32 [16].
A stored value is code * scale, with int8 codes (scale = max|x| / 127) or e4m3 codes (max|x| / 448),
one scale for each token and KV head.

A case is a dict of plain values:
  op       "append": the last tokens of each row are quantised into its pages
           "gather": the last tokens of each row are read back in fp16
           "decode": attention of one query token per row over the row's cache
  format   "int8" or "e4m3"
  batch    rows; `free` of them are empty slots of a serving batch (length 0)
  family, lo, hi, lengths  the rows' lengths: "uniform" in [lo, hi], "bimodal" (half short, half
           long), "zipf" (multiples of lo, heavy-tailed) or "equal" (all hi), from seed `lengths`
  part     append, gather: how much of each row: "token" (its last token), "chunk" (up to `chunk`
           last tokens, a length of its own for each row) or "row" (all of it)
  hq, hkv  query and KV heads
  fused    queries, keys and values are slices of one [tokens, (hq + 2 hkv) * 128] projection

Codes, scales, values, page order and holes come from the seed that prepare() gets.
"""
import math
import random

import torch

own = False

D = 128
PAGE = 16
K_BYTES = PAGE * D
RECORD = 2 * K_BYTES + 2 * PAGE * 4
TOP = {"int8": 127.0, "e4m3": 448.0}
MAX_TOKENS = 65536     # the longest row
MAX_DECODE = 3_400_000  # rows * longest row * KV heads of the largest drawn attention
MAX_MOVED = 500_000     # the same for a write or a read-back


def _case(name, op, format, batch, family, lo, hi, hkv, *, hq=32, lengths=1, part="row", chunk=0, free=0,
          fused=False):
    c = dict(op=op, format=format, batch=batch, family=family, lo=lo, hi=hi, hkv=hkv, hq=hq, lengths=lengths,
             part=part, chunk=chunk, free=free, fused=fused)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # the smallest attention call: one short chat turn
        _case("decode_short", "decode", "int8", 1, "equal", 77, 77, 8),
        # one long document being read: the benchmark's B1 configuration
        _case("decode_b1_32k", "decode", "int8", 1, "equal", 32769, 32769, 8),
        # short and long rows together: the benchmark's B8 bimodal configuration
        _case("decode_b8_bimodal", "decode", "e4m3", 8, "bimodal", 256, 32768, 8, lengths=20260623),
        # a serving batch of chats with free slots, queries from a fused projection
        _case("decode_b64_chat", "decode", "int8", 64, "uniform", 128, 4096, 8, free=5, fused=True),
        # many short rows, 8 query heads per KV head
        _case("decode_b256_short_g8", "decode", "e4m3", 256, "uniform", 16, 1024, 8, hq=64),
        # the largest: a full batch of long ragged rows
        _case("decode_b32_uniform", "decode", "int8", 32, "uniform", 1024, 32768, 8, lengths=7),
        # no grouping: each query head has its own KV head
        _case("decode_b4_bimodal_g1", "decode", "e4m3", 4, "bimodal", 256, 32768, 32, lengths=3),
        # the write of a decode step: one token for each row of a small batch
        _case("append_token_b8", "append", "int8", 8, "uniform", 256, 8192, 8, part="token", fused=True),
        # a prompt batch written at once, ragged, from a fused projection
        _case("append_prompts", "append", "int8", 32, "uniform", 33, 4096, 8, part="row", fused=True),
        # chunked prefill: the next chunk of each of a few long rows
        _case("append_chunks_e4m3", "append", "e4m3", 8, "uniform", 1024, 16384, 8, part="chunk", chunk=2048),
        # a cached prefix read back for a short follow-up prompt
        _case("gather_prefix", "gather", "int8", 1, "equal", 1003, 1003, 8),
        # the rows of a batch read back for chunked prefill
        _case("gather_rows_e4m3", "gather", "e4m3", 16, "uniform", 100, 8192, 8, lengths=9),
    ]


def draw(rng):
    """One more case: the operator, the format, the heads, the batch (1..256) and the longest row (up
    to MAX_TOKENS), both evenly over their logarithms."""
    op = rng.choice(("decode", "decode", "append", "gather"))
    hq, hkv = rng.choice(((32, 8), (32, 8), (32, 4), (64, 8), (32, 16), (32, 32), (40, 8), (28, 4), (24, 8)))
    batch = round(math.exp(rng.uniform(0.0, math.log(256))))
    family = rng.choice(("uniform", "uniform", "bimodal", "zipf", "equal"))
    top = min(MAX_TOKENS, (MAX_DECODE if op == "decode" else MAX_MOVED) // (hkv * batch))
    hi = round(math.exp(rng.uniform(math.log(min(16, top)), math.log(top))))
    lo = min(hi, rng.choice((1, 16, 200, max(1, hi // 16))))
    part = rng.choice(("token", "chunk", "row")) if op != "decode" else "row"
    free = rng.randint(0, batch // 4) if rng.random() < 0.3 else 0
    return _case(None, op, rng.choice(("int8", "e4m3")), batch, family, lo, hi, hkv, hq=hq,
                 lengths=rng.randrange(1 << 30), part=part, chunk=rng.randint(2, 2048) if part == "chunk" else 0,
                 free=free, fused=rng.random() < 0.5)


def _lengths(case):
    """Row lengths: a function of the case alone."""
    r = random.Random(case["lengths"])
    lo, hi, n = case["lo"], case["hi"], case["batch"]
    if case["family"] == "uniform":
        lens = [r.randint(lo, hi) for _ in range(n)]
    elif case["family"] == "bimodal":
        short = [r.randint(lo, max(lo, hi // 16)) for _ in range(n // 2)]
        lens = short + [r.randint(max(lo, hi // 2), hi) for _ in range(n - n // 2)]
        r.shuffle(lens)
    elif case["family"] == "zipf":
        lens = [min(hi, int(lo * r.paretovariate(0.5))) for _ in range(n)]
    else:
        lens = [hi] * n
    for i in r.sample(range(n), case["free"]):
        lens[i] = 0
    return lens


def _counts(case, lens):
    """How many of each row's last tokens the call takes."""
    if case["part"] == "token":
        return [min(1, n) for n in lens]
    if case["part"] == "row":
        return list(lens)
    r = random.Random(case["lengths"] + 1)
    return [min(n, r.randint(1, case["chunk"])) for n in lens]


def _pool_views(cache):
    """K codes, V codes and both scales of a pool, as views of it."""
    pages, heads = cache.shape[:2]
    k = cache[:, :, :K_BYTES].unflatten(2, (PAGE, D))
    v = cache[:, :, K_BYTES:2 * K_BYTES].unflatten(2, (PAGE // 4, D, 4))
    s = cache[:, :, 2 * K_BYTES:].view(torch.float32)
    return k, v, s[:, :, :PAGE], s[:, :, PAGE:]


def _typed(codes, format):
    return codes.view(torch.int8 if format == "int8" else torch.float8_e4m3fn)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, hq, hkv, format = _lengths(case), case["hq"], case["hkv"], case["format"]
    B = len(lens)
    pages = [-(-n // PAGE) for n in lens]
    total = sum(pages)
    num_pages = total + total // 8 + 1
    table = torch.zeros((B, max(pages) + 2), dtype=torch.int32, device="cuda")
    perm = torch.randperm(num_pages, generator=gen, device="cuda", dtype=torch.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    # a pool as it stands after some use: codes and scales as values near N(0, 1) leave them
    cache = torch.empty((num_pages, hkv, RECORD), dtype=torch.uint8, device="cuda")
    k, v, ks, vs = _pool_views(cache)
    unit = 40.0 if format == "int8" else 100.0
    for codes in (k, v):
        x = torch.randn(codes.shape, generator=gen, device="cuda").mul_(unit).clamp_(-TOP[format], TOP[format])
        _typed(codes, format).copy_(x.round_() if format == "int8" else x)
        del x
    for s in (ks, vs):
        s.copy_((torch.rand(s.shape, generator=gen, device="cuda") * 0.4 + 0.8) / unit)
    st = dict(format=format, cache=cache, table=table, B=B, hq=hq, hkv=hkv, op=case["op"],
              lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), longest=max(lens))
    if case["op"] == "decode":
        q = torch.randn((B, hq + (2 * hkv if case["fused"] else 0), D), generator=gen, device="cuda").half()
        st["q"] = q[:, :hq]
        st["scale"] = 1.0 / math.sqrt(D)
        st["out"] = torch.empty((B, hq, D), dtype=torch.float16, device="cuda")
        return st
    counts = _counts(case, lens)
    st["offsets"] = None
    if case["part"] != "token":
        st["offsets"] = torch.tensor([sum(counts[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    tokens = B if case["part"] == "token" else sum(counts)
    st["counts"] = torch.tensor(counts, dtype=torch.int64, device="cuda")
    if case["op"] == "append":
        if case["fused"]:
            x = torch.randn((tokens, hq + 2 * hkv, D), generator=gen, device="cuda", dtype=torch.float16)
            st["k"], st["v"] = x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            st["k"], st["v"] = (torch.randn((tokens, hkv, D), generator=gen, device="cuda", dtype=torch.float16)
                                for _ in "kv")
    else:
        st["k"], st["v"] = (torch.zeros((tokens, hkv, D), dtype=torch.float16, device="cuda") for _ in "kv")
    return st


def _where(s):
    """Of each token that a call takes: its place among the call's tokens, its page and its slot."""
    counts, dev = s["counts"], s["lens"].device
    row = torch.repeat_interleave(torch.arange(s["B"], device=dev), counts, output_size=s["k"].shape[0]
                                  if s["offsets"] is not None else None)
    first = torch.cumsum(counts, 0) - counts
    nth = torch.arange(row.shape[0], device=dev) - first[row]
    pos = s["lens"].long()[row] - counts[row] + nth
    at = row if s["offsets"] is None else first[row] + nth
    return at, s["table"].long()[row, pos // PAGE], pos % PAGE


def _plain_append(s):
    at, page, slot = _where(s)
    k, v, ks, vs = _pool_views(s["cache"])
    top = TOP[s["format"]]
    for x, codes, scales in ((s["k"], k, ks), (s["v"], v, vs)):
        x = x[at].float()
        a = x.abs().amax(-1, keepdim=True)
        y = torch.where(a > 0, x * top / torch.where(a > 0, a, 1.0), 0.0)
        c = y.round().to(torch.int8) if s["format"] == "int8" else y.to(torch.float8_e4m3fn)
        if codes.dim() == 4:
            codes[page, :, slot] = c.view(torch.uint8)
        else:
            codes[page, :, slot // 4, :, slot % 4] = c.view(torch.uint8)
        scales[page, :, slot] = a[..., 0] / top
    return _pool_outputs(s)


def _pool_outputs(s):
    k, v, ks, vs = _pool_views(s["cache"])
    return {"k": _typed(k, s["format"]), "v": _typed(v, s["format"]), "k_scale": ks, "v_scale": vs}


def _plain_gather(s):
    at, page, slot = _where(s)
    k, v, ks, vs = _pool_views(s["cache"])
    out = []
    for codes, scales in ((k, ks), (v, vs)):
        c = codes[page, :, slot] if codes.dim() == 4 else codes[page, :, slot // 4, :, slot % 4]
        y = torch.zeros((s["k"].shape[0], s["hkv"], D), dtype=torch.float16, device=c.device)
        y[at] = (_typed(c, s["format"]).float() * scales[page, :, slot][..., None]).half()
        out.append(y)
    return {"k": out[0], "v": out[1]}


def _plain_decode(s):
    B, hq, hkv = s["B"], s["hq"], s["hkv"]
    pages = max(1, -(-s["longest"] // PAGE))
    rec = s["cache"][s["table"][:, :pages].long()]                  # [B, pages, Hkv, RECORD]
    k, v, ks, vs = _pool_views(rec.flatten(0, 1))
    k = _typed(k, s["format"]).float() * ks[..., None]              # [B * pages, Hkv, 16, D]
    k = k.unflatten(0, (B, pages)).transpose(1, 2).reshape(B * hkv, pages * PAGE, D)
    q = s["q"].float().reshape(B * hkv, hq // hkv, D)
    x = torch.bmm(k, q.transpose(1, 2).contiguous()) * s["scale"]   # [B * Hkv, tokens, G]
    del k
    there = torch.arange(pages * PAGE, device=x.device)[None] < s["lens"].long().repeat_interleave(hkv)[:, None]
    x = torch.where(there[..., None], x, -math.inf)
    m = x.amax(1, keepdim=True)
    p = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    total = p.sum(1)                                                # [B * Hkv, G]
    v = _typed(v, s["format"]).permute(0, 1, 2, 4, 3).float().flatten(2, 3) * vs[..., None]
    v = v.unflatten(0, (B, pages)).transpose(1, 2).reshape(B * hkv, pages * PAGE, D)
    o = torch.bmm(p.transpose(1, 2).contiguous(), v)
    o = torch.where(total[..., None] > 0, o / torch.where(total > 0, total, 1.0)[..., None], 0.0)
    return {"out": o.reshape(B, hq, D).half()}


def run(s):
    if not own:
        return {"append": _plain_append, "gather": _plain_gather, "decode": _plain_decode}[s["op"]](s)
    import paper_2606_26666_amd as pkv
    ws = s.get("ws")
    if ws is None:  # a program allocates its workspace once
        s["ws"] = ws = pkv.Kv8Buffers(s["B"], s["hq"], s["hkv"], D, "cuda").ws
    format = pkv.PKV_KV8_INT8 if s["format"] == "int8" else pkv.PKV_KV8_E4M3
    if s["op"] == "append":
        pkv.pkv_kv8_append(s["k"], s["v"], s["cache"], s["table"], s["lens"], ws, format=format, offsets=s["offsets"])
        return _pool_outputs(s)
    if s["op"] == "gather":
        pkv.pkv_kv8_gather(s["cache"], s["table"], s["lens"], s["k"], s["v"], ws, format=format, offsets=s["offsets"])
        return {"k": s["k"], "v": s["v"]}
    pkv.pkv_kv8_decode(s["q"], s["cache"], s["table"], s["lens"], s["scale"], s["out"], ws, format=format)
    return {"out": s["out"]}


def work(case):
    """Records, values, queries, lengths and page ids read or written once."""
    lens = _lengths(case)
    hkv, hq = case["hkv"], case["hq"]
    if case["op"] == "decode":
        n, rows = sum(lens), len(lens)
        pages = sum(-(-x // PAGE) for x in lens)
        return {"bytes": n * hkv * (2 * D + 8) + rows * hq * D * 4 + 4 * (pages + rows), "flops": 4 * hq * D * n}
    n = sum(_counts(case, lens))
    pages = sum(-(-x // PAGE) for x in _counts(case, lens))
    return {"bytes": n * hkv * (2 * D + 8 + 4 * D) + 4 * (pages + 2 * len(lens)), "flops": 8 * n * hkv * D}


def exact(case, seed):
    """From the definitions, a row at a time, in 64 bits."""
    s = prepare(case, seed)
    lens, hkv, hq = _lengths(case), case["hkv"], case["hq"]
    kc, vc, ks, vs = _pool_views(s["cache"])
    table = s["table"].cpu().tolist()

    def stored(i, begin, end):
        """K and V [end - begin, Hkv, D] of row i as the pool holds them."""
        ids = torch.tensor(table[i][begin // PAGE:-(-end // PAGE)], device="cuda")
        cut = slice(begin % PAGE, begin % PAGE + end - begin)
        k = _typed(kc[ids], case["format"]).double() * ks[ids].double().unsqueeze(3)
        v = _typed(vc[ids], case["format"]).double().transpose(3, 4).reshape(len(ids), hkv, PAGE, D)
        v = v * vs[ids].double().unsqueeze(3)
        return tuple(x.transpose(1, 2).reshape(-1, hkv, D)[cut] for x in (k, v))

    if case["op"] == "decode":
        out = torch.zeros((len(lens), hq, D), dtype=torch.float64, device="cuda")
        for i, n in enumerate(lens):
            if n == 0:
                continue
            k, v = (x.transpose(0, 1).contiguous() for x in stored(i, 0, n))
            q = s["q"][i].double().reshape(hkv, hq // hkv, D)
            x = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
            out[i] = torch.bmm(torch.softmax(x, -1), v).reshape(hq, D)
        return {"out": out}
    counts = _counts(case, lens)
    if case["op"] == "gather":
        k, v = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s["k"], s["v"]))
        at = 0
        for i, (n, c) in enumerate(zip(lens, counts)):
            at = i if case["part"] == "token" else at
            if c:
                k[at:at + c], v[at:at + c] = stored(i, n - c, n)
            at += c
        return {"k": k, "v": v}
    top = TOP[case["format"]]
    ks, vs = ks.double(), vs.double()
    at = 0
    for i, (n, c) in enumerate(zip(lens, counts)):
        at = i if case["part"] == "token" else at
        for page in range((n - c) // PAGE, -(-n // PAGE)) if c else ():
            b, e = max(n - c, page * PAGE), min(n, (page + 1) * PAGE)
            src = slice(at + b - (n - c), at + e - (n - c))
            dst = slice(b % PAGE, b % PAGE + e - b)
            for x, codes, scales in ((s["k"], kc, ks), (s["v"], vc, vs)):
                x = x[src].double().transpose(0, 1)                  # [Hkv, tokens, D]
                a = x.abs().amax(-1)
                y = x * top / a.clamp_min(1e-300).unsqueeze(-1)
                y = y.round().to(torch.int8) if case["format"] == "int8" else y.to(torch.float8_e4m3fn)
                y = y.view(torch.uint8)
                rec = codes[table[i][page]]
                if rec.dim() == 3:
                    rec[:, dst] = y
                else:
                    whole = rec.transpose(2, 3).reshape(hkv, PAGE, D)  # a copy
                    whole[:, dst] = y
                    rec.copy_(whole.unflatten(1, (PAGE // 4, 4)).transpose(2, 3))
                scales[table[i][page]][:, dst] = a / top
        at += c
    return {"k": _typed(kc, case["format"]), "v": _typed(vc, case["format"]), "k_scale": ks, "v_scale": vs}
