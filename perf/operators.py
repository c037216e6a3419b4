"""The calls around a paged key/value cache held in 4 bits, timed on one GPU over the range of sizes that serving meets after a
prefill: block tables, writes, the way back to rows, and attention for single tokens, chunks and both together.

A case is a dict of plain values.  `op` is the operator:

  tables  Context.block_tables: tables, row starts, positions and slots of a step, from the requests' lengths
  write   Context.rope_kv4_write and Context.kv4_load: new tokens rotated and written, and read back as rows
  store   Context.kv4_store and Context.kv4_load: rows that a prefill left put into pages, and read back
  attn    Context.attn_kv4: attention of a ragged batch over the pages

`shard` names the heads of a tensor-parallel rank.  `B` requests have lengths between `lo` and `hi` (spread over the logarithm,
the same for every seed); each has `new` tokens in this step, the first `chunks` of them `chunk` instead.

The cache format: 32 neighbouring elements of a head share a scale 2^(byte - 127), an element is sign and one of eight
magnitudes (LEVELS).  The exponent is the least with max|x| <= 7 * 2^e; ties between two levels go to the even code.
"""
import functools
import math

import torch

own = False

# local query heads, local key/value heads, head_dim, element type
SHARDS = {
    "tiny": (4, 4, 64, "f32"),
    "30b_tp4": (13, 13, 128, "bf16"),
    "70b_tp8": (8, 1, 128, "bf16"),
    "70b_tp4": (16, 2, 128, "bf16"),
    "heads64": (32, 8, 64, "bf16"),
}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
ROPE_BASE = 10000.0
WRITTEN = 8320                           # no case writes a token behind it


def listed():
    return [
        # one decoding step of a full batch: a row per request, a new page for one in sixty-four of them
        {"name": "tables_decode_256", "op": "tables", "B": 256, "lo": 64, "hi": 8192, "new": 1, "chunks": 0, "chunk": 0, "page": 64},
        # prompts of all lengths entering at once, every page of theirs new
        {"name": "tables_prompts_100k", "op": "tables", "B": 96, "lo": 64, "hi": 4096, "new": 0, "chunks": 96, "chunk": 0, "page": 16},
        # the tokens of one decoding step of the GQA shard
        {"name": "write_70b_tp4_64", "op": "write", "shard": "70b_tp4", "T": 64, "lo": 64, "hi": 8192, "page": 64},
        # a chunk of a prompt through the multi-head shard, odd length
        {"name": "write_30b_tp4_2047", "op": "write", "shard": "30b_tp4", "T": 2047, "lo": 0, "hi": 2047, "page": 64},
        # a short fp32 prompt kept for later
        {"name": "store_tiny_128", "op": "store", "shard": "tiny", "T": 128, "page": 16},
        # one layer's cache of the 16k prompt of the repository's benchmark
        {"name": "store_70b_tp8_16k", "op": "store", "shard": "70b_tp8", "T": 16384, "page": 64},
        # the smallest answer: single tokens of three fp32 requests over short prompts
        {"name": "attn_tiny_3", "op": "attn", "shard": "tiny", "B": 3, "lo": 17, "hi": 200, "new": 1, "chunks": 0, "chunk": 0, "page": 16},
        # one user with the longest prompt of the workloads, one token at a time
        {"name": "attn_70b_tp8_128k", "op": "attn", "shard": "70b_tp8", "B": 1, "lo": 131072, "hi": 131072, "new": 1, "chunks": 0, "chunk": 0, "page": 64},
        # a batch of answers, heads of 64, ragged lengths, two tokens at a time (a drafted one is checked along)
        {"name": "attn_heads64_48", "op": "attn", "shard": "heads64", "B": 48, "lo": 300, "hi": 8192, "new": 2, "chunks": 0, "chunk": 0, "page": 32},
        # a batch of answers of the multi-head shard: every key head has one row
        {"name": "attn_30b_tp4_40", "op": "attn", "shard": "30b_tp4", "B": 40, "lo": 500, "hi": 8192, "new": 1, "chunks": 0, "chunk": 0, "page": 64},
        # a 2k chunk deep inside a long prompt
        {"name": "attn_70b_tp8_2k_at_30k", "op": "attn", "shard": "70b_tp8", "B": 1, "lo": 32768, "hi": 32768, "new": 0, "chunks": 1, "chunk": 2048, "page": 64},
        # answers and pieces of two new prompts in the same step
        {"name": "attn_70b_tp4_mixed", "op": "attn", "shard": "70b_tp4", "B": 24, "lo": 700, "hi": 6000, "new": 1, "chunks": 2, "chunk": 509, "page": 64},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "write", "store", "attn", "attn", "attn", "attn"))
    page = rng.choice((16, 32, 64, 128))
    shard = rng.choice(("tiny", "30b_tp4", "70b_tp8", "70b_tp4", "heads64"))
    if op == "tables":
        B, hi = _log_int(rng, 1, 256), _log_int(rng, 64, 8192)
        prompts = rng.random() < 0.4
        if prompts:
            hi = min(hi, 4096, 400000 // B)
        return {"op": op, "B": B, "lo": max(1, hi // 50), "hi": hi, "new": 0 if prompts else rng.randint(1, 4), "chunks": B if prompts else 0,
                "chunk": 0, "page": page}
    if op == "write":
        T = _log_int(rng, 1, 512 if shard == "tiny" else 2048)
        lo = rng.choice((0, 100))
        return {"op": op, "shard": shard, "T": T, "lo": lo, "hi": max(T + lo, _log_int(rng, 200, 8192)), "page": page}
    if op == "store":
        return {"op": op, "shard": shard, "T": _log_int(rng, 1, 512 if shard == "tiny" else 16384), "page": page}
    kind = rng.choice(("one", "batch", "batch", "chunk", "mixed"))
    if shard == "tiny":
        B, hi = _log_int(rng, 1, 8), _log_int(rng, 16, 1024)
        return {"op": op, "shard": shard, "B": B, "lo": max(1, hi // 9), "hi": hi, "new": rng.choice((1, 1, 3)), "chunks": rng.choice((0, 1)),
                "chunk": _log_int(rng, 5, 100), "page": page}
    if kind == "one":
        hi = _log_int(rng, 200, 131072 if shard[:3] == "70b" else 16384)
        return {"op": op, "shard": shard, "B": 1, "lo": hi, "hi": hi, "new": rng.choice((1, 1, 2, 5)), "chunks": 0, "chunk": 0, "page": page}
    if kind == "batch":
        hi = _log_int(rng, 200, 8192)
        return {"op": op, "shard": shard, "B": _log_int(rng, 2, 40), "lo": max(1, int(hi * rng.uniform(0.05, 1.0))), "hi": hi,
                "new": rng.choice((1, 1, 1, 2, 4)), "chunks": 0, "chunk": 0, "page": page}
    if kind == "chunk":
        C = _log_int(rng, 16, 2048)
        hi = C + rng.choice((0, _log_int(rng, 64, 30000 if shard == "70b_tp8" else 6000)))
        return {"op": op, "shard": shard, "B": 1, "lo": hi, "hi": hi, "new": 0, "chunks": 1, "chunk": C, "page": page}
    hi = _log_int(rng, 700, 6000)
    return {"op": op, "shard": shard, "B": rng.randint(3, 24), "lo": max(64, hi // 8), "hi": hi, "new": 1, "chunks": rng.randint(1, 2),
            "chunk": rng.randint(20, 509), "page": page}


# ------------------------------------------------------------------------------------------------ sizes that a case stands for

def lengths(case):
    """(kv_len, fresh) of every request, plain lists: what follows from the case alone."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    kv = [int(round(lo * (hi / lo) ** ((1 + i * 0.6180339887498949) % 1.0 if B > 1 else 1.0))) for i in range(B)]
    fresh = [min(k, (case["chunk"] or k) if i < case["chunks"] else case["new"]) for i, k in enumerate(kv)]
    return kv, fresh


# ------------------------------------------------------------------------------------------------ the format, in plain steps

def encode(x):
    """[..., d] values (their own precision is kept) -> code bytes [..., d / 2], scale bytes [..., d / 32]."""
    b = x.unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 3, e - 2)
    e = torch.where(top > 0, e, -125).clamp(-125, 125)
    fine = torch.isfinite(b).all(-1, keepdim=True)
    e = torch.where(fine, e, 0)
    u = torch.ldexp(b.abs().double(), -e)
    code = ((u > 0.25).byte() + (u >= 0.75) + (u > 1.25) + (u >= 1.75) + (u > 2.5) + (u >= 3.5) + (u > 5.0)) | ((b < 0).byte() << 3)
    code = torch.where(fine, code, 0).flatten(-2)
    scale = torch.where(fine, e + 127, 255).to(torch.uint8).squeeze(-1)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def decode(codes, scales):
    """fp32 values of code bytes [..., d / 2] and scale bytes [..., d / 32]."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device, dtype=torch.float32)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    factor = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    factor = torch.where(scales == 255, torch.nan, factor)
    return (level[code.int()].unflatten(-1, (-1, BLOCK)) * factor[..., None]).flatten(-2)


def put(cache, which, rows, slots, page):
    """Writes rows [T, nkv, d] into the pages."""
    codes, scales = encode(rows)
    pg, at = slots.long() // page, slots.long() % page
    cache[which][pg, :, at] = codes
    cache[which + "_scale"][pg, :, at] = scales


def take(cache, which, slots, page):
    """fp32 rows [T, nkv, d] that the slots hold."""
    pg, at = slots.long() // page, slots.long() % page
    return decode(cache[which][pg, :, at], cache[which + "_scale"][pg, :, at])


def rotary(positions, d):
    """The table that the framework rotates with: angles and their functions in 64 bits, kept in 32."""
    inv = torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device=positions.device),
                    torch.arange(d // 2, device=positions.device, dtype=torch.float64) * (-2.0 / d))
    ang = positions.double()[:, None, None] * inv
    return ang.cos().float(), ang.sin().float()


def rotate(x, c, s):
    lo, hi = x.chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


# ------------------------------------------------------------------------------------------------ inputs

def _cache(n_pages, nkv, page, d):
    z = lambda w: torch.zeros((n_pages, nkv, page, w), device="cuda", dtype=torch.uint8)  # noqa: E731
    return {"k": z(d // 2), "v": z(d // 2), "k_scale": z(d // BLOCK), "v_scale": z(d // BLOCK)}


def _context(heads, positions):
    """The context that a serving program keeps: one for each shard, with a rotary table for the positions that are written (the other
    calls use nothing of it but the heads and the type)."""
    return _contexts(heads, positions, torch.cuda.current_stream())


@functools.lru_cache(maxsize=None)
def _contexts(heads, positions, stream):
    import paper_2409_11155_amd as iso
    nq, nkv, d, dt = heads
    return iso.Context(iso.make_cfg(64, nq, nkv, d, 64, dt, positions, rope_base=ROPE_BASE), stream0=stream)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    page, dev = case["page"], "cuda"
    ints = lambda v: torch.tensor(v, device=dev, dtype=torch.int32)  # noqa: E731
    if case["op"] == "tables":
        kv, fresh = lengths(case)
        width = max(-(-k // page) for k in kv) + 2
        have = ints([-(-(k - f) // page) for k, f in zip(kv, fresh)])
        pool = torch.randperm(2 * sum(-(-k // page) for k in kv) + 8, generator=gen, device=dev).int()
        used = int(have.sum())
        table = torch.full((len(kv), width), -1, device=dev, dtype=torch.int32)
        table[torch.arange(width, device=dev) < have[:, None]] = pool[:used]
        rows = sum(fresh)
        st = {"case": case, "cached": ints([k - f for k, f in zip(kv, fresh)]), "fresh": ints(fresh), "free": pool[used:].contiguous(),
              "head": ints([0]), "table": table, "rows": rows, "start": ints([0] * (len(kv) + 1)), "kv": ints([0] * len(kv)),
              "positions": ints([0] * rows), "slots": ints([0] * rows), "next": ints([0])}
        if own:
            st["ctx"] = _context(SHARDS["70b_tp8"], 64)
        return st
    heads = nq, nkv, d, dt = SHARDS[case["shard"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev).to(TORCH[dt])  # noqa: E731
    if case["op"] in ("write", "store"):
        T = case["T"]
        n_pages = -(-T // page) + 3
        st = {"case": case, "cache": _cache(n_pages, nkv, page, d), "slots": torch.randperm(n_pages * page, generator=gen, device=dev)[:T].int(),
              "k": torch.zeros((T, nkv, d), device=dev, dtype=TORCH[dt]), "v": torch.zeros((T, nkv, d), device=dev, dtype=TORCH[dt])}
        if case["op"] == "store":        # whole pages in any order, the last one in part
            order = torch.randperm(n_pages, generator=gen, device=dev)
            st["slots"] = (order[:, None] * page + torch.arange(page, device=dev)).flatten()[:T].int()
            st["k0"], st["v0"] = normal(T, nkv, d), normal(T, nkv, d)
        else:
            lo, hi = case["lo"], case["hi"]
            span_ = torch.arange(T, device=dev) if lo == 0 else torch.randint(lo, hi, (T,), generator=gen, device=dev)
            st["positions"], st["qkv"] = span_.int(), normal(T, nq + 2 * nkv, d)
            st["q"] = torch.zeros((T, nq, d), device=dev, dtype=TORCH[dt])
        if own:
            import paper_2409_11155_amd as iso
            st["ctx"] = _context(heads, 64 if case["op"] == "store" else WRITTEN)
            st["kv4"] = iso.Kv4Cache(page=page, **st["cache"])
        return st
    kv, fresh = lengths(case)
    need = [-(-k // page) for k in kv]
    order = torch.randperm(sum(need) + 5, generator=gen, device=dev).int()
    table = torch.full((len(kv), max(need)), -1, device=dev, dtype=torch.int32)
    table[torch.arange(max(need), device=dev) < ints(need)[:, None]] = order[: sum(need)]
    cache = _cache(sum(need) + 5, nkv, page, d)
    for w in ("k", "v"):                 # a few pages at a time: the values are made in 32 bits
        step = max(1, (1 << 26) // (nkv * page * d))
        for p in range(0, cache[w].shape[0], step):
            cache[w][p:p + step], cache[w + "_scale"][p:p + step] = encode(torch.randn((min(step, cache[w].shape[0] - p), nkv, page, d),
                                                                                     generator=gen, device=dev))
    rows = sum(fresh)
    st = {"case": case, "cache": cache, "table": table, "kv": ints(kv), "start": ints([sum(fresh[:i]) for i in range(len(kv) + 1)]),
          "q": normal(rows, nq, d), "out": torch.zeros((rows, nq, d), device=dev, dtype=TORCH[dt]), "rows": rows, "most": max(fresh), "longest": max(kv)}
    if own:
        import paper_2409_11155_amd as iso
        st["ctx"] = _context(heads, 64)
        st["kv4"] = iso.Kv4Cache(page=page, **cache)
        bytes_ = st["ctx"].attn_kv4_workspace(len(kv), rows)
        st["ws"] = torch.zeros(bytes_, device=dev, dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["op"] == "tables":
        return _tables(state, case["page"])
    page, cache = case["page"], state["cache"]
    if case["op"] == "attn":
        return [_attention(state, case)]
    nq, nkv, d, dt = SHARDS[case["shard"]]
    got = []
    if case["op"] == "write":
        c, s = rotary(state["positions"], d)
        q, k, v = state["qkv"].split((nq, nkv, nkv), 1)
        got = [rotate(q.float(), c, s).to(TORCH[dt])]
        k = rotate(k.double(), c.double(), s.double())
    else:
        k, v = state["k0"], state["v0"]
    put(cache, "k", k, state["slots"], page)
    put(cache, "v", v, state["slots"], page)
    return got + [take(cache, "k", state["slots"], page).to(TORCH[dt]), take(cache, "v", state["slots"], page).to(TORCH[dt])]


def _run_own(st, case):
    ctx, stream = st["ctx"], torch.cuda.current_stream()
    if case["op"] == "tables":
        ctx.block_tables(st["cached"], st["fresh"], len(st["kv"]), case["page"], st["free"], len(st["free"]), st["head"], st["table"],
                         st["table"].shape[1], st["start"], st["kv"], st["positions"], st["slots"], st["rows"], st["next"], stream)
        return [st[n] for n in ("table", "start", "kv", "positions", "slots", "next")]
    if case["op"] == "attn":
        nq, nkv, d, _ = SHARDS[case["shard"]]
        ctx.attn_kv4(st["q"], nq * d, st["kv4"], st["table"], st["table"].shape[1], st["start"], st["kv"], len(st["kv"]), st["rows"],
                     st["most"], st["out"], st["ws"], st["ws"].numel(), stream)
        return [st["out"]]
    T, got = case["T"], []
    if case["op"] == "write":
        ctx.rope_kv4_write(st["qkv"], st["q"], st["kv4"], st["positions"], st["slots"], T, stream)
        got = [st["q"]]
    else:
        ctx.kv4_store(st["k0"], st["v0"], st["kv4"], st["slots"], T, stream)
    ctx.kv4_load(st["kv4"], st["slots"], st["k"], st["v"], T, stream)
    return got + [st["k"], st["v"]]


def _tables(st, page):
    cached, fresh, free, table, rows = st["cached"].long(), st["fresh"].long(), st["free"], st["table"], st["rows"]
    start = torch.nn.functional.pad(fresh.cumsum(0), (1, 0))
    kv = cached + fresh
    have, want = (cached + page - 1) // page, (kv + page - 1) // page
    taken = want - have
    col = torch.arange(table.shape[1], device=table.device)
    at = (st["head"] + taken.cumsum(0) - taken - have)[:, None] + col
    new = torch.where(at < len(free), free[at.clamp(0, len(free) - 1)], -1)
    table = torch.where((col >= have[:, None]) & (col < want[:, None]), new, table)
    r = torch.arange(rows, device=table.device)
    i = torch.searchsorted(start[1:], r, right=True)
    p = cached[i] + r - start[i]
    pg = table[i, p // page]
    slots = torch.where(pg >= 0, pg * page + p % page, -1)
    return [t.int() for t in (table, start, kv, p, slots, st["head"] + taken.sum())]


def _attention(st, case):
    nq, nkv, d, dt = SHARDS[case["shard"]]
    cache, table, kv, start, G = st["cache"], st["table"].long().clamp(min=0), st["kv"].long(), st["start"].long(), nq // nkv
    B, most = len(kv), st["most"]

    def keys(w):                         # [B, nkv, keys, d] in 32 bits
        return decode(cache[w][table], cache[w + "_scale"][table]).transpose(1, 2).flatten(2, 3)[:, :, :st["longest"]]

    n = start[1:] - start[:-1]
    t = torch.arange(most, device=kv.device)
    row = (start[:-1, None] + t).clamp(max=st["rows"] - 1)
    q = st["q"][row].float().view(B, most, nkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, nkv, most * G, d)
    s = torch.matmul(q * (1.0 / math.sqrt(d)), keys("k").transpose(-1, -2).contiguous())
    j = torch.arange(st["longest"], device=kv.device)
    seen = j <= (kv - n)[:, None, None] + t[:, None]                       # [B, most, keys]
    seen = (seen & (j < kv[:, None, None])).repeat_interleave(G, 1)[:, None]
    s = s.masked_fill_(~seen, -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s, keys("v").contiguous()) / s.sum(-1, keepdim=True)
    o = o.view(B, nkv, most, G, d).permute(0, 2, 1, 3, 4).reshape(B, most, nq, d)
    return o[t < n[:, None]].to(TORCH[dt])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "tables":
        kv, fresh = lengths(case)
        P, B, rows = case["page"], case["B"], sum(fresh)
        new = sum(-(-k // P) - -(-(k - f) // P) for k, f in zip(kv, fresh))
        return {"bytes": 4 * (2 * B + 2 * B + 1 + 2 * rows + 2 * new + 2), "flops": 0}
    nq, nkv, d, dt = SHARDS[case["shard"]]
    e = 4 if dt == "f32" else 2
    packed = 2 * nkv * (d // 2 + d // BLOCK)          # bytes of a token's K and V in the cache
    if case["op"] == "store":
        return {"bytes": case["T"] * (2 * packed + 4 * nkv * d * e + 4), "flops": 0}
    if case["op"] == "write":
        return {"bytes": case["T"] * ((nq + 2 * nkv) * d * e + nq * d * e + 4 * d + 2 * packed + 2 * nkv * d * e + 8), "flops": 6.0 * (nq + nkv) * d * case["T"]}
    kv, fresh = lengths(case)
    pairs = sum(f * (k - f) + f * (f + 1) / 2 for k, f in zip(kv, fresh))
    return {"bytes": sum(kv) * packed + 2 * sum(fresh) * nq * d * e + 4 * (sum(-(-k // case["page"]) for k in kv) + 2 * len(kv)),
            "flops": 4.0 * d * nq * pairs}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _stand(codes, scales):
    """Value of every code by the format's definition, one power of two at a time."""
    nib = torch.empty(codes.shape + (2,), dtype=torch.int64, device=codes.device)
    nib[..., 0], nib[..., 1] = codes & 15, codes >> 4
    nib = nib.flatten(-2)
    expo, man = (nib >> 1) & 3, (nib & 1).double()
    mag = torch.where(expo == 0, 0.5 * man, (1.0 + 0.5 * man) * torch.exp2(expo.double() - 1.0))
    sign = 1.0 - 2.0 * (nib >> 3).double()
    return sign * mag * torch.exp2(scales.double() - 127.0).repeat_interleave(BLOCK, -1)


def _nearest(x):
    """x [..., d] in 64 bits -> the value that the format keeps for it."""
    x = x.unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -140)
    e = torch.ceil(torch.log2(top / 7.0))
    e = torch.where(top <= 7.0 * torch.exp2(e - 1), e - 1, torch.where(top > 7.0 * torch.exp2(e), e + 1, e)).clamp(-125, 125)
    u = x.abs() * torch.exp2(-e)
    step = torch.where(u < 2.0, 0.5, torch.where(u < 4.0, 1.0, 2.0)).double()
    u = (torch.round(u / step) * step).clamp(max=6.0)       # halfway: to the even multiple, which has the even code
    return (torch.sign(x) * u * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    if case["op"] == "tables":
        return None
    nq, nkv, d, dt = SHARDS[case["shard"]]
    st = prepare(case, seed)
    if case["op"] == "store":
        return [_nearest(st["k0"].double()), _nearest(st["v0"].double())]
    if case["op"] == "write":
        pos = st["positions"].cpu().double()
        ang = pos[:, None] * torch.tensor([ROPE_BASE ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64)
        c, s = (f.float().double()[:, None].cuda() for f in (ang.cos(), ang.sin()))
        x = st["qkv"].double()
        a, b = x[..., : d // 2], x[..., d // 2:]
        y = torch.empty_like(x)
        y[..., : d // 2], y[..., d // 2:] = a * c - b * s, b * c + a * s
        return [y[:, :nq], _nearest(y[:, nq:nq + nkv]), _nearest(x[:, nq + nkv:])]
    kv, fresh = lengths(case)
    out, r0, G = [], 0, nq // nkv
    for i, (n, f) in enumerate(zip(kv, fresh)):
        pages = st["table"][i, : -(-n // case["page"])].long()
        k, v = (_stand(st["cache"][w][pages], st["cache"][w + "_scale"][pages]).transpose(0, 1).flatten(1, 2)[:, :n] for w in ("k", "v"))
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - f, n, device="cuda")[:, None]
        heads = []
        for h in range(nq):
            s = (st["q"][r0:r0 + f, h].double() @ k[h // G].T) * d ** -0.5
            s[hidden] = -math.inf
            heads.append(torch.softmax(s, -1) @ v[h // G])
        out.append(torch.stack(heads, 1))
        r0 += f
    return [torch.cat(out)]
