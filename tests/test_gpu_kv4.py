"""The paged 4-bit cache on the GPU against its definition in 64 bits (oracle/kv4_oracle.py).

Bounds.  Integers, codes and scales are equal.  What a slot holds is loaded exactly.  Attention, per element, with u the half step of
the type (bf16 2^-8, fp32 2^-24), A the probability-weighted mean of |v| and N the number of keys:
  u |out|                      the result is rounded once
  u A                          the probabilities are rounded to the type for the second product (their sum is not)
  2 E A                        E: what a score is off by, (d + 8) 2^-24 of the sum of its products' magnitudes, in units of the base-2
                               exponent (fp32 accumulation of exact products; scale, maximum and argument of the exponential) + 2^-22
                               (the exponential itself)
  (2 N + 16) 2^-24 A           fp32 accumulation of N terms, sums and rescaling
"""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def ints(a):
    return iso.DeviceArray.from_numpy(np.ascontiguousarray(a, dtype=np.int32), "i32")


def f64(a, dt):
    return iso_inputs.to_f64(a.numpy() if hasattr(a, "ptr") else a, dt)


def make_ctx(nq, nkv, d, dt, max_seq=256):
    return iso.Context(iso.make_cfg(64, nq, nkv, d, 64, dt, max_seq))


def device_cache(codes, scales, page):
    up = lambda a: iso.DeviceArray.from_numpy(a, "u8")  # noqa: E731
    return iso.Kv4Cache(page, up(codes[0]), up(codes[1]), up(scales[0]), up(scales[1]))


# ------------------------------------------------------------------------------------------------ block tables

TABLES = [([0], [1], 16), ([0], [0], 16), ([15], [2], 16), ([16, 0, 31, 64], [1, 1, 1, 1], 32), ([5, 0, 300, 16], [12, 0, 1, 48], 16),
          ([0] * 70, [3] * 70, 64), (list(range(300)), [1] * 300, 16), ([0, 0, 0], [1000, 0, 77], 128), ([-4, 7], [3, -2], 16),
          (list(range(0, 3 * 1111, 3)), [i % 4 for i in range(1111)], 256), ([9] * 4096, [1] * 4096, 16)]


@pytest.mark.parametrize("cached,fresh,page", TABLES)
@pytest.mark.parametrize("head,short,narrow,slack", [(None, 0, 0, 3), (2, 0, 0, 0), (0, 3, 0, 1), (1, 0, 1, 300)])
def test_block_tables(cached, fresh, page, head, short, narrow, slack):
    """head: start in the list; short: pages that the list lacks; narrow: columns that the table lacks; slack: rows more than there are
    (0: three fewer, so that some do not fit)."""
    rng = np.random.default_rng(len(cached) + page)
    have = [-(-max(0, c) // page) for c in cached]
    want = [-(-(max(0, c) + max(0, f)) // page) for c, f in zip(cached, fresh)]
    width = max(1, max(want) - narrow)
    pool = rng.permutation(sum(want) + 50)
    table, at = np.full((len(cached), width), -7), 0
    for i, n in enumerate(have):
        table[i, :n] = pool[at:at + n][:width]
        at += n
    need = sum(min(w, width) - min(h, width) for w, h in zip(want, have))
    free = pool[at:at + max(0, need + (head or 0) - short)]
    total = sum(max(0, f) for f in fresh)
    rows = max(1, total + slack if slack else total - 3)
    ref = ko.block_tables(cached, fresh, page, free, head or 0, table, rows)
    with make_ctx(4, 4, 64, "f32") as ctx:
        out = {n: ints(np.full(s, -99)) for n, s in (("start", len(cached) + 1), ("kv", len(cached)), ("pos", rows + 8), ("slots", rows + 8), ("next", 1))}
        td, fd = ints(table), ints(free) if len(free) else None
        for _ in range(2):                                      # the same call again gives the same
            ctx.block_tables(ints(cached), ints(fresh), len(cached), page, fd, len(free), None if head is None else ints([head]), td, width,
                             out["start"], out["kv"], out["pos"], out["slots"], rows, out["next"], ctx.stream0)
            ctx.sync()
            got = (td, *(out[n] for n in ("start", "kv", "pos", "slots", "next")))
            for g, w in zip(got, ref):
                g = g.numpy()
                if g.size == rows + 8:
                    assert (g[rows:] == -99).all()
                    g = g[:rows]
                np.testing.assert_array_equal(g, np.reshape(w, g.shape))


# ------------------------------------------------------------------------------------------------ writes and reads

def rows_with_everything(T, heads, d, dt, seed):
    """Values of many sizes, zero blocks, values on the borders of two codes, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, heads, d)) * np.exp2(rng.integers(-20, 20, (T, heads, 1)))
    x[rng.random((T, heads)) < 0.05] = 0.0
    edge = rng.random((T, heads)) < 0.2
    x[edge] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -5.0, 6.0], x[edge].shape)
    for bad in (np.nan, np.inf, -np.inf):
        x[rng.random(x.shape) < 0.0005] = bad
    return iso_inputs.store(x.astype(np.float32), dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nkv,d,T,page", [(1, 128, 1, 64), (2, 64, 3, 16), (5, 128, 100, 32), (8, 64, 333, 256), (13, 128, 257, 128)])
def test_rows_into_pages_and_back(dt, nkv, d, T, page):
    rng = np.random.default_rng(T)
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32)
    skip = rng.random(T) < 0.1
    slots[skip] = rng.choice([-1, -1000, n_pages * page, n_pages * page + 5, 2 ** 31 - 1], skip.sum())
    k, v = (rows_with_everything(T, nkv, d, dt, s) for s in (T, T + 1))
    with make_ctx(nkv, nkv, d, dt) as ctx:
        cache = ctx.kv4_cache(n_pages, page, fill_byte=0xA5)
        sd = ints(slots)
        ctx.kv4_store(iso.DeviceArray.from_numpy(k, dt), iso.DeviceArray.from_numpy(v, dt), cache, sd, T, ctx.stream0)
        out = [iso.DeviceArray((T, nkv, d), dt, fill_byte=0x5A) for _ in range(2)]
        ctx.kv4_load(cache, sd, out[0], out[1], T, ctx.stream0)
        ctx.sync()
        for x, codes, scales, back in ((k, cache.k, cache.k_scale, out[0]), (v, cache.v, cache.v_scale, out[1])):
            ref_c, ref_s = ko.encode(f64(x, dt))
            want_c, want_s = np.full(codes.shape, 0xA5, np.uint8), np.full(scales.shape, 0xA5, np.uint8)
            keep = ~skip
            want_c[slots[keep] // page, :, slots[keep] % page] = ref_c[keep]
            want_s[slots[keep] // page, :, slots[keep] % page] = ref_s[keep]
            np.testing.assert_array_equal(scales.numpy(), want_s)
            np.testing.assert_array_equal(codes.numpy(), want_c)
            got = f64(back, dt)
            np.testing.assert_array_equal(got[keep], ko.decode(ref_c, ref_s)[keep])
            np.testing.assert_array_equal(back.numpy()[skip].view(np.uint8), 0x5A)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,d,T,page,in_place", [(8, 1, 128, 1, 64, False), (4, 4, 64, 77, 16, True), (13, 13, 128, 130, 32, False), (16, 2, 128, 300, 64, True)])
def test_rotated_rows_into_pages(dt, nq, nkv, d, T, page, in_place):
    """q as iso_rope_kv_write rotates it (the same bits), k's codes those of the rotation in 64 bits, v's those of the row."""
    max_seq, rng = 4000, np.random.default_rng(T)
    n_pages, heads = -(-T // page) + 1, nq + 2 * nkv
    slots, pos = rng.permutation(n_pages * page)[:T].astype(np.int32), rng.integers(0, max_seq, T).astype(np.int32)
    if T > 10:
        slots[3], pos[5], pos[6], pos[7] = -1, -1, max_seq, 2 ** 31 - 1
    qkv = rows_with_everything(T, heads, d, dt, T)
    with make_ctx(nq, nkv, d, dt, max_seq) as ctx:
        cache = ctx.kv4_cache(n_pages, page, fill_byte=0xA5)
        xd, qo = iso.DeviceArray.from_numpy(qkv, dt), iso.DeviceArray((T, nq, d), dt, fill_byte=0x5A)
        ctx.rope_kv4_write(xd, None if in_place else qo, cache, ints(pos), ints(slots), T, ctx.stream0)
        ctx.sync()
        row_ok = (pos >= 0) & (pos < max_seq)
        after = xd.numpy()
        got_q = after[:, :nq] if in_place else qo.numpy()
        np.testing.assert_array_equal(after[:, nq:], qkv[:, nq:])
        if not in_place:
            np.testing.assert_array_equal(after, qkv)
        if in_place:
            np.testing.assert_array_equal(got_q[~row_ok], qkv[~row_ok][:, :nq])
        else:
            assert (got_q[~row_ok].view(np.uint8) == 0x5A).all()
        # the framework's own rotation of the same rows, one at a time (it takes consecutive positions)
        one_k, one_v = (iso.DeviceArray((max_seq, nkv, d), dt) for _ in range(2))
        for t in np.flatnonzero(row_ok)[:40]:
            row = iso.DeviceArray.from_numpy(qkv[t:t + 1], dt)
            ctx.rope_kv_write(row, one_k, one_v, 1, int(pos[t]), ctx.stream0)
            ctx.sync()
            np.testing.assert_array_equal(row.numpy()[0, :nq], got_q[t])
        x = f64(qkv, dt)
        with np.errstate(invalid="ignore"):
            rot = ko.rotate(x[:, nq:nq + nkv], np.where(row_ok, pos, 0))
        kept = row_ok & (slots >= 0)
        for val, codes, scales in ((rot, cache.k, cache.k_scale), (x[:, nq + nkv:], cache.v, cache.v_scale)):
            ref_c, ref_s = ko.encode(val)
            want_c, want_s = np.full(codes.shape, 0xA5, np.uint8), np.full(scales.shape, 0xA5, np.uint8)
            want_c[slots[kept] // page, :, slots[kept] % page] = ref_c[kept]
            want_s[slots[kept] // page, :, slots[kept] % page] = ref_s[kept]
            np.testing.assert_array_equal(scales.numpy(), want_s)
            np.testing.assert_array_equal(ko.decode(codes.numpy(), np.full_like(want_s, 127)), ko.decode(want_c, np.full_like(want_s, 127)))


# ------------------------------------------------------------------------------------------------ attention

def batch(kv, fresh, page, seed, spare=3):
    """(table, row_start, n_pages) with the pages in any order; entries behind a request's last page name a page of another one."""
    rng = np.random.default_rng(seed)
    need = [-(-k // page) for k in kv]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table, at = rng.choice(order, (len(kv), max(max(need), 1) + 1)).astype(np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, np.concatenate(([0], np.cumsum(fresh))).astype(np.int32), n_pages


def wide(table, page, keys):
    """The table with room for `keys` tokens a request: kernels are chosen by it."""
    return np.pad(table, ((0, 0), (0, max(0, keys // page - table.shape[1]))))


def fill(n_pages, nkv, page, d, seed, table=None, kv=None):
    """Codes and scales of normal values in every place that a token has, NaN scales (and codes of six) everywhere else."""
    rng = np.random.default_rng(seed)
    codes, scales = [], []
    for _ in range(2):
        pick = rng.integers(0, min(n_pages, 40), n_pages)        # pages drawn from a few that are encoded
        c, s = (a[pick] for a in ko.encode(rng.standard_normal((min(n_pages, 40), nkv, page, d))))
        used = np.zeros((n_pages, page), bool)
        for i, n in enumerate(kv):
            j = np.arange(min(max(int(n), 0), table.shape[1] * page))
            ok = (table[i, j // page] >= 0) & (table[i, j // page] < n_pages)
            used[table[i, j[ok] // page], j[ok] % page] = True
        c[~used.repeat(nkv, 0).reshape(n_pages, nkv, page)] = 0x77
        s[~used.repeat(nkv, 0).reshape(n_pages, nkv, page)] = 255
        codes.append(c)
        scales.append(s)
    return codes, scales


def attend(ctx, q, cache, table, row_start, kv, dt, nq, d, max_rows=None, stride=None, ws=None):
    rows = q.shape[0]
    stride = stride or nq * d
    qp = np.zeros((rows, stride), q.dtype)
    qp[:, : nq * d] = q.reshape(rows, -1)
    fresh = np.diff(row_start)
    out = iso.DeviceArray((rows, nq, d), dt, fill_byte=0xFF)
    n = ctx.attn_kv4_workspace(len(kv), rows)
    ws = ws or iso.DeviceArray((n,), "u8", fill_byte=0)
    ctx.attn_kv4(iso.DeviceArray.from_numpy(qp, dt), stride, cache, ints(table), table.shape[1], ints(row_start), ints(kv), len(kv), rows,
                 int(max_rows or max(1, fresh.max())), out, ws, n, ctx.stream0)
    ctx.sync()
    return out


def check(got, q, k, v, table, page, row_start, kv, group, dt, n_pages):
    rows, nq, d = q.shape
    ref, A, reach = ko.attention(q, k, v, table, page, row_start, kv, group, n_pages)
    u, keys = HALF_STEP[dt], max(1, max(kv))
    E = (d + 8) * 2.0 ** -24 * np.nan_to_num(reach)[..., None] * 1.4427 + 2.0 ** -22
    tol = u * np.abs(ref) + A * (u + 2 * E + (2 * keys + 16) * 2.0 ** -24)
    mine = ~np.isnan(A)
    err = np.abs(got - ref)
    assert (err[mine] <= tol[mine]).all(), float(np.nanmax(np.where(mine, err / np.maximum(tol, 1e-30), 0)))
    return ref


# head layouts: nq, nkv, head_dim
HEADS = [(8, 1, 128), (13, 13, 128), (16, 2, 128), (32, 8, 64), (4, 4, 64), (20, 1, 64), (3, 1, 128)]
# (kv_len, fresh) of every request, page
BATCHES = {
    "one_key": ([1], [1], 16),
    "few_keys": ([2, 15, 16, 17, 31, 32, 33], [1] * 7, 16),
    "tile_ends": ([63, 64, 65, 127, 128, 129, 255, 256, 257], [1] * 9, 32),
    "long": ([4099], [1], 64),
    "ragged": ([5, 900, 1, 2049, 333, 64], [1] * 6, 64),
    "drafts": ([700, 41, 1300], [2, 3, 5], 128),
    "prompts": ([7, 130, 33], [7, 130, 33], 16),
    "chunk": ([1100], [257], 256),
    "mixed": ([600, 90, 1025, 40, 1], [1, 90, 130, 0, 1], 64),
    "none": ([0, 40, 0, 3], [1, 0, 0, 5], 16),                  # a row without a token, a request without rows, more rows than tokens
}
FLAGS = [0, iso.ISO_FLAG_SIMPLE_ATTN]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("dt,heads", [("bf16", h) for h in HEADS] + [("f32", h) for h in ((4, 4, 64), (8, 2, 128), (20, 1, 64))])
def test_attention(dt, heads, name, flags):
    nq, nkv, d = heads
    kv, fresh, page = BATCHES[name]
    table, row_start, n_pages = batch(kv, fresh, page, seed=len(name))
    codes, scales = fill(n_pages, nkv, page, d, 7, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        ctx.set_flags(flags)
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, dt, nq, d), dt)
    ref = check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, dt, n_pages)
    if name == "none":
        assert (got[ref == 0] == 0).all() and (ref[0] == 0).all()


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("heads", HEADS)
def test_attention_through_a_table_with_room_for_more(heads, name):
    """What much work would be done by: 32 rows a tile, 128 for the longest chunks."""
    nq, nkv, d = heads
    kv, fresh, page = BATCHES[name]
    table, row_start, n_pages = batch(kv, fresh, page, seed=len(name))
    table = wide(table, page, 1 << 20)
    codes, scales = fill(n_pages, nkv, page, d, 7, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, d, "bf16") as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, "bf16", nq, d), "bf16")
    check(got, f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, "bf16", n_pages)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("dt,heads", [("bf16", (8, 1, 128)), ("bf16", (8, 8, 64)), ("f32", (4, 2, 64))])
@pytest.mark.parametrize("max_rows", [1, 7, 1000])
def test_rows_that_belong_to_no_request_and_pages_that_are_not_there(dt, heads, flags, max_rows):
    """Two rows in front, five behind stay as they were; entries that name no page hide their keys; any max_rows is right."""
    nq, nkv, d = heads
    kv, fresh, page = [300, 90, 450, 5], [1, 90, 40, 1], 32
    table, row_start, n_pages = batch(kv, fresh, page, seed=3)
    row_start = row_start + 2
    rows = int(row_start[-1]) + 5
    table[0, 3], table[1, 0], table[2, 5], table[2, 13], table[3, 0] = -1, n_pages, 2 ** 31 - 1, -2 ** 31, -1
    codes, scales = fill(n_pages, nkv, page, d, 8, table, kv)
    q = iso_inputs.randn((rows, nq, d), seed=4, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        ctx.set_flags(flags)
        out = attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, dt, nq, d, max_rows, stride=(nq + 2 * nkv) * d)
    got = f64(out, dt)
    ref = check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, dt, n_pages)
    assert (out.numpy().view(np.uint8).reshape(rows, -1)[[0, 1, *range(rows - 5, rows)]] == 0xFF).all()
    assert (ref[row_start[3]] == 0).all() and (got[row_start[3]] == 0).all()
    assert (ref[row_start[1]:row_start[1] + 32] == 0).all() and (got[row_start[1]:row_start[1] + 32] == 0).all()


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("dt,heads", [("bf16", (8, 1, 128)), ("bf16", (6, 2, 64)), ("f32", (4, 4, 64)), ("f32", (3, 1, 128))])
@pytest.mark.parametrize("kv,fresh,bad", [(200, 3, 198), (200, 40, 170), (700, 300, 555), (64, 64, 0), (65, 2, 64)])
def test_a_token_that_holds_nan_reaches_only_the_rows_that_see_it(dt, heads, flags, kv, fresh, bad):
    """Block 1 of V and, in the last kv head, block 0 of K of token `bad` are NaN."""
    nq, nkv, d = heads
    page = 32
    table, row_start, n_pages = batch([kv], [fresh], page, seed=5)
    codes, scales = fill(n_pages, nkv, page, d, 6, table, [kv])
    at = (table[0, bad // page], slice(None), bad % page)
    clean = [s.copy() for s in scales]
    scales[1][at][:, 1] = 255
    scales[0][table[0, bad // page], nkv - 1, bad % page, 0] = 255
    q = iso_inputs.randn((fresh, nq, d), seed=4, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        ctx.set_flags(flags)
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, [kv], dt, nq, d), dt)
    sees = max(0, bad - (kv - fresh))                           # first row that sees it
    assert np.isnan(got[sees:, :, 32:64]).all()
    last = slice(nq - nq // nkv, nq)
    assert np.isnan(got[sees:, last]).all()
    k, v = ko.decode(codes[0], clean[0]), ko.decode(codes[1], clean[1])
    without = ko.attention(f64(q, dt), k, v, table, page, row_start, [kv], nq // nkv)[0]
    check(np.where(np.isnan(got), without, got), f64(q, dt), k, v, table, page, row_start, [kv], nq // nkv, dt, n_pages)
    assert not np.isnan(got[:sees]).any()
    if nkv > 1:
        assert not np.isnan(got[:, : nq - nq // nkv, :32]).any()


# ------------------------------------------------------------------------------------------------ long chunks: tiles of 128 rows

# rows x query heads from 4096 on, and tables with room for many keys: head layouts with many heads reach it with few rows
MANY = [(64, 1, 64), (64, 64, 64), (64, 2, 128), (66, 22, 128), (104, 8, 64)]
LONG = {
    "fresh": ([256], [256], 64),
    "odd": ([1301], [257], 16),
    "two": ([290, 1000], [290, 259], 256),
    "mixed": ([700, 40, 1, 901, 77, 0], [300, 1, 1, 2, 0, 3], 32),
    "short_of_tokens": ([100], [256], 64),                       # the first 156 rows see nothing
}


@pytest.mark.parametrize("heads", MANY)
@pytest.mark.parametrize("name", LONG)
def test_long_chunks(heads, name):
    nq, nkv, d = heads
    kv, fresh, page = LONG[name]
    table, row_start, n_pages = batch(kv, fresh, page, seed=len(name))
    table = wide(table, page, 8192)
    codes, scales = fill(n_pages, nkv, page, d, 7, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, d, "bf16") as ctx:
        cache = device_cache(codes, scales, page)
        ws = iso.DeviceArray((ctx.attn_kv4_workspace(len(kv), q.shape[0]),), "u8", fill_byte=0)
        out = [attend(ctx, q, cache, table, row_start, kv, "bf16", nq, d, ws=ws).numpy() for _ in range(3)]
    np.testing.assert_array_equal(out[0], out[1])                # the workspace is left ready, the order of arrivals does not show
    np.testing.assert_array_equal(out[0], out[2])
    ref = check(f64(out[0], "bf16"), f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv,
                nq // nkv, "bf16", n_pages)
    assert (f64(out[0], "bf16")[(ref == 0).all((1, 2))] == 0).all()


@pytest.mark.parametrize("heads", [(64, 1, 64), (64, 2, 128)])
@pytest.mark.parametrize("kv,fresh,bad", [(900, 260, 700), (900, 260, 30), (256, 256, 0)])
def test_long_chunks_with_a_nan_and_missing_pages(heads, kv, fresh, bad):
    nq, nkv, d = heads
    page = 16
    table, row_start, n_pages = batch([kv], [fresh], page, seed=5)
    table, row_start = wide(table, page, 8192), row_start + 1
    gone = [2, 9] if kv > 300 else [5]
    table[0, gone] = [-1, n_pages][: len(gone)]
    codes, scales = fill(n_pages, nkv, page, d, 6, table, [kv])
    clean = scales[1].copy()
    scales[1][table[0, bad // page], :, bad % page, 1] = 255
    q = iso_inputs.randn((fresh + 3, nq, d), seed=4, dtype="bf16")
    with make_ctx(nq, nkv, d, "bf16") as ctx:
        out = attend(ctx, q, device_cache(codes, scales, page), table, row_start, [kv], "bf16", nq, d)
    got = f64(out, "bf16")
    sees = 1 + max(0, bad - (kv - fresh))
    assert np.isnan(got[sees:-2, :, 32:64]).all() and not np.isnan(got[1:sees]).any()
    k, v = ko.decode(codes[0], scales[0]), ko.decode(codes[1], clean)
    without = ko.attention(f64(q, "bf16"), k, v, table, page, row_start, [kv], nq // nkv, n_pages)[0]
    inside = np.where(np.isnan(got), without, got)
    check(inside, f64(q, "bf16"), k, v, table, page, row_start, [kv], nq // nkv, "bf16", n_pages)
    assert (out.numpy().view(np.uint8).reshape(fresh + 3, -1)[[0, -2, -1]] == 0xFF).all()
    assert not np.isnan(got[1:-2, :, :32]).any()


@pytest.mark.parametrize("dt,heads", [("bf16", (8, 1, 128)), ("bf16", (3, 3, 128)), ("bf16", (16, 4, 64)), ("f32", (4, 2, 64))])
@pytest.mark.parametrize("room", [0, 1 << 20])
@pytest.mark.parametrize("kv,fresh", [([40000], [1]), ([9000, 3, 20011], [1, 1, 6]), ([900] * 33, [1] * 33)])
def test_many_pieces_and_one_workspace_for_all(dt, heads, kv, fresh, room):
    """Keys dealt to hundreds of workgroups and folded in two rounds; calls of other shapes on the same workspace in between."""
    nq, nkv, d = heads
    page = 64
    table, row_start, n_pages = batch(kv, fresh, page, seed=2)
    table = wide(table, page, room)
    codes, scales = fill(n_pages, nkv, page, d, 3, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype=dt)
    other = batch([300, 77], [40, 1], page, seed=4)
    with make_ctx(nq, nkv, d, dt) as ctx:
        cache = device_cache(codes, scales, page)
        ws = iso.DeviceArray((max(ctx.attn_kv4_workspace(len(kv), q.shape[0]), ctx.attn_kv4_workspace(2, 41)),), "u8", fill_byte=0)
        out = []
        for _ in range(3):
            out.append(attend(ctx, q, cache, table, row_start, kv, dt, nq, d, ws=ws).numpy())
            attend(ctx, iso_inputs.randn((41, nq, d), seed=1, dtype=dt), cache, other[0] % n_pages, other[1], [300, 77], dt, nq, d, ws=ws)
    np.testing.assert_array_equal(out[0], out[1])
    np.testing.assert_array_equal(out[0], out[2])
    check(f64(out[0], dt), f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, dt, n_pages)


@pytest.mark.parametrize("n_seqs", [64, 65, 200, 4096])
def test_many_requests(n_seqs):
    """More requests than a wave has lanes; every third has no row, lengths from one."""
    nq, nkv, d, page, dt = 4, 2, 64, 16, "bf16"
    rng = np.random.default_rng(n_seqs)
    kv = rng.integers(1, 60, n_seqs)
    fresh = np.where(np.arange(n_seqs) % 3 == 1, 0, np.minimum(kv, rng.integers(1, 4, n_seqs)))
    table, row_start, n_pages = batch(list(kv), list(fresh), page, seed=1)
    codes, scales = fill(n_pages, nkv, page, d, 3, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, list(kv), dt, nq, d), dt)
    check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, list(kv), nq // nkv, dt, n_pages)
