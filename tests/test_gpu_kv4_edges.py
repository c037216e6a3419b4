"""The paged 4-bit cache where its sizes end: caches of more than 4 GB, page numbers that no cache can have, many heads, keys that are
NaN, fewer rows than the requests have."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_kv4 import FLAGS, attend, batch, check, device_cache, f64, fill, ints, make_ctx, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,nq,d,kv,fresh", [("bf16", 8, 128, 600, 1), ("bf16", 8, 128, 600, 5), ("bf16", 64, 128, 700, 260), ("f32", 4, 128, 600, 2),
                                              ("bf16", 16, 64, 500, 1), ("bf16", 64, 64, 600, 300)])
def test_a_cache_of_more_than_4_GB(dt, nq, d, kv, fresh):
    """Pages on both sides of the places where the codes' offsets pass 2^31 and 2^32 bytes, and the last one."""
    page = 16
    per_page = page * d // 2
    ends = [2 ** 31 // per_page, 2 ** 32 // per_page]
    n_pages = ends[1] + 100
    need = -(-kv // page)
    pages = np.unique(np.concatenate([[0, n_pages - 1]] + [np.arange(e - 6, e + 6) for e in ends] + [np.arange(need)]))[::-1][:need]
    pages = np.random.default_rng(kv).permutation(pages).astype(np.int32)
    assert len(pages) == need and {ends[0] - 1, ends[0], ends[1] - 1, ends[1], n_pages - 1} <= set(pages.tolist())
    tok = np.arange(need * page)
    slots = pages[tok // page] * page + tok % page
    rng = np.random.default_rng(1)
    k, v = (iso_inputs.store(rng.standard_normal((need * page, 1, d)).astype(np.float32), dt) for _ in range(2))
    q = iso_inputs.randn((fresh, nq, d), seed=9, dtype=dt)
    with make_ctx(nq, 1, d, dt) as ctx:
        cache = ctx.kv4_cache(n_pages, page)
        sd = ints(slots)
        ctx.kv4_store(iso.DeviceArray.from_numpy(k, dt), iso.DeviceArray.from_numpy(v, dt), cache, sd, len(slots), ctx.stream0)
        back = [iso.DeviceArray((len(slots), 1, d), dt, fill_byte=0xFF) for _ in range(2)]
        ctx.kv4_load(cache, sd, back[0], back[1], len(slots), ctx.stream0)
        out = iso.DeviceArray((fresh, nq, d), dt, fill_byte=0xFF)
        n = ctx.attn_kv4_workspace(1, fresh)
        ws = iso.DeviceArray((n,), "u8", fill_byte=0)
        ctx.attn_kv4(iso.DeviceArray.from_numpy(q, dt), nq * d, cache, ints(wide(pages[None], page, 1 << 20)), (1 << 20) // page, ints([0, fresh]), ints([kv]), 1, fresh, fresh, out, ws, n,
                     ctx.stream0)
        ctx.sync()
        got, rows = f64(out, dt), [f64(b, dt) for b in back]
    vals = [ko.decode(*ko.encode(f64(x, dt))) for x in (k, v)]
    for r, w in zip(rows, vals):
        np.testing.assert_array_equal(r, w)
    kk, vv = (x.reshape(need, page, 1, d).transpose(0, 2, 1, 3) for x in vals)
    check(got, f64(q, dt), kk, vv, np.arange(need, dtype=np.int32)[None], page, [0, fresh], [kv], nq, dt, need)


def test_page_numbers_whose_slots_pass_31_bits_are_no_pages():
    page, most = 64, 2 ** 31 // 64
    free = np.array([most - 1, most, 2 ** 31 - 1, 5], np.int32)
    table = np.array([[most, -9, -9], [most - 1, -9, -9]], np.int32)
    with make_ctx(4, 4, 64, "f32") as ctx:
        td, start, lens, pos, slots, nxt = (ints(a) for a in (table, [0] * 3, [0] * 2, [-5] * 200, [-5] * 200, [0]))
        ctx.block_tables(ints([60, 62]), ints([100, 70]), 2, page, ints(free), 4, None, td, 3, start, lens, pos, slots, 200, nxt, ctx.stream0)
        ctx.sync()
        got = slots.numpy()
    want = np.full(200, -1, np.int64)
    p = np.arange(60, 160)
    want[:100] = np.where(p // page == 1, (most - 1) * page + p % page, -1)
    p = np.arange(62, 132)
    want[100:170] = np.select([p // page == 0, p // page == 2], [(most - 1) * page + p % page, 5 * page + p % page], -1)
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("nq,nkv,d", [(130, 1, 64), (200, 2, 64), (65, 1, 128)])
@pytest.mark.parametrize("kv,fresh", [([70, 1, 500], [1, 1, 1]), ([300, 40], [260, 2])])
def test_more_than_64_query_heads_of_a_key_head(nq, nkv, d, kv, fresh):
    table, row_start, n_pages = batch(kv, fresh, 32, seed=1)
    codes, scales = fill(n_pages, nkv, 32, d, 7, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, d, "bf16") as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, 32), table, row_start, kv, "bf16", nq, d), "bf16")
    check(got, f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, 32, row_start, kv, nq // nkv, "bf16", n_pages)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("dt,nq,nkv,d", [("bf16", 8, 1, 128), ("bf16", 64, 1, 128), ("bf16", 64, 1, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("kv,fresh,bad", [(900, 260, 700), (900, 1, 899), (700, 3, 698), (64, 64, 0)])
def test_a_key_that_is_nan_reaches_the_rows_that_see_it_whole_and_no_others(dt, nq, nkv, d, kv, fresh, bad, flags):
    page = 16
    table, row_start, n_pages = batch([kv], [fresh], page, seed=5)
    table = wide(table, page, 8192)
    codes, scales = fill(n_pages, nkv, page, d, 6, table, [kv])
    clean = scales[0].copy()
    scales[0][table[0, bad // page], :, bad % page, 0] = 255
    q = iso_inputs.randn((fresh, nq, d), seed=4, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        ctx.set_flags(flags)
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, [kv], dt, nq, d), dt)
    sees = max(0, bad - (kv - fresh))
    assert np.isnan(got[sees:]).all() and not np.isnan(got[:sees]).any()
    if sees:
        k, v = ko.decode(codes[0], clean), ko.decode(codes[1], scales[1])
        ref = ko.attention(f64(q, dt), k, v, table, page, row_start, [kv], nq // nkv, n_pages)[0]
        check(np.concatenate((got[:sees], ref[sees:])), f64(q, dt), k, v, table, page, row_start, [kv], nq // nkv, dt, n_pages)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("dt,nq,nkv,d", [("bf16", 8, 1, 128), ("bf16", 64, 1, 128), ("f32", 4, 2, 64)])
def test_rows_past_the_last_that_the_call_has(dt, nq, nkv, d, flags):
    """row_start ends at 420, the call has 300 rows: the second request's are cut, the third has none; the others are as ever."""
    kv, fresh, page, rows = [500, 333, 90], [257, 120, 43], 32, 300
    table, row_start, n_pages = batch(kv, fresh, page, seed=3)
    table = wide(table, page, 8192)
    codes, scales = fill(n_pages, nkv, page, d, 6, table, kv)
    q = iso_inputs.randn((rows, nq, d), seed=4, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        ctx.set_flags(flags)
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, dt, nq, d), dt)
    check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, dt, n_pages)
