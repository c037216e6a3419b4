"""Ragged batches through every attention kernel of the 4-bit cache: more requests than a wave has lanes, long chunks beside single tokens
for any number of query heads a key head, row tiles folded from many pieces (bounds: see test_gpu_kv4.py)."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_graph import Captured, hip_runtime
from test_gpu_kv4 import attend, batch, check, device_cache, f64, fill, ints, make_ctx, wide

pytestmark = pytest.mark.gpu


def several(nq, nkv, d, kv, fresh, page, room, launches, dt="bf16", seed=7):
    """Three calls on one workspace give the same, within the bounds, in as many launches each as they should have."""
    table, row_start, n_pages = batch(kv, fresh, page, seed=seed)
    table = wide(table, page, room)
    codes, scales = fill(n_pages, nkv, page, d, seed, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, d), seed=9, dtype=dt)
    with make_ctx(nq, nkv, d, dt) as ctx:
        cache = device_cache(codes, scales, page)
        ws = iso.DeviceArray((ctx.attn_kv4_workspace(len(kv), q.shape[0]),), "u8", fill_byte=0)
        ctx.timing_enable(True)
        out = [attend(ctx, q, cache, table, row_start, kv, dt, nq, d, ws=ws).numpy() for _ in range(3)]
        assert ctx.timing_read()["attn"][1] == 3 * launches
    np.testing.assert_array_equal(out[0], out[1])
    np.testing.assert_array_equal(out[0], out[2])
    check(f64(out[0], dt), f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, dt, n_pages)


# Query heads a key head: 1, 3 (does not divide 128), 5, 8, 33.  A request belongs to the tiles of 128 rows from 1024 (row, query head)
# pairs of a key head on: LONG rows; the ones below it, one short, stay with the line.
LAYOUTS = [(4, 4, 64), (4, 4, 128), (6, 2, 128), (6, 2, 64), (10, 2, 64), (8, 1, 128), (33, 1, 128), (66, 2, 64)]


@pytest.mark.parametrize("nq,nkv,d", LAYOUTS)
@pytest.mark.parametrize("order", ["long_first", "long_last", "between"])
def test_long_chunks_beside_short_requests(nq, nkv, d, order):
    least = 1023 // (nq // nkv) + 1
    longest = max(least + 190, 4096 // nq + 1)
    long_ = [(longest + 300, longest), (least + 75, least)]
    short = [(700, 1), (40, 3), (0, 0), (least + 9, least - 1), (1, 1), (33, 0)]
    if order == "long_first":
        requests = long_ + short
    elif order == "long_last":
        requests = short + long_
    else:
        requests = short[:2] + long_[:1] + short[2:5] + long_[1:] + short[5:]
    kv, fresh = (list(x) for x in zip(*requests))
    several(nq, nkv, d, kv, fresh, 32, 1 << 16, launches=2)


@pytest.mark.parametrize("nq,nkv,d,n_seqs,fresh_of,room,launches", [
    (64, 1, 64, 65, (1, 0, 20, 70, 3), 1 << 16, 2),              # the line and tiles of 128 rows, long requests beyond the first 64 too
    (64, 1, 64, 150, (1, 0, 0, 16, 15, 70, 2), 1 << 16, 2),
    (64, 2, 128, 130, (0, 64, 1, 32, 31), 1 << 16, 2),
    (8, 1, 128, 150, (1, 0, 5, 9, 2), 1 << 16, 1),               # 32 rows a tile
    (8, 2, 64, 200, (1, 0, 5, 9, 2), 0, 1),
    (8, 1, 128, 150, (1, 0, 2), 0, 1),                           # 16 rows a tile, heads of 128
    (8, 1, 128, 4096, (1, 0, 0, 3), 1 << 12, 1),
])
def test_more_requests_than_a_wave_has_lanes(nq, nkv, d, n_seqs, fresh_of, room, launches):
    rng = np.random.default_rng(n_seqs)
    fresh = [fresh_of[i % len(fresh_of)] for i in range(n_seqs)]
    kv = [int(f + rng.integers(0, 40)) for f in fresh]
    several(nq, nkv, d, kv, fresh, 16, room, launches)


def test_more_fp32_requests_than_a_wave_has_lanes():
    rng = np.random.default_rng(1)
    fresh = [(1, 0, 5, 2)[i % 4] for i in range(130)]
    several(8, 2, 128, [int(f + rng.integers(0, 90)) for f in fresh], fresh, 16, 0, 1, dt="f32")


@pytest.mark.parametrize("nq,nkv,d,kv,fresh", [(64, 1, 64, [40000], [64]), (16, 1, 128, [20011], [257]), (32, 2, 128, [9000], [129]),
                                               (64, 1, 64, [30000, 77, 21000], [70, 1, 64])])
def test_long_chunks_folded_from_many_pieces(nq, nkv, d, kv, fresh):
    """Tiles of 128 rows are cut into up to 17 pieces: 512 workgroups to a line of 32 tiles."""
    several(nq, nkv, d, kv, fresh, 64, 0, launches=1 if len(kv) == 1 else 2)


@pytest.mark.parametrize("others", [([300, 77], [40, 1]), ([2000], [600]), ([9000], [1]), ([30] * 100, [1] * 100)])
def test_calls_of_other_shapes_between_replays_on_the_graphs_workspace(others):
    """A recorded step is replayed; between the replays the program makes calls of another shape on the same workspace: single tokens and
    chunks, 16, 32 and 128 rows a tile, hundreds of pieces."""
    dt, nq, nkv, d, page = "bf16", 8, 1, 128, 64
    kv, fresh = [20000, 500, 3000], [1, 2, 1]
    table, row_start, n_pages = batch(kv, fresh, page, seed=2)
    codes, scales = fill(n_pages, nkv, page, d, 3, table, kv)
    rows = int(row_start[-1])
    q = iso_inputs.randn((rows, nq, d), seed=1, dtype=dt)
    table2, row_start2, n2 = batch(*others, page, seed=4)
    table2, rows2 = wide(table2 % n_pages, page, 1 << 15), int(row_start2[-1])
    q2 = iso_inputs.randn((rows2, nq, d), seed=5, dtype=dt)
    rt = hip_runtime()
    with make_ctx(nq, nkv, d, dt) as ctx:
        cache = device_cache(codes, scales, page)
        alone = attend(ctx, q, cache, table, row_start, kv, dt, nq, d).numpy()
        alone2 = attend(ctx, q2, cache, table2, row_start2, others[0], dt, nq, d).numpy()
        n = max(ctx.attn_kv4_workspace(len(kv), rows), ctx.attn_kv4_workspace(len(others[0]), rows2))
        ws, out = iso.DeviceArray((n,), "u8", fill_byte=0), iso.DeviceArray((rows, nq, d), dt)
        qd, td, sd, kd = iso.DeviceArray.from_numpy(q, dt), ints(table), ints(row_start), ints(kv)

        def call():
            ctx.attn_kv4(qd, nq * d, cache, td, table.shape[1], sd, kd, len(kv), rows, max(fresh), out, ws, n, ctx.stream0)

        graph = Captured(rt, ctx.stream0.handle, call)
        for _ in range(5):
            out.fill(0xFF)
            graph.launch()
            ctx.sync()
            np.testing.assert_array_equal(out.numpy(), alone)
            got = attend(ctx, q2, cache, table2, row_start2, others[0], dt, nq, d, ws=ws).numpy()
            np.testing.assert_array_equal(got, alone2)
        graph.destroy()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_prefilled_prompt_and_its_next_chunk_element_by_element(dt, d):
    """A layer's cache rows stored, a chunk written behind them, and attention to both: each element within the bounds of one attention
    over the values that the pages hold."""
    hidden, nq, nkv, ffn, T, C, page = 256, 8, 2, 128, 300, 37, 32
    w = iso_inputs.make_layer(hidden, nq, nkv, d, ffn, seed=3, dtype=dt)
    kv = T + C
    with iso.Context(iso.make_cfg(hidden, nq, nkv, d, ffn, dt, kv)) as ctx:
        x = iso.DeviceArray.from_numpy(iso_inputs.make_hidden(T, hidden, seed=3, dtype=dt), dt)
        kc, vc = (iso.DeviceArray((kv, nkv, d), dt, fill_byte=0) for _ in range(2))
        ctx.layer_prefill(iso.upload_weights(w, dt), x, kc, vc, T, 0, iso.ISO_COMM_NONE)
        cache = ctx.kv4_cache(20, page, fill_byte=0xFF)
        free = np.random.default_rng(0).permutation(20)
        table, head = ints(np.full((1, 12), -1)), None
        lens, start = [ints([0])], None
        every = []
        for n in (T, C):
            start, new, pos, slots, nxt = (ints(np.full(s, -1)) for s in (2, 1, n, n, 1))
            ctx.block_tables(lens[-1], ints([n]), 1, page, ints(free), 20, head, table, 12, start, new, pos, slots, n, nxt, ctx.stream0)
            lens.append(new)
            if n == T:
                ctx.kv4_store(kc, vc, cache, slots, T, ctx.stream0)
            else:
                qkv = iso.DeviceArray.from_numpy(iso_inputs.randn((C, nq + 2 * nkv, d), seed=8, dtype=dt), dt)
                q = iso.DeviceArray((C, nq, d), dt)
                ctx.rope_kv4_write(qkv, q, cache, pos, slots, C, ctx.stream0)
            head = nxt
            ctx.sync()
            every.append(slots.numpy())
        out = iso.DeviceArray((C, nq, d), dt, fill_byte=0xFF)
        size = ctx.attn_kv4_workspace(1, C)
        ws = iso.DeviceArray((size,), "u8", fill_byte=0)
        ctx.attn_kv4(q, nq * d, cache, table, 12, start, lens[-1], 1, C, C, out, ws, size, ctx.stream0)
        ctx.sync()
        vals = [ko.decode(c.numpy(), s.numpy()) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        got, q, tb = f64(out, dt), f64(q, dt), table.numpy()
        rows = [f64(a, dt)[:T] for a in (kc, vc)]
    slots = np.concatenate(every)
    np.testing.assert_array_equal(tb[0, np.arange(kv) // page] * page + np.arange(kv) % page, slots)
    for val, x in zip(vals, rows):
        np.testing.assert_array_equal(val[slots[:T] // page, :, slots[:T] % page], ko.decode(*ko.encode(x)))
    check(got, q, vals[0], vals[1], tb, page, [0, C], [kv], nq // nkv, dt, 20)
