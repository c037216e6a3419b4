"""The calls around the 4-bit cache as a program uses them: after a prefill, step after step, recorded into graphs, on several streams."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_graph import Captured, hip_runtime
from test_gpu_kv4 import HALF_STEP, attend, batch, check, device_cache, f64, fill, ints, make_ctx, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_from_a_prefilled_prompt_to_the_next_chunk(dt):
    """A layer's cache rows go into pages; a chunk of further tokens attends to the pages as the framework's own chunk attention does to
    the same values loaded back into rows (bound: both round their probabilities and results, twice the half steps of the type)."""
    hidden, nq, nkv, d, ffn, T, C, page = 256, 8, 2, 64, 128, 300, 37, 32
    w = iso_inputs.make_layer(hidden, nq, nkv, d, ffn, seed=3, dtype=dt)
    kv = T + C
    with iso.Context(iso.make_cfg(hidden, nq, nkv, d, ffn, dt, kv)) as ctx:
        x = iso.DeviceArray.from_numpy(iso_inputs.make_hidden(T, hidden, seed=3, dtype=dt), dt)
        kc, vc = (iso.DeviceArray((kv, nkv, d), dt, fill_byte=0) for _ in range(2))
        ctx.layer_prefill(iso.upload_weights(w, dt), x, kc, vc, T, 0, iso.ISO_COMM_NONE)
        cache = ctx.kv4_cache(20, page, fill_byte=0xFF)
        free = np.random.default_rng(0).permutation(20)
        table, start, lens, pos, slots, nxt = (ints(np.full(s, -1)) for s in ((1, 12), 2, 1, T, T, 1))
        zero = ints([0])
        ctx.block_tables(zero, ints([T]), 1, page, ints(free), 20, None, table, 12, start, lens, pos, slots, T, nxt, ctx.stream0)
        ctx.kv4_store(kc, vc, cache, slots, T, ctx.stream0)
        # the chunk: its rows as a projection would leave them
        qkv = iso_inputs.randn((C, nq + 2 * nkv, d), seed=8, dtype=dt)
        qd, qo = iso.DeviceArray.from_numpy(qkv, dt), iso.DeviceArray((C, nq, d), dt)
        start2, lens2, pos2, slots2, nxt2 = (ints(np.full(s, -1)) for s in (2, 1, C, C, 1))
        ctx.block_tables(lens, ints([C]), 1, page, ints(free), 20, nxt, table, 12, start2, lens2, pos2, slots2, C, nxt2, ctx.stream0)
        ctx.rope_kv4_write(qd, qo, cache, pos2, slots2, C, ctx.stream0)
        out = iso.DeviceArray((C, nq, d), dt, fill_byte=0xFF)
        n = ctx.attn_kv4_workspace(1, C)
        ws = iso.DeviceArray((n,), "u8", fill_byte=0)
        ctx.attn_kv4(qo, nq * d, cache, table, 12, start2, lens2, 1, C, C, out, ws, n, ctx.stream0)
        # the same values as rows
        rows = [iso.DeviceArray((kv, nkv, d), dt) for _ in range(2)]
        ctx.sync()
        every = np.concatenate((slots.numpy(), slots2.numpy()))
        assert sorted(set(every // page)) == sorted(free[: -(-kv // page)]) and len(set(every)) == kv
        ctx.kv4_load(cache, ints(every), rows[0], rows[1], kv, ctx.stream0)
        ref = iso.DeviceArray((C, nq * d), dt, fill_byte=0xFF)
        ctx.attn_chunk(qo, rows[0], rows[1], ref, C, T, kv, ctx.stream0)
        ctx.sync()
        got, ref = f64(out, dt).reshape(C, -1), f64(ref, dt)
        v = f64(rows[1], dt)
    u = HALF_STEP[dt] if dt == "bf16" else 2.0 ** -18          # fp32: accumulation over 337 keys and 64 dims on both sides
    assert np.abs(got - ref).max() <= 4 * u * np.abs(v).max()
    assert int(lens2.numpy()[0]) == kv and int(nxt2.numpy()[0]) == -(-kv // page)


def test_steps_recorded_into_two_graphs_that_hand_over_to_each_other():
    """One decoding step: tables, write, attention.  Two recordings, one reading what the other leaves (lengths, head of the free list),
    are replayed in turn; lengths grow through pages and through a change of the number of pieces.  Every step against the oracle, with
    eager work on the same stream in between."""
    dt, nq, nkv, d, page, B = "bf16", 8, 2, 64, 16, 3
    first, steps, width = [700, 15, 0], 24, 64
    rng = np.random.default_rng(1)
    n_pages = 80
    order = rng.permutation(n_pages)
    have = [-(-n // page) for n in first]
    table, at = np.full((B, width), -1), 0
    for i, n in enumerate(have):
        table[i, :n] = order[at:at + n]
        at += n
    free = order[at:]
    codes, scales = fill(n_pages, nkv, page, d, 4, table, first)
    qkv = [iso_inputs.randn((B, nq + 2 * nkv, d), seed=s, dtype=dt) for s in range(steps)]
    rt = hip_runtime()
    with make_ctx(nq, nkv, d, dt, max_seq=width * page) as ctx:
        cache = device_cache(codes, scales, page)
        td, fd, one = ints(table), ints(free), ints([1] * B)
        lens, heads = [ints(first), ints([0] * B)], [ints([0]), ints([0])]
        start, pos, slots = ints([0] * (B + 1)), ints([0] * B), ints([0] * B)
        x, q, out = (iso.DeviceArray((B, n, d), dt, fill_byte=0) for n in (nq + 2 * nkv, nq, nq))
        n = ctx.attn_kv4_workspace(B, B)
        ws = iso.DeviceArray((n,), "u8", fill_byte=0)

        def step(a, b):
            ctx.block_tables(lens[a], one, B, page, fd, len(free), heads[a], td, width, start, lens[b], pos, slots, B, heads[b], ctx.stream0)
            ctx.rope_kv4_write(x, q, cache, pos, slots, B, ctx.stream0)
            ctx.attn_kv4(q, nq * d, cache, td, width, start, lens[b], B, B, 1, out, ws, n, ctx.stream0)

        graphs = [Captured(rt, ctx.stream0.handle, lambda a=a: step(a, 1 - a)) for a in (0, 1)]
        assert [g.nodes() for g in graphs] == [3, 3]
        want_table, kv, head = table, list(first), 0
        for s in range(steps):
            x.upload(qkv[s])
            graphs[s % 2].launch()
            ctx.sync()
            want_table, want_start, want_kv, want_pos, want_slots, head = ko.block_tables(kv, [1] * B, page, free, head, want_table, B)
            kv = list(want_kv)
            np.testing.assert_array_equal(td.numpy(), want_table)
            np.testing.assert_array_equal(lens[1 - s % 2].numpy(), want_kv)
            np.testing.assert_array_equal(slots.numpy(), want_slots)
            assert int(heads[1 - s % 2].numpy()[0]) == head
            vals = [ko.decode(c.numpy(), sc.numpy()) for c, sc in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
            rot = ko.rotate(f64(qkv[s], dt)[:, nq:nq + nkv], want_pos)
            np.testing.assert_array_equal(vals[0][want_slots // page, :, want_slots % page], ko.decode(*ko.encode(rot)))
            check(f64(out, dt), f64(q, dt), vals[0], vals[1], want_table, page, want_start, kv, nq // nkv, dt, n_pages)
            # the program's own work on the stream and on the same workspace
            attend(ctx, iso_inputs.randn((41, nq, d), seed=s, dtype=dt), cache, *batch([300, 77], [40, 1], page, seed=s)[:2], [300, 77], dt, nq, d, ws=None)
            if s % 3 == 0:
                ctx.attn_kv4(q, nq * d, cache, td, width, start, lens[1 - s % 2], B, B, 1, out, ws, n, ctx.stream0)
        for g in graphs:
            g.destroy()


@pytest.mark.parametrize("shape", ["line", "rows"])
def test_two_streams_with_a_workspace_each(shape):
    """Calls that overlap in time on streams of the caller's, one recorded and replayed, give what they give alone."""
    dt, page = "bf16", 64
    nq, nkv, d, kv, fresh = (8, 1, 128, [20000, 500], [1, 2]) if shape == "line" else (64, 2, 128, [900], [300])
    table, row_start, n_pages = batch(kv, fresh, page, seed=2)
    table = wide(table, page, 8192 if shape == "rows" else 0)
    codes, scales = fill(n_pages, nkv, page, d, 3, table, kv)
    rows = int(row_start[-1])
    qs = [iso_inputs.randn((rows, nq, d), seed=s, dtype=dt) for s in (1, 2)]
    rt = hip_runtime()
    with make_ctx(nq, nkv, d, dt) as ctx:
        cache = device_cache(codes, scales, page)
        alone = [attend(ctx, q, cache, table, row_start, kv, dt, nq, d).numpy() for q in qs]
        n = ctx.attn_kv4_workspace(len(kv), rows)
        streams = [iso.Stream(), iso.Stream()]
        td, sd, kd = ints(table), ints(row_start), ints(kv)
        qd = [iso.DeviceArray.from_numpy(q, dt) for q in qs]
        ws = [iso.DeviceArray((n,), "u8", fill_byte=0) for _ in range(2)]
        out = [iso.DeviceArray((rows, nq, d), dt, fill_byte=0xFF) for _ in range(2)]

        def call(i):
            ctx.attn_kv4(qd[i], nq * d, cache, td, table.shape[1], sd, kd, len(kv), rows, max(fresh), out[i], ws[i], n, streams[i])

        call(1)
        iso.device_sync()
        graph = Captured(rt, streams[1].handle, lambda: call(1))
        for _ in range(4):
            for o in out:
                o.fill(0xFF)
            for _ in range(5):
                call(0)
                graph.launch()
            iso.device_sync()
            for o, a in zip(out, alone):
                np.testing.assert_array_equal(o.numpy(), a)
        graph.destroy()


def test_timing_records_the_calls():
    nq, nkv, d, page, dt = 4, 2, 64, 16, "bf16"
    with make_ctx(nq, nkv, d, dt) as ctx:
        table, row_start, n_pages = batch([40], [1], page, seed=2)
        codes, scales = fill(n_pages, nkv, page, d, 3, table, [40])
        cache = device_cache(codes, scales, page)
        ctx.timing_enable(True)
        attend(ctx, iso_inputs.randn((1, nq, d), seed=1, dtype=dt), cache, table, row_start, [40], dt, nq, d)
        rows = iso.DeviceArray((1, nkv, d), dt, fill_byte=0)
        ctx.kv4_store(rows, rows, cache, ints([0]), 1, ctx.stream0)
        ctx.kv4_load(cache, ints([0]), rows, iso.DeviceArray((1, nkv, d), dt), 1, ctx.stream0)
        ctx.block_tables(ints([0]), ints([1]), 1, page, ints([0]), 1, None, ints([[0]]), 1, ints([0, 0]), ints([0]), ints([0]), ints([0]), 1, ints([0]), ctx.stream0)
        ctx.rope_kv4_write(iso.DeviceArray((1, nq + 2 * nkv, d), dt, fill_byte=0), None, cache, ints([0]), ints([0]), 1, ctx.stream0)
        t = ctx.timing_read()
        assert [t[k][1] for k in ("attn", "quant", "tables", "rope_kv")] == [1, 2, 1, 1]
