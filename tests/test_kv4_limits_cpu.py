"""Where the calls around the 4-bit cache end, without a GPU: sizes, buffers and types that they refuse, kernels that they leave out
(the library's HIP calls go to tests/fake_hip.cpp)."""
from test_host_side_cpu import fake, run                       # noqa: F401  (fixture)


def test_tables_with_room_for_more_keys_than_are_counted_in_31_bits(fake):       # noqa: F811
    """The kernels' key counters run some 300 past the last key (tiles requested ahead), so a table ends 1024 short of 2^31 tokens."""
    run(fake, """
for dt, flags in (("bf16", 0), ("bf16", iso.ISO_FLAG_SIMPLE_ATTN), ("f32", 0)):
    with iso.Context(iso.make_cfg(64, 64, 1, 64, 64, dt, 256)) as ctx:
        ctx.set_flags(flags)
        i = iso.DeviceArray((64,), "i32")
        q, out = (iso.DeviceArray((64, 64, 64), dt) for _ in range(2))
        n = ctx.attn_kv4_workspace(1, 64)
        ws = iso.DeviceArray((n,), "u8")
        for page in (16, 64, 256):
            cache = ctx.kv4_cache(4, page)
            for rows in (1, 64):
                for pages, ok in (((2 ** 31 - 1024) // page, True), ((2 ** 31 - 1024) // page + 1, False), (2 ** 31 // page, False), (2 ** 31 - 1, False)):
                    log()
                    try:
                        ctx.attn_kv4(q, 64 * 64, cache, i, pages, i, i, 1, rows, rows, out, ws, n)
                        assert ok, (page, rows, pages)
                        assert len([l for l in log() if l[0] == "kernel"]) == 1
                    except iso.IsoError as e:
                        assert not ok and e.code == -2 and "at most 2147482624 tokens" in str(e), (page, rows, pages, e)
                        assert log() == []
""")
