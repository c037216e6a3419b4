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


def test_more_rows_than_a_launch_has_lanes_for(fake):          # noqa: F811
    """Every launch that is let through has fewer than 2^32 lanes.  (No memory is touched: the addresses are far apart and nowhere.)"""
    run(fake, """
L = iso.load()
def lanes():
    return [l for l in log() if l[0] == "kernel"]
far = [(i + 1) << 44 for i in range(8)]
for dt, nq, nkv, d in (("bf16", 1, 1, 128), ("bf16", 8, 1, 128), ("bf16", 13, 13, 64), ("f32", 4, 4, 64), ("bf16", 1, 1, 64)):
    with iso.Context(iso.make_cfg(64, nq, nkv, d, 64, dt, 256)) as ctx:
        c = ctypes.byref(iso.IsoKv4(far[0], far[1], far[2], far[3], 4, 16))
        def calls(T):
            return [L.iso_rope_kv4_write(ctx._h, far[4], None, c, far[6], far[7], T, None), L.iso_rope_kv4_write(ctx._h, far[4], far[5], c, far[6], far[7], T, None),
                    L.iso_kv4_store(ctx._h, far[4], far[5], c, far[6], T, None), L.iso_kv4_load(ctx._h, c, far[6], far[4], far[5], T, None)]
        log()
        most = (2 ** 35 // d - 1) // (nq + 2 * nkv)
        assert calls(min(most, 2 ** 31 - 1)) == [0] * 4, iso.last_error()
        assert len(lanes()) == 4
        for lanes_each in (16, 8):
            assert most * (nq + 2 * nkv) * d // lanes_each <= 2 ** 32
        for T in (most + 1, 2 * most, 2 ** 31 - 1):
            if most < T < 2 ** 31:
                assert calls(T) == [-2] * 4 and "2^35" in iso.last_error(), T
        assert lanes() == []
        ctx.set_flags(iso.ISO_FLAG_SIMPLE_ATTN)
        n = ctypes.c_size_t()
        for rows, want in ((2 ** 26 - 4, 0), (2 ** 26 - 3, -2)):
            if rows * nq < 2 ** 31:
                assert L.iso_attn_kv4_workspace(ctx._h, 1, rows, ctypes.byref(n)) == 0
                assert L.iso_attn_kv4(ctx._h, far[4], nq * d, c, far[6], 4, far[6], far[6], 1, rows, rows, far[5], far[7], n, None) == want, iso.last_error()
        log()
""")


def test_what_is_written_lies_apart_from_everything_else(fake):            # noqa: F811
    """The cache, tables, positions and slots too, to the byte on both sides."""
    run(fake, """
L = iso.load()
NKV, D, T, PAGE, PAGES = 2, 64, 8, 16, 4
far = [(i + 1) << 40 for i in range(20)]
for dt, e in (("bf16", 2), ("f32", 4)):
    with iso.Context(iso.make_cfg(64, 4, NKV, D, 64, dt, 256)) as ctx:
        h = ctx._h
        codes, scales = PAGES * PAGE * NKV * D // 2, PAGES * PAGE * NKV * D // 32
        n = ctx.attn_kv4_workspace(3, T)
        size = dict(k=codes, v=codes, ks=scales, vs=scales, qkv=T * 8 * D * e, q=T * 4 * D * e, kr=T * NKV * D * e, vr=T * NKV * D * e, pos=4 * T, slots=4 * T,
                    out=T * 4 * D * e, ws=n, table=4, start=16, lens=12)
        at = dict(zip(size, far))
        def cache(a):
            return ctypes.byref(iso.IsoKv4(a["k"], a["v"], a["ks"], a["vs"], PAGES, PAGE))
        calls = {
            "write": lambda a: L.iso_rope_kv4_write(h, a["qkv"], a["q"], cache(a), a["pos"], a["slots"], T, None),
            "write in place": lambda a: L.iso_rope_kv4_write(h, a["qkv"], None, cache(a), a["pos"], a["slots"], T, None),
            "store": lambda a: L.iso_kv4_store(h, a["kr"], a["vr"], cache(a), a["slots"], T, None),
            "load": lambda a: L.iso_kv4_load(h, cache(a), a["slots"], a["kr"], a["vr"], T, None),
            "attn": lambda a: L.iso_attn_kv4(h, a["q"], 4 * D, cache(a), a["table"], 4, a["start"], a["lens"], 3, T, T, a["out"], a["ws"], n, None)}
        four = ("k", "v", "ks", "vs")
        outs = {"write": ("q", *four), "write in place": ("qkv", *four), "store": four, "load": ("kr", "vr"), "attn": ("out", "ws")}
        ins = {"write": ("qkv", "pos", "slots"), "write in place": ("pos", "slots"), "store": ("kr", "vr", "slots"), "load": (*four, "slots"),
               "attn": (*four, "q", "table", "start", "lens")}
        for name, call in calls.items():
            assert call(at) == 0, iso.last_error()
            log()
            for o in outs[name]:
                for x in outs[name] + ins[name]:
                    if x == o:
                        continue
                    align = 4 if x in ("pos", "slots", "table", "start", "lens") else 16
                    up = -(-size[o] // align) * align              # x behind o, and its last byte in front of it
                    for place, want in ((at[o], -2), (at[o] + up - align, -2), (at[o] + up, 0), (at[o] - (size[x] - align) // align * align, -2),
                                        (at[o] - -(-size[x] // align) * align, 0)):
                        if up - align >= size[o] and place == at[o] + up - align:
                            continue
                        assert call({**at, x: place}) == want, (name, o, x, place - at[o], iso.last_error())
                        assert want == 0 or "overlap" in iso.last_error()
            assert all(l[0] == "kernel" for l in log())
        same = dict(at, vr=at["kr"])                             # inputs may be one another
        assert calls["store"](same) == 0 and calls["load"](dict(at, v=at["k"], vs=at["ks"])) == 0 and calls["attn"](dict(at, v=at["k"], start=at["lens"])) == 0
""")


def test_index_buffers_of_another_type(fake):                  # noqa: F811
    """Every length, table, position and slot of every call; torch's tensors are known by the name of their type."""
    run(fake, """
class Type:
    def __init__(self, name):
        self.name = name
    def __repr__(self):
        return self.name
class Tensor:                                                    # what the binding asks a tensor for
    def __init__(self, dtype, ptr, contiguous=True):
        self.dtype, self.ptr, self.contiguous = dtype, ptr, contiguous
    def is_contiguous(self):
        return self.contiguous
    def data_ptr(self):
        return self.ptr
i32, i64 = Type("torch.int32"), Type("torch.int64")
with iso.Context(iso.make_cfg(64, 4, 2, 64, 64, "bf16", 256)) as ctx:
    cache = ctx.kv4_cache(4, 16)
    a, b = (iso.DeviceArray((8, 8, 64), "bf16") for _ in range(2))
    n = ctx.attn_kv4_workspace(2, 8)
    ws = iso.DeviceArray((n,), "u8")
    calls = {"block_tables": (dict(cached=1, fresh=1, n_seqs=2, page=16, free_pages=1, n_free=4, free_head=1, block_table=1, max_pages=4, row_start=1, kv_len=1,
                                   positions=1, slots=1, max_rows=8, free_next=1), "cached fresh free_pages free_head block_table row_start kv_len positions slots free_next"),
             "rope_kv4_write": (dict(qkv=a, q_out=b, cache=cache, positions=1, slots=1, T=8), "positions slots"),
             "kv4_store": (dict(k=a, v=b, cache=cache, slots=1, T=8), "slots"),
             "kv4_load": (dict(k=a, v=b, cache=cache, slots=1, T=8), "slots"),
             "attn_kv4": (dict(q=a, q_stride=256, cache=cache, block_table=1, max_pages=4, row_start=1, kv_len=1, n_seqs=2, total_rows=8, max_rows=8, out=b, ws=ws, ws_bytes=n),
                          "block_table row_start kv_len")}
    for name, (kw, ints) in calls.items():
        ints = ints.split()
        bufs = {x: iso.DeviceArray((64,), "i32") for x in ints}
        f = getattr(ctx, name)
        f(**{**kw, **bufs})
        f(**{**kw, **{x: y.ptr for x, y in bufs.items()}})       # addresses
        for _ in range(2):
            f(**{**kw, **{x: Tensor(i32, y.ptr) for x, y in bufs.items()}})
        log()
        for x in ints:
            for bad in (Tensor(i64, bufs[x].ptr), Tensor(Type("torch.float32"), bufs[x].ptr), Tensor(i32, bufs[x].ptr, False), iso.DeviceArray((64,), "f32"),
                        iso.DeviceArray((256,), "u8")):
                try:
                    f(**{**kw, **bufs, x: bad})
                    assert False, (name, x, bad.dtype)
                except ValueError as e:
                    assert ("32-bit integers" if bad.dtype is not i32 else "contiguous") in str(e)
        assert not [l for l in log() if l[0] == "kernel"]
    ctx.block_tables(bufs["kv_len"], bufs["row_start"], 1, 16, None, 0, None, *(x if isinstance(x, int) else iso.DeviceArray((64,), "i32") for x in ("t", 4, "s", "l", "p", "q", 8, "n")))
    try:
        iso.Kv4Cache(16, *(iso.DeviceArray((4, 2, 16, w), "bf16") for w in (32, 32, 2, 2)))
        assert False
    except ValueError as e:
        assert "bytes" in str(e)
""")


def test_torch_tensors_of_32_bits_only():
    import pytest
    torch = pytest.importorskip("torch")
    import paper_2409_11155_amd as iso
    t = torch.zeros(5, dtype=torch.int32)
    for _ in range(2):
        assert iso._ints(t) == t.data_ptr()
    for bad in (torch.zeros(5, dtype=torch.int64), torch.zeros(5), torch.zeros(5, dtype=torch.int16), t[::2]):
        with pytest.raises(ValueError):
            iso._ints(bad)
    assert iso._ints(None) is None and iso._ints(4096) == 4096


def test_no_launch_for_requests_that_there_cannot_be(fake):    # noqa: F811
    """Of several requests the tiles of 128 rows take those of more than 1023 (row, query head) pairs of a KEY head.  Where max_rows allows
    none, the launch beside the line is left out, and the line takes requests of any size (max_rows is a hint)."""
    run(fake, """
def kernels(nq, nkv, d, n_seqs, rows, most, keys=1 << 16):
    with iso.Context(iso.make_cfg(64, nq, nkv, d, 64, "bf16", 256)) as ctx:
        cache = ctx.kv4_cache(4, 16)
        i = iso.DeviceArray((n_seqs * keys // 16,), "i32")
        q, out = (iso.DeviceArray((rows, nq, d), "bf16") for _ in range(2))
        n = ctx.attn_kv4_workspace(n_seqs, rows)
        ws = iso.DeviceArray((n,), "u8")
        log()
        ctx.attn_kv4(q, nq * d, cache, i, keys // 16, i, i, n_seqs, rows, most, out, ws, n)
        return ["rows" if "rows" in l[2].split()[0] else "line" for l in log() if l[0] == "kernel"]
for nq, nkv, d in ((13, 13, 128), (64, 64, 64), (66, 22, 128), (16, 2, 128), (8, 1, 128), (32, 8, 64)):
    G = nq // nkv
    first = 1023 // G + 1                                        # rows of the first request that is long enough
    assert kernels(nq, nkv, d, 2, 2 * first - 2, first - 1) == ["line"], (nq, nkv)
    assert kernels(nq, nkv, d, 2, 2 * first, first) == (["line", "rows"] if first * nq >= 4096 else ["line"]), (nq, nkv)
    assert kernels(nq, nkv, d, 2, first, 2 ** 31 - 1) == (["line", "rows"] if first * nq >= 4096 else ["line"]), (nq, nkv)
    one = 4096 // nq + 1                                         # a single request has one launch, whatever its pairs of a key head
    assert kernels(nq, nkv, d, 1, one, one) == ["rows"] and kernels(nq, nkv, d, 1, one - 2, one) == ["line"], (nq, nkv)
""")


def test_how_far_an_element_is_off_over_the_whole_range():
    """2^e between the ends of the scale; beyond them 2^126 above (what is larger than 6 * 2^125 becomes that) and 2^-126 below."""
    import numpy as np
    from oracle import kv4_oracle as ko
    rng = np.random.default_rng(0)
    top = np.exp2(rng.integers(-150, 128, 20000).astype(float)) * (1 + rng.random(20000) * (1 - 2.0 ** -24))
    top[:8] = [7 * 2.0 ** -126, np.nextafter(7 * 2.0 ** -126, 1), 7 * 2.0 ** 125, np.nextafter(7 * 2.0 ** 125, np.inf), 2.0 ** 128 * (1 - 2.0 ** -24), 2.0 ** -127, 2.0 ** -149, 3.4e38]
    x = rng.uniform(-1, 1, (20000, 32)) * top[:, None]
    x[:, 5] = top
    codes, scales = ko.encode(x)
    off = np.abs(x - ko.decode(codes, scales)).max(1)
    small, large = top <= 7 * 2.0 ** -126, top > 7 * 2.0 ** 125
    inside = ~small & ~large
    assert small.sum() > 1000 and large.sum() > 10 and inside.sum() > 10000
    assert (off[inside] <= np.exp2(scales[inside, 0] - 127.0)).all() and (off[inside] < 2 / 7 * top[inside]).all()
    assert (scales[large] == 252).all() and (off[large] <= 2.0 ** 126).all() and off[large].max() > 1.9 * 2.0 ** 125
    assert (ko.decode(codes, scales)[large, 5] == 6 * 2.0 ** 125).all()
    assert (scales[small] == 2).all() and (off[small] <= 2.0 ** -126).all()
    gone = top <= 2.0 ** -127
    assert (ko.decode(codes, scales)[gone] == 0).all() and gone.sum() > 1000
