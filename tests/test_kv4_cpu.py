"""The 4-bit cache without a GPU: the oracle against hand values and slow definitions, and what the entry points refuse (the
library's HIP calls go to tests/fake_hip.cpp)."""
import numpy as np
import pytest

from oracle import kv4_oracle as ko
from test_host_side_cpu import fake, run                       # noqa: F401  (fixture)


def test_levels_ties_and_saturation():
    x = np.zeros(32)
    x[:16] = [0.25, 0.26, 0.74, 0.75, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 6.9, -0.75, -5.0, 7.0]   # 7: the scale stays 1
    codes, scales = ko.encode(x)
    assert scales.tolist() == [127]
    assert ko.decode(codes, scales)[:16].tolist() == [0, .5, .5, 1, 1, 1.5, 2, 2, 3, 4, 4, 6, 6, -1, -4, 6]
    x[15] = np.nextafter(7.0, 8.0)                             # just above: the next power of two
    assert ko.encode(x)[1].tolist() == [128]


def test_order_of_bytes_and_elements():
    x = np.zeros(64)
    x[0], x[1], x[33] = 1.0, -6.0, 0.5
    codes, scales = ko.encode(x)
    assert codes[0] == 2 | 15 << 4 and codes[16] == 6 << 4 and not codes[1:16].any() and scales.tolist() == [127, 124]    # 0.5 = 4 / 8


def test_scale_ends_and_values_that_are_not_finite():
    for top, byte in ((0.0, 2), (1e-45, 2), (2.0 ** -126, 2), (7 * 2.0 ** -125, 2), (7.1 * 2.0 ** -125, 3), (3.4e38, 252), (2.0 ** 120, 127 + 118)):
        assert ko.encode(np.full(32, top))[1].tolist() == [byte], top
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(64)
        x[40] = bad
        codes, scales = ko.encode(x)
        assert scales[0] == 125 and scales[1] == 255 and (codes[16:] == 0).all()
        assert np.isnan(ko.decode(codes, scales)[32:]).all() and np.isfinite(ko.decode(codes, scales)[:32]).all()


def test_every_element_is_within_two_sevenths_of_the_largest():
    x = np.random.default_rng(0).standard_normal((2000, 32)) * np.exp2(np.random.default_rng(1).integers(-30, 30, (2000, 1)))
    y = ko.decode(*ko.encode(x))
    assert (np.abs(x - y) <= 2 / 7 * np.abs(x).max(-1, keepdims=True)).all()
    codes, scales = ko.encode(y)                               # a value of the format is itself again
    np.testing.assert_array_equal(ko.decode(codes, scales), y)


def test_attention_of_one_request_is_the_layers_definition():
    from oracle import iso_oracle as orc
    rng = np.random.default_rng(3)
    nq, nkv, d, kv, n, page = 4, 2, 64, 37, 5, 16
    q = rng.standard_normal((n, nq, d))
    k, v = rng.standard_normal((2, 5, nkv, page, d))
    table = np.array([[3, 0, 4]])
    rows = lambda a: a[table[0]].transpose(0, 2, 1, 3).reshape(-1, nkv, d)[:kv]  # noqa: E731
    ref = orc.attention_chunk(q, rows(k), rows(v), kv - n, kv).reshape(n, nq, d)
    out, _, _ = ko.attention(q, k, v, table, page, [0, n], [kv], nq // nkv)
    np.testing.assert_allclose(out, ref, rtol=0, atol=1e-13)


def test_block_tables_by_hand():
    table, start, kv, pos, slots, nxt = ko.block_tables([5, 0, 16], [12, 0, 1], 16, [7, 9], 0, [[3, -1], [-1, -1], [2, -1]], 15)
    assert table.tolist() == [[3, 7], [-1, -1], [2, 9]] and start.tolist() == [0, 12, 12, 13] and kv.tolist() == [17, 0, 17] and nxt == 2
    assert pos.tolist() == list(range(5, 17)) + [16, -1, -1]
    assert slots.tolist() == [48 + p for p in range(5, 16)] + [7 * 16, 9 * 16, -1, -1]


REFUSALS = """
vp = ctypes.c_void_p
L = iso.load()
def launches():
    return [l[0] for l in log() if l[0] == "kernel"]
def code(f, *a):
    return getattr(L, "iso_" + f)(*a)
with iso.Context(iso.make_cfg(64, 4, 2, 64, 64, DT, 256)) as ctx:
    h, ok = ctx._h, 4096
    i = lambda n=64: iso.DeviceArray((n,), "i32")
    cache = ctx.kv4_cache(4, 16)
    ck = ctypes.byref(cache.handle)
    def cache_with(**kw):
        c = iso.IsoKv4(cache.handle.k, cache.handle.v, cache.handle.k_scale, cache.handle.v_scale, 4, 16)
        for n, x in kw.items():
            setattr(c, n, x)
        return ctypes.byref(c)
    bad_caches = [(None, -1), (cache_with(k=None), -1), (cache_with(v_scale=None), -1), (cache_with(page=15), -2), (cache_with(page=48), -2),
                  (cache_with(page=512), -2), (cache_with(page=0), -2), (cache_with(n_pages=0), -2), (cache_with(n_pages=1 << 27), -2),
                  (cache_with(v=cache.handle.v + 8), -2)]
    log()
    # block tables
    bufs = [i() for _ in range(10)]
    p = [b.ptr for b in bufs]
    good = [h, p[0], p[1], 2, 16, p[2], 8, p[3], p[4], 4, p[5], p[6], p[7], p[8], 8, p[9], None]
    def tables(**kw):
        a = list(good)
        for n, x in kw.items():
            a[int(n[1:])] = x
        return code("block_tables", *a)
    assert tables() == 0, iso.last_error()
    assert launches() == ["kernel"]
    assert tables(_5=None, _6=0) == 0 and tables(_7=None) == 0
    log()
    for n in (0, 1, 2, 5, 8, 10, 11, 12, 13, 15):
        assert tables(**{f"_{n}": None}) == -1, n
    for kw in (dict(_3=0), dict(_3=4097), dict(_4=24), dict(_4=8), dict(_4=-16), dict(_6=-1), dict(_9=0), dict(_14=0), dict(_11=p[0]), dict(_11=p[1]),
               dict(_15=p[3]), dict(_12=p[7] + 2)):
        assert tables(**kw) == -2, kw
    # writes and reads
    rows = [iso.DeviceArray((8, 8, 64), DT) for _ in range(3)]
    r = [b.ptr for b in rows]
    assert code("rope_kv4_write", h, r[0], r[1], ck, p[0], p[1], 8, None) == 0
    assert code("rope_kv4_write", h, r[0], None, ck, p[0], p[1], 8, None) == 0
    assert code("kv4_store", h, r[0], r[1], ck, p[1], 8, None) == 0 and code("kv4_load", h, ck, p[1], r[0], r[1], 8, None) == 0
    assert launches() == ["kernel"] * 4
    for a in ((None, r[0], r[1], ck, p[0], p[1], 8), (h, None, r[1], ck, p[0], p[1], 8), (h, r[0], r[1], ck, None, p[1], 8), (h, r[0], r[1], ck, p[0], None, 8)):
        assert code("rope_kv4_write", *a, None) == -1
    for a in ((None, r[0], r[1], ck, p[1], 8), (h, None, r[1], ck, p[1], 8), (h, r[0], None, ck, p[1], 8), (h, r[0], r[1], ck, None, 8)):
        assert code("kv4_store", *a, None) == -1
    for a in ((None, ck, p[1], r[0], r[1], 8), (h, ck, None, r[0], r[1], 8), (h, ck, p[1], None, r[1], 8), (h, ck, p[1], r[0], None, 8)):
        assert code("kv4_load", *a, None) == -1
    for T in (0, -3):
        assert code("rope_kv4_write", h, r[0], r[1], ck, p[0], p[1], T, None) == -2
        assert code("kv4_store", h, r[0], r[1], ck, p[1], T, None) == -2 and code("kv4_load", h, ck, p[1], r[0], r[1], T, None) == -2
    assert code("rope_kv4_write", h, r[0] + 8, r[1], ck, p[0], p[1], 8, None) == -2 and code("rope_kv4_write", h, r[0], r[1] + 2, ck, p[0], p[1], 8, None) == -2
    assert code("kv4_store", h, r[0] + 8, r[1], ck, p[1], 8, None) == -2 and code("kv4_load", h, ck, p[1] + 1, r[0], r[1], 8, None) == -2
    for c, want in bad_caches:
        assert code("rope_kv4_write", h, r[0], r[1], c, p[0], p[1], 8, None) == want
        assert code("kv4_store", h, r[0], r[1], c, p[1], 8, None) == want and code("kv4_load", h, c, p[1], r[0], r[1], 8, None) == want
    # attention
    n = ctypes.c_size_t()
    assert code("attn_kv4_workspace", h, 3, 8, ctypes.byref(n)) == 0 and n.value >= 256
    assert code("attn_kv4_workspace", None, 3, 8, ctypes.byref(n)) == -1 and code("attn_kv4_workspace", h, 3, 8, None) == -1
    for s, t in ((0, 8), (4097, 8), (3, 0), (3, -1)):
        assert code("attn_kv4_workspace", h, s, t, ctypes.byref(n)) == -2
    code("attn_kv4_workspace", h, 3, 8, ctypes.byref(n))
    ws = iso.DeviceArray((n.value,), "u8", fill_byte=0)
    log()
    good = [h, r[0], 256, ck, p[0], 4, p[1], p[2], 3, 8, 4, r[1], ws.ptr, n.value, None]
    def attn(**kw):
        a = list(good)
        for k, x in kw.items():
            a[int(k[1:])] = x
        return code("attn_kv4", *a)
    assert attn() == 0 and attn(_2=264) == 0 and attn(_10=1) == 0 and attn(_10=1000) == 0
    assert len(launches()) >= 4
    for k in (0, 1, 3, 4, 6, 7, 11, 12):
        assert attn(**{f"_{k}": None}) == -1, k
    for kw in (dict(_2=248), dict(_2=257), dict(_5=0), dict(_8=0), dict(_8=4097), dict(_9=0), dict(_10=0), dict(_1=r[0] + 8), dict(_11=r[1] + 4),
               dict(_12=ws.ptr + 8), dict(_4=p[0] + 1)):
        assert attn(**kw) == -2, kw
    assert attn(_13=n.value - 1) == -5
    for c, want in bad_caches:
        assert attn(_3=c) == want
    assert launches() == []                                      # nothing that was refused launched anything
    try:
        ctx.kv4_store(rows[0], rows[1], iso.Kv4Cache(16, *(iso.DeviceArray((4, 1, 16, 2 * w), "u8") for w in (16, 16, 1, 1))), bufs[0], 8)
        assert False
    except ValueError as e:
        assert "heads" in str(e)
try:
    iso.Kv4Cache(16, *(iso.DeviceArray((4, 2, 16, w), "u8") for w in (32, 32, 2, 4)))
    assert False
except ValueError:
    pass
"""


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_refusals(fake, dt):                                    # noqa: F811
    run(fake, f"DT = {dt!r}\n" + REFUSALS)


def test_which_kernels_a_batch_gets(fake):                     # noqa: F811
    """One launch for single tokens and short chunks, with 16 rows a tile where no request has more pairs or there is little to do for
    heads of 128; long chunks go to the tiles of 128 rows where the table has room for many keys, beside a launch for the short requests of
    the batch if there can be any; fp32 stays on the line."""
    run(fake, """
def kernels(dt, nq, nkv, d, n_seqs, rows, most, keys):
    with iso.Context(iso.make_cfg(64, nq, nkv, d, 64, dt, 256)) as ctx:
        cache = ctx.kv4_cache(4, 16)
        i = iso.DeviceArray((64,), "i32")
        q, out = (iso.DeviceArray((rows, nq, d), dt) for _ in range(2))
        n = ctx.attn_kv4_workspace(n_seqs, rows)
        ws = iso.DeviceArray((n,), "u8")
        log()
        ctx.attn_kv4(q, nq * d, cache, i, keys // 16, i, i, n_seqs, rows, most, out, ws, n)
        return [l[2].split()[0] for l in log() if l[0] == "kernel"]
def line(name, rt):
    return "attn_kv4_kernel" in name and name.split("Li")[-1].startswith(str(rt))
k = kernels("bf16", 8, 1, 128, 5, 5, 1, 8192);       assert len(k) == 1 and line(k[0], 1), k
k = kernels("bf16", 8, 1, 128, 5, 5, 2, 8192);       assert len(k) == 1 and line(k[0], 1), k
k = kernels("bf16", 8, 1, 128, 5, 50, 3, 8192);      assert len(k) == 1 and line(k[0], 1), k
k = kernels("bf16", 8, 1, 128, 5, 2000, 3, 8192);    assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 8, 4, 64, 5, 9, 9, 64);          assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 8, 1, 128, 1, 511, 511, 16384);  assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 8, 1, 128, 1, 512, 512, 8192);   assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 8, 1, 128, 1, 512, 1, 16384);    assert len(k) == 1 and "rows" in k[0], k
k = kernels("bf16", 8, 1, 128, 1, 512, 1, 1 << 30);  assert len(k) == 1 and "rows" in k[0], k
k = kernels("bf16", 8, 1, 128, 2, 4096, 512, 8192);  assert len(k) == 2 and line(k[0], 2) and "rows" in k[1], k
k = kernels("bf16", 8, 1, 128, 2, 4096, 511, 8192);  assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 8, 1, 128, 2, 4096, 512, 4096);  assert len(k) == 1 and line(k[0], 2), k
k = kernels("bf16", 130, 1, 64, 1, 200, 200, 8192);  assert len(k) == 1 and line(k[0], 2), k
k = kernels("f32", 8, 1, 128, 1, 4096, 4096, 8192);  assert len(k) == 1 and line(k[0], 1), k
""")


OVERLAPS = """
L = iso.load()
with iso.Context(iso.make_cfg(64, 4, 2, 64, 64, "bf16", 256)) as ctx:
    h = ctx._h
    cache = ctx.kv4_cache(4, 16)
    def refuses(f, *a):
        assert getattr(L, "iso_" + f)(h, *a, None) == -2, (f, a)
        assert "overlap" in iso.last_error()
    mem = iso.DeviceArray((1 << 16,), "u8").ptr                # places in one buffer; 8 rows of 8 heads are 8192 bytes
    # lengths, free pages, table of 2 x 4, starts, lengths, positions, slots of 8 rows, next
    at = {n: mem + 64 * i for i, n in enumerate("cached fresh free_pages head table start kv_len positions slots next".split())}
    def tables(**kw):
        p = {**at, **kw}
        return (p["cached"], p["fresh"], 2, 16, p["free_pages"], 8, p["head"], p["table"], 4, p["start"], p["kv_len"], p["positions"], p["slots"], 8, p["next"])
    assert L.iso_block_tables(h, *tables(), None) == 0, iso.last_error()
    assert L.iso_block_tables(h, *tables(fresh=at["cached"], next=at["head"] + 4), None) == 0      # inputs may be one another
    for kw in (dict(kv_len=at["cached"]), dict(kv_len=at["fresh"] + 4), dict(next=at["head"]), dict(table=at["free_pages"] + 28), dict(slots=at["positions"] + 28),
               dict(start=at["kv_len"] - 8), dict(positions=at["cached"] - 28), dict(next=at["table"] + 28)):
        refuses("block_tables", *tables(**kw))
    ck = cache.ref
    i = mem + 60000
    assert L.iso_rope_kv4_write(h, mem, mem + 8192, ck, i, i, 8, None) == 0
    for q in (mem, mem + 8192 - 16, mem + 4096):
        refuses("rope_kv4_write", mem, q, ck, i, i, 8)
    refuses("rope_kv4_write", mem + 4096, mem + 16, ck, i, i, 8)
    assert L.iso_kv4_load(h, ck, i, mem, mem + 2048, 8, None) == 0
    refuses("kv4_load", ck, i, mem, mem + 2032, 8)
    assert L.iso_kv4_store(h, mem, mem, ck, i, 8, None) == 0    # inputs may be
    n = ctx.attn_kv4_workspace(1, 8)
    ws = iso.DeviceArray((n + 4096,), "u8").ptr
    def attn(q, out, w):
        return (q, 512, ck, i, 4, i, i, 1, 8, 8, out, w, n)
    end = 7 * 1024 + 512                                       # of q: rows 512 elements apart, 256 of them read
    assert L.iso_attn_kv4(h, *attn(mem, mem + end, ws), None) == 0, iso.last_error()
    refuses("attn_kv4", *attn(mem, mem, ws))
    refuses("attn_kv4", *attn(mem, mem + end - 16, ws))
    refuses("attn_kv4", *attn(ws + n - 16, mem, ws))
    refuses("attn_kv4", *attn(mem, ws, ws))
"""


def test_overlapping_buffers_are_refused(fake):                # noqa: F811
    run(fake, OVERLAPS)
