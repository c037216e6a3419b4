"""The 4-bit cache at the ends of what its calls take, on the GPU (bounds: see test_gpu_kv4.py)."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_kv4 import attend, check, device_cache, f64, make_ctx

pytestmark = pytest.mark.gpu
MOST_KEYS = 2 ** 31 - 1024


@pytest.mark.parametrize("dt,nq,d,fresh", [("bf16", 1, 64, 1), ("bf16", 4, 128, 5), ("f32", 1, 64, 1), ("bf16", 64, 64, 64)])
@pytest.mark.parametrize("kv", [MOST_KEYS, 2 ** 31 - 1])
def test_as_many_keys_as_a_table_may_have(dt, nq, d, fresh, kv):
    """Pages of the first and the last keys only, all others are missing: what is seen is known.  Of 2^31 - 1 keys the last 1023 have no
    place in the table."""
    page = 256
    width, n_pages = MOST_KEYS // page, 4
    cols = np.array([0, 1, width - 2, width - 1])
    table = np.full((1, width), -1, np.int32)
    table[0, cols] = [2, 0, 3, 1]
    rng = np.random.default_rng(3)
    codes, scales = zip(*(ko.encode(rng.standard_normal((n_pages, 1, page, d))) for _ in range(2)))
    q = iso_inputs.randn((fresh, nq, d), seed=5, dtype=dt)
    with make_ctx(nq, 1, d, dt) as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, np.array([0, fresh]), [kv], dt, nq, d), dt)
    # the same keys, close together: a row sees as many fewer than the last as before
    gone = (width - 4) * page
    check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table[:, cols], page, [0, fresh], [kv - gone], nq, dt, n_pages)


def whole_range(T, heads, d, dt, seed):
    """Blocks of every magnitude of the type, denormal numbers and the largest ones among them, and the borders of two codes at both
    ends of the scale."""
    rng = np.random.default_rng(seed)
    x = rng.uniform(-1, 1, (T, heads, d)) * np.exp2(rng.integers(-149, 128, (T, heads, d // 32)).repeat(32, -1))
    at_end = rng.random((T, heads, d // 32)).repeat(32, -1)
    edges = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -5.0, 6.0, 0.125, 0.3125], x.shape)
    x = np.where(at_end < 0.1, edges * 2.0 ** -125, np.where(at_end > 0.9, edges * 2.0 ** 125, x))
    x[rng.random(x.shape) < 0.02] = 3.3895e38
    return iso_inputs.store(x.astype(np.float32), dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_over_the_whole_range_of_the_type(dt, d):
    """Codes, scales and loaded values, stored and rotated, equal the definition from the least denormal number to the largest."""
    T, nkv, page, nq = 300, 2, 32, 4
    n_pages = -(-T // page)
    slots = np.random.default_rng(1).permutation(n_pages * page)[:T].astype(np.int32)
    k, v = (whole_range(T, nkv, d, dt, s) for s in (1, 2))
    with make_ctx(nq, nkv, d, dt, 4000) as ctx:
        up = lambda a: iso.DeviceArray.from_numpy(a, dt)  # noqa: E731
        cache = ctx.kv4_cache(n_pages, page, fill_byte=0)
        sd, back = iso.DeviceArray.from_numpy(slots, "i32"), [iso.DeviceArray((T, nkv, d), dt) for _ in range(2)]
        ctx.kv4_store(up(k), up(v), cache, sd, T, ctx.stream0)
        ctx.kv4_load(cache, sd, back[0], back[1], T, ctx.stream0)
        ctx.sync()
        for x, codes, scales, b in ((k, cache.k, cache.k_scale, back[0]), (v, cache.v, cache.v_scale, back[1])):
            rc, rs = ko.encode(f64(x, dt))
            np.testing.assert_array_equal(scales.numpy()[slots // page, :, slots % page], rs)
            np.testing.assert_array_equal(codes.numpy()[slots // page, :, slots % page], rc)
            np.testing.assert_array_equal(f64(b, dt), ko.decode(rc, rs))
        qkv = whole_range(T, nq + 2 * nkv, d, dt, 3)
        pos = np.random.default_rng(4).integers(0, 4000, T).astype(np.int32)
        ctx.rope_kv4_write(up(qkv), iso.DeviceArray((T, nq, d), dt), cache, iso.DeviceArray.from_numpy(pos, "i32"), sd, T, ctx.stream0)
        ctx.sync()
        x = f64(qkv, dt)
        for val, codes, scales in ((ko.rotate(x[:, nq:nq + nkv], pos), cache.k, cache.k_scale), (x[:, nq + nkv:], cache.v, cache.v_scale)):
            rc, rs = ko.encode(val)
            np.testing.assert_array_equal(scales.numpy()[slots // page, :, slots % page], rs)
            one = np.full_like(rs, 127)                          # (a zero of either sign is a zero)
            np.testing.assert_array_equal(ko.decode(codes.numpy()[slots // page, :, slots % page], one), ko.decode(rc, one))
