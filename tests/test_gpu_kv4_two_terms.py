"""Attention over the 4-bit cache in bf16 where a probability is two bf16 terms: heads of 64, as exact as the framework's attention over
rows, which has two there as well, and tiles of 16 (row, head) pairs.

Bound per element, with A the probability-weighted mean of |v| and N the number of keys:
  2^-8 |out|                   the result is rounded once
  2^-16 A                      the probabilities: the nearest bf16 number is off by 2^-8 at most, the second term by 2^-8 of that
  2 E A + (2 N + 16) 2^-24 A   scores and fp32 accumulation, see test_gpu_kv4.py
With one term the second line would be 2^-8 A; elements far below A then leave the bound."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_kv4 import attend, batch, device_cache, f64, fill, ints, make_ctx, wide

pytestmark = pytest.mark.gpu


def check_two_terms(got, q, k, v, table, page, row_start, kv, group, n_pages):
    d = q.shape[-1]
    ref, A, reach = ko.attention(q, k, v, table, page, row_start, kv, group, n_pages)
    E = (d + 8) * 2.0 ** -24 * np.nan_to_num(reach)[..., None] * 1.4427 + 2.0 ** -22
    tol = 2.0 ** -8 * np.abs(ref) + A * (2.0 ** -16 + 2 * E + (2 * max(1, max(kv)) + 16) * 2.0 ** -24)
    err = np.abs(got - ref)
    assert (err <= tol)[~np.isnan(A)].all(), float(np.nanmax(err / np.maximum(tol, 1e-30)))


@pytest.mark.parametrize("room", [0, 1 << 20])                  # 16 or 32 rows a tile; 32 or 128
@pytest.mark.parametrize("heads", [(32, 8), (4, 4), (20, 1), (64, 1), (64, 64)])
@pytest.mark.parametrize("kv,fresh,page", [([1], [1], 16), ([700, 41, 1300], [2, 3, 5], 128), ([7, 130, 33], [7, 130, 33], 16), ([1100], [257], 256),
                                           ([900] * 12, [1] * 12, 64)])
def test_probabilities_keep_sixteen_bits(heads, kv, fresh, page, room):
    nq, nkv = heads
    table, row_start, n_pages = batch(kv, fresh, page, seed=2)
    table = wide(table, page, room)
    codes, scales = fill(n_pages, nkv, page, 64, 3, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, 64), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, 64, "bf16") as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, "bf16", nq, 64), "bf16")
    check_two_terms(got, f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, n_pages)


@pytest.mark.parametrize("kv,fresh", [(777, 777), (2500, 500), (3000, 1)])
def test_pages_are_attended_to_as_exactly_as_rows(kv, fresh):
    """The same values in pages and in rows: the distance to 64 bits is that of the framework's attention over rows (the same number of
    roundings in another order: within 2 % of it over 500 000 elements, 20 % over 2048)."""
    nq, nkv, d, page = 32, 8, 64, 32
    table, row_start, n_pages = batch([kv], [fresh], page, seed=2)
    codes, scales = fill(n_pages, nkv, page, d, 3, table, [kv])
    q = iso_inputs.randn((fresh, nq, d), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, d, "bf16", max_seq=4096) as ctx:
        cache = device_cache(codes, scales, page)
        out = attend(ctx, q, cache, table, row_start, [kv], "bf16", nq, d)
        rows = [iso.DeviceArray((kv, nkv, d), "bf16") for _ in range(2)]
        j = np.arange(kv)
        ctx.kv4_load(cache, ints(table[0, j // page] * page + j % page), rows[0], rows[1], kv, ctx.stream0)
        other = iso.DeviceArray((fresh, nq, d), "bf16", fill_byte=0xFF)
        ctx.attn_chunk(iso.DeviceArray.from_numpy(q, "bf16"), rows[0], rows[1], other, fresh, kv - fresh, kv, ctx.stream0)
        ctx.sync()
        got, base = f64(out, "bf16"), f64(other, "bf16").reshape(fresh, nq, d)
    ref = ko.attention(f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, [kv], nq // nkv, n_pages)[0]
    mine, theirs = (float(np.sqrt(((x - ref) ** 2).mean() / (ref ** 2).mean())) for x in (got, base))
    print(f"{kv} {fresh}: {mine:.4e} {theirs:.4e}")
    assert mine <= theirs * (1.02 if fresh > 400 else 1.2)


@pytest.mark.parametrize("heads", [(8, 1), (13, 13), (16, 2), (3, 1)])
@pytest.mark.parametrize("kv,fresh,page", [([1], [1], 16), ([5, 900, 1, 2049, 333, 64], [1] * 6, 64), ([20000], [1], 64), ([700, 41, 1300], [2, 3, 5], 128),
                                           ([2000] * 40, [1] * 40, 64)])
def test_tiles_of_sixteen_keep_sixteen_bits_for_heads_of_128_too(heads, kv, fresh, page):
    nq, nkv = heads
    table, row_start, n_pages = batch(kv, fresh, page, seed=2)
    codes, scales = fill(n_pages, nkv, page, 128, 3, table, kv)
    q = iso_inputs.randn((int(row_start[-1]), nq, 128), seed=9, dtype="bf16")
    with make_ctx(nq, nkv, 128, "bf16") as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, row_start, kv, "bf16", nq, 128), "bf16")
    check_two_terms(got, f64(q, "bf16"), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table, page, row_start, kv, nq // nkv, n_pages)
