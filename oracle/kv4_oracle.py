"""Definition, in plain numpy and 64 bits, of the paged 4-bit key/value cache: the format, the block tables, the writes and the
attention that reads it.  Test infrastructure only; nothing under the product package imports it."""
from __future__ import annotations

import numpy as np

BLOCK = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x):
    """x [..., d] -> (codes [..., d / 2] uint8, scales [..., d / 32] uint8).  Per block: e = least integer with max|x| <= 7 * 2^e,
    kept in [-125, 125]; each element the nearest level times 2^e, ties to the even code; NaN or infinity anywhere: byte 255."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (-1, BLOCK))
    fine = np.isfinite(b).all(-1)
    b = np.where(fine[..., None], b, 0.0)
    top = np.abs(b).max(-1)
    m, e = np.frexp(np.where(top > 0, top, 1.0))               # top = m * 2^e, m in [0.5, 1); 7 * 2^k = 0.875 * 2^(k + 3)
    e = np.where(top > 0, np.where(m <= 0.875, e - 3, e - 2), -125).clip(-125, 125)
    u = np.abs(b) / np.exp2(e.astype(np.float64))[..., None]
    dist = np.abs(u[..., None] - LEVELS)                        # first of the nearest two, then the even one of a tie
    code = dist.argmin(-1)
    nxt = np.minimum(code + 1, 7)
    tie = (np.take_along_axis(dist, nxt[..., None], -1)[..., 0] == dist.min(-1)) & (nxt != code) & (nxt % 2 == 0)
    code = np.where(tie, nxt, code) + 8 * np.signbit(b)
    code = np.where(fine[..., None], code, 0).reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(fine, e + 127, 255).astype(np.uint8)


def decode(codes, scales):
    """Values [..., d] of codes [..., d / 2] and scales [..., d / 32]."""
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (-1,)).astype(np.int64)
    v = np.where(nib < 8, 1.0, -1.0) * LEVELS[nib & 7]
    f = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return v * np.repeat(f, BLOCK, -1)


def rotate(x, positions, base=10000.0):
    """x [T, heads, d] rotated in pairs (i, i + d/2) with the framework's table (angles in 64 bits, cosine and sine kept in 32)."""
    d = x.shape[-1]
    inv = np.power(float(base), -2.0 * np.arange(d // 2) / d)
    ang = np.asarray(positions, dtype=np.float64)[:, None] * inv
    c, s = (f.astype(np.float32).astype(np.float64)[:, None, :] for f in (np.cos(ang), np.sin(ang)))
    lo, hi = x[..., : d // 2], x[..., d // 2:]
    return np.concatenate((lo * c - hi * s, hi * c + lo * s), -1)


def block_tables(cached, fresh, page, free_pages, head, table, max_rows):
    """(table, row_start, kv_len, positions, slots, free_next) of one step, request by request and token by token."""
    table = np.array(table)
    width = table.shape[1]
    start, kv, pos, slots = [0], [], [-1] * max_rows, [-1] * max_rows
    for i, (c, f) in enumerate(zip(cached, fresh)):
        c, f = max(0, int(c)), max(0, int(f))
        for col in range(min(width, -(-c // page)), min(width, -(-(c + f) // page))):
            table[i, col] = free_pages[head] if 0 <= head < len(free_pages) else -1
            head += 1
        for t in range(f):
            r, p = start[-1] + t, c + t
            if r < max_rows:
                pos[r] = p
                if p // page < width and table[i, p // page] >= 0:
                    slots[r] = table[i, p // page] * page + p % page
        start.append(start[-1] + f)
        kv.append(c + f)
    return table, np.array(start), np.array(kv), np.array(pos), np.array(slots), head


def attention(q, k, v, table, page, row_start, kv_len, group, n_pages=None):
    """q [rows, nq, d]; k, v [n_pages, nkv, page, d] values.  Returns (out, spread, reach), zero / untouched (NaN) where a row sees
    nothing / belongs to no request: out [rows, nq, d]; spread = the same average of |v|; reach [rows, nq] = the largest sum of
    |q_e k_e| / sqrt(d) over the keys a row sees (what the rounding of a score is relative to)."""
    rows, nq, d = q.shape
    out, spread, reach = (np.full(s, np.nan) for s in (q.shape, q.shape, (rows, nq)))
    n_pages = len(k) if n_pages is None else n_pages
    for i, n_keys in enumerate(kv_len):
        lo, hi = int(row_start[i]), int(row_start[i + 1])
        r = np.arange(max(lo, 0), min(hi, rows))
        if not r.size:
            continue
        keys = np.arange(min(max(int(n_keys), 0), table.shape[1] * page))
        pg = table[i, keys // page]
        there = (pg >= 0) & (pg < n_pages)
        keys, pg = keys[there], pg[there]
        seen = keys[None] <= int(n_keys) - (hi - lo) + (r - lo)[:, None]           # [rows, keys]
        some = seen.any(1)
        out[r], spread[r], reach[r] = 0.0, 0.0, 0.0
        if not some.any():
            continue
        r, seen = r[some], seen[some]
        for h in range(nq):
            kk, vv = k[pg, h // group, keys % page], v[pg, h // group, keys % page]
            s = np.where(seen, q[r, h] @ kk.T / np.sqrt(d), -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            out[r, h], spread[r, h] = p @ vv, p @ np.abs(vv)
            reach[r, h] = np.where(seen, np.abs(q[r, h]) @ np.abs(kk).T, 0.0).max(1) / np.sqrt(d)
    return out, spread, reach
