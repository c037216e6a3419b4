// Attention over the paged 4-bit cache for many rows (bf16): chunks of prompts.  Bound by the instructions of the softmax and of unpacking
// beside the matrix cores: both pipes are busy half of the time, one after the other more than at once.
//
// A row tile is up to 128 (token, query head) pairs of one key head, whole tokens, 32 rows a wave.  All of a key head's queries share a
// tile, so the cache is unpacked once for them: tiles of 64 keys go from the pages to registers (requested one tile ahead), are unpacked
// there (exact, see attn_kv4.hip) and written to LDS as bf16 rows, two stages, one barrier a tile.  The conversions ride behind the
// first product's matrix instructions.  From LDS on it is the bf16 kernel's layout (attn_bf16_dtl.hip): S^T = K Q^T with
// v_mfma_f32_32x32x16_bf16, statistics per lane, V read transposed (ds_read_b64_tr_b16), O^T = V^T P^T.
// 16-byte chunks are XOR-swizzled by the row: any 16 neighbouring lanes of a read or a write touch different banks (the LDS works in 48 %
// of the cycles, a quarter of that counted as conflicts).
//
// Work: as in attn_kv4.hip one line cut into equal shares, here in keys per key head: the k-th row tile of a request has
// max(0, kv_len - rows) + (k + 1) * tokens places (a row tile further down sees more keys) behind SETUP places for its start and end, so a
// request's length on the line is a closed form and a place's tile the root of a quadratic.  Shares begin at multiples of 64 keys of a tile.
// Pieces of a tile are parked and folded in order by the last to arrive.
//
// Measured: 8 heads over 1, 2048 rows over 32768 keys 266 to 321 us (1000 to 830 TFLOP/s, the first after a pause of the card), over 131072 keys 1065
// (990); 16 heads over 2, 8192 of 8192 301 to 350 (910 to 790).  Heads of 64 (two terms a probability), 32 over 8: 2048 rows of 2048 47 (370), over
// 32768 keys 905 (590).  In the first vector instructions take 52 %, matrix instructions 48 % of the cycles; products
// of 8192^3 reach 1500 TFLOP/s here, the framework's bf16 attention 960 on the same rows and keys.
#include "kv4.h"
#include <type_traits>

namespace {

constexpr int BM = 128, BN = 64, THREADS = 256;
constexpr u64 SETUP = 256;             // what a row tile's start and end cost, in keys
constexpr int MIN_SHARE = 512;           // keys of a share, at least
constexpr int PIECES = 32;               // shares that a row tile is cut into, at most (and one more where it begins inside one)
template <int D> constexpr int part_bytes() { return D / 8 * THREADS * 16 + THREADS * 8; }      // D / 8 float4 and (maximum, sum) a lane

struct rows_args {
    const bf16_t *q;
    bf16_t *out;
    unsigned char *part;
    unsigned *cnt;
    kv4_view c;
    kv4_batch b;
    int q_stride, nq, nkv, G, toks;      // toks: tokens of a row tile
    int most;                            // requests of at most this many (row, head) pairs belong to another launch
};

// As in attn_bf16_dtl.hip: the transposing read as an instruction, and the wait for all but the N youngest LDS reads.
template <int OFF> __device__ __forceinline__ bf16x4_v read_tr(uint32_t addr) {
    bf16x4_v r;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF));
    return r;
}
template <int N> __device__ __forceinline__ void tr_wait(bf16x8_t &a, bf16x8_t &b, bf16x8_t &c, bf16x8_t &d) {
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a), "+v"(b), "+v"(c), "+v"(d) : "n"(N));
}
__device__ __forceinline__ float half_swap_max(float v) {
    const unsigned u = __float_as_uint(v);
    const u32x2_v r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D> __global__ __launch_bounds__(THREADS, 2) void attn_kv4_rows_kernel(rows_args a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int WPL = D / 32;                  // code words (8 elements) a lane takes of a key: a quarter of its head
    constexpr int NV = kv4_terms(D, BM);             // bf16 terms of a probability
    constexpr int ROW_B = 2 * D, TILE_B = BN * ROW_B, STAGE_B = 2 * TILE_B;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    __shared__ u64 nan_v[2][4];                  // per stage and loading wave: V blocks that are NaN (masked tiles only)
    __shared__ int there[2][4];                  // ... and whether its 16 keys have a page
    __shared__ int last_arriver;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const kv4_batch &b = a.b;
    const int shift = a.c.page_shift, G = a.G, kvh = blockIdx.x, wg = blockIdx.y;
    const uint32_t lds_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    const int lcol = lane & 31, lgrp = lane >> 5;

    // ---- the line: places in front of every request, and in all
    struct Req { int first, n, base, keys, tiles; u64 places; };
    auto places = [&](u64 from, u64 tiles) { return tiles * (from + SETUP) + (u64)a.toks * (tiles * (tiles + 1) / 2); };
    auto request = [&](int i) {
        const kv4_rows r = kv4_rows_of(scalar(b.row_start), scalar(b.kv_len), b.total_rows, i);
        const int keys = kv4_keys_of(scalar(b.kv_len), b.max_pages, i, shift);
        Req q{r.first, r.n, min(r.base, keys), keys, 0, 0};
        if (r.n * G > a.most) q.tiles = (r.n + a.toks - 1) / a.toks;
        q.places = places((u64)max(0, q.base), (u64)q.tiles);
        return q;
    };
    u64 mine = 0, longest = 0;                   // longest: places of a row tile
    for (int i0 = 0; i0 < b.n_seqs; i0 += 64) {
        const Req q = request(min(i0 + lane, b.n_seqs - 1));
        if (i0 + lane < b.n_seqs) mine += q.places;
        if (q.tiles) longest = max(longest, (u64)max(0, q.base) + (u64)q.tiles * a.toks + SETUP);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) longest = max(longest, (u64)__shfl_xor(longest, o, 64));
    auto scan = [&](u64 x) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const u64 y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        return x;
    };
    u64 incl = scan(mine);
    const u64 all = uniform((u64)__shfl(incl, 63, 64));
    const u64 per = uniform(max(max((all + gridDim.y - 1) / gridDim.y, (u64)MIN_SHARE), (longest + PIECES - 1) / PIECES));
    u64 at = (u64)wg * per;
    const u64 end = min(all, at + per);
    if (at >= end) return;
    const double inv_per = 1.0 / (double)per;
    auto share_of = [&](u64 place) {             // place / per (the quotient is small: off by one at most before it is set right)
        const int w = (int)((double)place * inv_per);
        const u64 p = (u64)w * per;
        return uniform(place < p ? w - 1 : place - p >= per ? w + 1 : w);
    };
    int seq = 0;
    u64 inside = at;                             // place inside the request
    for (int i0 = 0;; i0 += 64) {
        if (b.n_seqs > 64) {
            const Req q = request(min(i0 + lane, b.n_seqs - 1));
            incl = scan(i0 + lane < b.n_seqs ? q.places : 0);
        }
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= inside));
        if (n < 64) {
            seq = i0 + n;
            if (n) inside -= uniform((u64)__shfl(incl, n - 1, 64));
            break;
        }
        inside -= uniform((u64)__shfl(incl, 63, 64));
    }

    // ---- LDS addresses
    const int k_swz = D == 128 ? (lcol & 15) : (lcol >> 1 & 7), k_row = lcol * ROW_B;      // K: lane = key lcol of a 32-key block
    auto v_swz = [](int row) { return D == 128 ? (row & 3) * 5 : ((row >> 1 & 1) << 2 | (row >> 2 & 1)); };
    const int s16 = lane & 15, half16 = lane >> 4 & 1;
    const int v_row = 4 * lgrp + (s16 >> 2);                                               // + 32 sub + 16 t + 8 h
    const int v_chunk = 2 * half16 + ((s16 & 3) >> 1), v_byte = (s16 & 1) << 3;
    const int in_key = lane >> 2, in_q = lane & 3;                                         // on the way in: 16 keys a wave, a quarter a lane
    const int in_row = wave * 16 + in_key;
    const unsigned code_at = in_key * (D / 2) + in_q * WPL * 4, scale_at = in_key * (D / KV4_BLOCK) + in_q * WPL / 4;
    const float sc = 1.4426950408889634f / sqrtf((float)D);

    for (;;) {
        const Req rq = request(seq);
        // ---- the row tile that place `inside` lies in: the largest k with places(k) <= inside
        const u64 from = (u64)max(0, rq.base);
        int tile;
        {
            const double c = (double)from + SETUP + 0.5 * a.toks;
            int k = (int)((sqrt(c * c + 2.0 * a.toks * (double)inside) - c) / a.toks);
            k = max(0, min(rq.tiles - 1, k));
            while (k > 0 && places(from, k) > inside) --k;
            while (k + 1 < rq.tiles && places(from, k + 1) <= inside) ++k;
            tile = uniform(k);
        }
        const u64 begin = uniform(places(from, tile)), span = uniform(places(from, tile + 1)) - begin;
        const u64 s0 = at - (inside - begin);                                  // on the line
        const u64 stop = min(end, s0 + span);
        // ---- this tile's rows
        const int tok0 = tile * a.toks, toks = min(a.toks, rq.n - tok0);
        auto limit = [&](int tok) { return (int)max(0ll, min((long long)rq.keys, (long long)rq.base + tok + 1)); };
        const int lim_lo = limit(tok0), lim_hi = limit(tok0 + toks - 1);
        // keys of this piece, and the workgroups that have pieces of the tile
        auto key_at = [&](u64 place) { return place - s0 < SETUP ? 0 : (int)min((place - s0 - SETUP) / BN, (u64)(KV4_MAX_KEYS / BN)) * BN; };      // (places may pass 31 bits)
        const int ka = key_at(at), kb = stop == s0 + span ? lim_hi : min(lim_hi, key_at(stop));
        auto owner = [&](int block) { return share_of(min(s0 + span, s0 + SETUP + (u64)BN * (block + 1)) - 1); };
        const int w_a = lim_hi > 0 ? owner(0) : share_of(s0), w_b = lim_hi > 0 ? owner((lim_hi - 1) / BN) : w_a;
        const bool has_part = wg >= w_a && wg <= w_b;
        if (has_part) {
            const int row = wave * 32 + lcol, t = row / G, head = kvh * G + (row - t * G);
            const bool real = t < toks;
            const int lim = real ? limit(tok0 + t) : lim_lo;
            bf16x8_t qf[D / 16];
            {
                const bf16_t *qp = a.q + (size_t)(rq.first + tok0 + (real ? t : 0)) * a.q_stride + (size_t)(real ? head : 0) * D + lgrp * 8;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t *>(qp + ks * 16);
            }
            f32x16_t o[D / 32];
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
            float m_run = -INFINITY, l_run = 0.f;                              // maximum in units of the base-2 exponent

            const scalar_ints table = scalar(b.table + (size_t)seq * b.max_pages);
            // whether every key of the piece has a page: then only the tiles at the diagonal are masked
            bool gaps = false;
            for (int p0 = ka >> shift; p0 <= (kb - 1) >> shift; p0 += 64) {
                const int e = table[min(p0 + lane, (kb - 1) >> shift)];
                gaps = gaps || __builtin_amdgcn_ballot_w64((unsigned)e >= (unsigned)a.c.n_pages) != 0;
            }
            struct Codes { unsigned k[WPL], v[WPL]; unsigned ks, vs; int there; };
            auto page_of = [&](int k0) { return k0 + wave * 16 < kb ? table[(k0 + wave * 16) >> shift] : -1; };
            // the wave's 16 keys of the tile at k0 (without a page: whatever the first page holds)
            auto fetch = [&](int k0, int page, Codes &c) {
                c.there = (unsigned)page < (unsigned)a.c.n_pages;
                const u64 tok = (((u64)(unsigned)(c.there ? page : 0) * (unsigned)a.nkv + (unsigned)kvh) << shift) + ((k0 + wave * 16) & (a.c.page - 1));
                const u64 at_c = tok * (D / 2), at_s = tok * (D / KV4_BLOCK);
                const auto rk = beyond(a.c.k, at_c), rv = beyond(a.c.v, at_c), rks = beyond(a.c.ks, at_s), rvs = beyond(a.c.vs, at_s);
                if constexpr (D == 128) {
                    const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(rk, code_at, 0, 0);
                    const u32x4_t y = __builtin_amdgcn_raw_buffer_load_b128(rv, code_at, 0, 0);
#pragma unroll
                    for (int w = 0; w < WPL; ++w) c.k[w] = x[w], c.v[w] = y[w];
                } else {
                    const u32x2_v x = __builtin_amdgcn_raw_buffer_load_b64(rk, code_at, 0, 0);
                    const u32x2_v y = __builtin_amdgcn_raw_buffer_load_b64(rv, code_at, 0, 0);
#pragma unroll
                    for (int w = 0; w < WPL; ++w) c.k[w] = x[w], c.v[w] = y[w];
                }
                c.ks = __builtin_amdgcn_raw_buffer_load_b8(rks, scale_at, 0, 0);
                c.vs = __builtin_amdgcn_raw_buffer_load_b8(rvs, scale_at, 0, 0);
            };
            auto masked = [&](int k0) { return gaps || k0 + BN > lim_lo; };
            // In a masked tile some row does not see some key: V must hold no NaN there (0 x NaN is NaN); where it does is noted, and
            // given to the rows that see it afterwards.
            auto guard = [&](int k0, int stage, Codes &c) {
                const bool seen = c.there && k0 + in_row < lim_hi;
                const uint64_t bad = __builtin_amdgcn_ballot_w64(seen && c.vs == 255);
                if (!seen || c.vs == 255) {
                    c.vs = 127;
#pragma unroll
                    for (int w = 0; w < WPL; ++w) c.v[w] = 0;
                }
                if (lane == 0) nan_v[stage][wave] = bad, there[stage][wave] = c.there;
            };
            auto put_k = [&](int stage, const Codes &c, int w) {
                const int chunk = (in_q * WPL + w) ^ (D == 128 ? (in_row & 15) : (in_row >> 1 & 7));
                *reinterpret_cast<bf16x8_t *>(lds + stage * STAGE_B + in_row * ROW_B + (chunk << 4)) = unpack8(c.k[w], kv4_scale(c.ks));
            };
            auto put_v = [&](int stage, const Codes &c, int w) {
                const int chunk = (in_q * WPL + w) ^ v_swz(in_row);
                *reinterpret_cast<bf16x8_t *>(lds + stage * STAGE_B + TILE_B + in_row * ROW_B + (chunk << 4)) = unpack8(c.v[w], kv4_scale(c.vs));
            };

            // ---- S^T of the tile; behind each matrix instruction of the last groups a part of the next tile is unpacked
            auto scores = [&](int stage, f32x16_t (&s)[2], auto &&behind) {
                const unsigned char *kb_ = lds + stage * STAGE_B;
                constexpr int GPS = D / 64, NGRP = 2 * GPS;                    // groups of four k-steps per 32-key block, and in all
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[sub][r] = 0.f;
                bf16x8_t kf[2][4];
                auto read_k = [&](int buf, int grp) {
                    const int sub = grp / GPS, ks0 = grp % GPS * 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        kf[buf][i] = *reinterpret_cast<const bf16x8_t *>(kb_ + sub * 32 * ROW_B + k_row + (((2 * (ks0 + i) + lgrp) ^ k_swz) << 4));
                };
                read_k(0, 0);
#pragma unroll
                for (int grp = 0; grp < NGRP; ++grp) {
                    if (grp + 1 < NGRP) read_k((grp + 1) & 1, grp + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[grp / GPS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[grp & 1][i], qf[grp % GPS * 4 + i], s[grp / GPS], 0, 0, 0);
                    behind(grp, NGRP);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            auto softmax = [&](int k0, int stage, bool mask, f32x16_t (&s)[2], bf16x8_t (&pb)[NV][2][2]) {
                if (mask) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int vis = there[stage][w] ? lim - k0 - 4 * lgrp : 0;     // of the 16 keys that wave w brought
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            const int key = w * 16 + 8 * (r / 4) + r % 4;
                            s[w / 2][8 * (w % 2) + r] = key < vis ? s[w / 2][8 * (w % 2) + r] : -INFINITY;
                        }
                    }
                }
                float mx = -INFINITY;
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[sub][r]);
                mx *= sc;
                if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {            // some row of the wave saw a new maximum
                    const float m_new = fmaxf(m_run, half_swap_max(mx));
                    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                    m_run = m_new;
                    l_run *= alpha;
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
                }
                const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
                float psum = 0.f;
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[sub][r], sc, neg_m));
                        psum += p;
                        pb[0][sub][r / 8][r % 8] = (bf16_t)p;
                        if constexpr (NV == 2) pb[1][sub][r / 8][r % 8] = (bf16_t)(p - (float)(bf16_t)p);
                    }
                l_run += psum;
            };
            // O^T += V^T P^T: k-slots 8 lgrp .. +8 of step (sub, t) hold keys 32 sub + 16 t + 4 lgrp + {0..3} and the same + 8
            auto second = [&](int stage, bf16x8_t (&pb)[NV][2][2]) {
                bf16x8_t vf[2][4];
                const uint32_t base = lds_addr + (uint32_t)(stage * STAGE_B + TILE_B + v_row * ROW_B + v_byte);
                auto read_v = [&](int buf, int dt) {
                    const uint32_t x = base + (uint32_t)(((4 * dt + v_chunk) ^ v_swz(v_row)) << 4);
                    vf[buf][0] = __builtin_shufflevector(read_tr<0 * ROW_B>(x), read_tr<8 * ROW_B>(x), 0, 1, 2, 3, 4, 5, 6, 7);
                    vf[buf][1] = __builtin_shufflevector(read_tr<16 * ROW_B>(x), read_tr<24 * ROW_B>(x), 0, 1, 2, 3, 4, 5, 6, 7);
                    vf[buf][2] = __builtin_shufflevector(read_tr<32 * ROW_B>(x), read_tr<40 * ROW_B>(x), 0, 1, 2, 3, 4, 5, 6, 7);
                    vf[buf][3] = __builtin_shufflevector(read_tr<48 * ROW_B>(x), read_tr<56 * ROW_B>(x), 0, 1, 2, 3, 4, 5, 6, 7);
                };
                read_v(0, 0);
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    if (dt + 1 < D / 32) {
                        read_v((dt + 1) & 1, dt + 1);
                        __builtin_amdgcn_sched_barrier(0);
                        tr_wait<8>(vf[dt & 1][0], vf[dt & 1][1], vf[dt & 1][2], vf[dt & 1][3]);
                    } else {
                        __builtin_amdgcn_sched_barrier(0);
                        tr_wait<0>(vf[dt & 1][0], vf[dt & 1][1], vf[dt & 1][2], vf[dt & 1][3]);
                    }
#pragma unroll
                    for (int st = 0; st < 4; ++st)
#pragma unroll
                        for (int p = 0; p < NV; ++p)
                            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt & 1][st], pb[p][st >> 1][st & 1], o[dt], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            auto give_nan = [&](int k0, int stage) {
                unsigned blocks = 0;                                           // bit = a quarter of the head
                for (int w = 0; w < 4; ++w)
                    for (uint64_t m = nan_v[stage][w]; m; m &= m - 1) {
                        const int bit = __builtin_ctzll(m);
                        if (k0 + w * 16 + (bit >> 2) < lim) blocks |= 1u << (bit & 3);
                    }
                if (__builtin_amdgcn_ballot_w64(blocks != 0) == 0) return;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (blocks >> (D == 128 ? dt : dt * 2 + r / 8) & 1) o[dt][r] = NAN;
            };

            if (ka < kb) {
                // Two tiles of codes are on their way: what is unpacked behind the products of tile j was requested before those of j - 1.
                Codes c0, c1;
                fetch(ka, page_of(ka), c0);
                fetch(ka + BN, page_of(ka + BN), c1);                          // behind the piece: no page, not used
                int page = page_of(ka + 2 * BN);
                if (masked(ka)) guard(ka, 0, c0);
#pragma unroll
                for (int w = 0; w < WPL; ++w) put_k(0, c0, w), put_v(0, c0, w);
                int k0 = ka;
                auto step = [&](auto stage_c, Codes &next, Codes &later) {     // stage_c: LDS stage of the tile at k0; next: the tile behind it
                    constexpr int stage = decltype(stage_c)::value;
                    fetch(k0 + 2 * BN, page, later);
                    page = page_of(k0 + 3 * BN);
                    __syncthreads();                                           // this stage is written, the other one read
                    const bool mask = masked(k0);
                    if (masked(k0 + BN)) guard(k0 + BN, stage ^ 1, next);
                    f32x16_t s[2];
                    bf16x8_t pb[NV][2][2];
                    // Products go before the other workgroup's softmax: 2048 rows over 32768 keys 352 -> 330 us, over 131072 1197 -> 1131.
                    __builtin_amdgcn_s_setprio(1);
                    scores(stage, s, [&](int grp, int of) {                    // a word of K and one of V behind each group
                        put_k(stage ^ 1, next, grp * WPL / of);
                        put_v(stage ^ 1, next, grp * WPL / of);
                    });
                    __builtin_amdgcn_s_setprio(0);
                    softmax(k0, stage, mask, s, pb);
                    __builtin_amdgcn_s_setprio(1);
                    second(stage, pb);
                    __builtin_amdgcn_s_setprio(0);
                    if (mask) give_nan(k0, stage);
                    k0 += BN;
                };
                while (k0 < kb) {
                    step(std::integral_constant<int, 0>{}, c1, c0);
                    if (k0 >= kb) break;
                    step(std::integral_constant<int, 1>{}, c0, c1);
                }
            }
            l_run += __shfl_xor(l_run, 32, 64);

            bool writes = true;
            if (w_b > w_a) {
                const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(a.part + (size_t)kvh * gridDim.y * 2 * part_bytes<D>()), 0, (int)(gridDim.y * 2 * part_bytes<D>()), 0x00020000);
                auto slot = [&](int w) { return (unsigned)(2 * w + (w == w_a ? 1 : 0)) * part_bytes<D>(); };
                {
                    const unsigned p = slot(wg);
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const f32x4_t v = {o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]};
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), rp, p + ((dt * 4 + x) * THREADS + tid) * 16, 0, COHERENT);
                        }
                    const u32x2_v ml = {__float_as_uint(m_run), __float_as_uint(l_run)};
                    __builtin_amdgcn_raw_buffer_store_b64(ml, rp, p + D / 8 * THREADS * 16 + tid * 8, 0, COHERENT);
                }
                __builtin_amdgcn_s_waitcnt(0);       // my stores have reached memory ...
                __syncthreads();                     // ... and so have everybody's, before the arrival is counted
                if (tid == 0) {
                    unsigned *cnt = a.cnt + kvh * gridDim.y + w_a;
                    const unsigned n = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
                    last_arriver = n == (unsigned)(w_b - w_a);
                    if (last_arriver) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
                }
                __syncthreads();
                writes = last_arriver != 0;
                if (writes) {
                    m_run = -INFINITY;
                    l_run = 0.f;
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
                    for (int w = w_a; w <= w_b; ++w) {
                        const unsigned p = slot(w);
                        f32x4_t v[D / 8];
#pragma unroll
                        for (int x = 0; x < D / 8; ++x)
                            v[x] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rp, p + (x * THREADS + tid) * 16, 0, COHERENT));
                        const u32x2_v ml = __builtin_amdgcn_raw_buffer_load_b64(rp, p + D / 8 * THREADS * 16 + tid * 8, 0, COHERENT);
                        const float mw = __uint_as_float(ml[0]), m_new = fmaxf(m_run, mw);
                        const float fa = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                        const float fb = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw - m_new);
                        m_run = m_new;
                        l_run = l_run * fa + __uint_as_float(ml[1]) * fb;
#pragma unroll
                        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                            for (int r = 0; r < 16; ++r) o[dt][r] = o[dt][r] * fa + v[dt * 4 + r / 4][r % 4] * fb;
                    }
                }
            }
            if (writes && real) {
                const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
                bf16_t *op = a.out + ((size_t)(rq.first + tok0 + t) * a.nq + head) * D;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const bf16x4_v v = {(bf16_t)(o[dt][4 * x] * inv), (bf16_t)(o[dt][4 * x + 1] * inv), (bf16_t)(o[dt][4 * x + 2] * inv),
                                            (bf16_t)(o[dt][4 * x + 3] * inv)};
                        *reinterpret_cast<bf16x4_v *>(op + dt * 32 + 8 * x + 4 * lgrp) = v;
                    }
            }
            __syncthreads();                         // the stages are read; the next tile writes them
        }
        // ---- on along the line
        at = uniform(stop);
        if (at >= end) break;
        inside = begin + span;                       // a new tile: stop was the end of this one
        if (tile + 1 == rq.tiles) {
            inside = 0;
            do {
                seq = uniform(seq + 1);
            } while (request(seq).tiles == 0);
        }
    }
#endif
}

int rows_wgs(int nkv, int ncu) { return max(1, 2 * min(ncu, 512) / nkv); }     // per key head: two workgroups on a compute unit

}  // namespace

size_t iso_attn_kv4_rows_ws_bytes(int nkv, int d, int ncu) {
    const size_t wgs = (size_t)rows_wgs(nkv, ncu) * nkv;
    return ((wgs * 4 + 255) & ~(size_t)255) + wgs * 2 * (d == 64 ? part_bytes<64>() : part_bytes<128>());
}

hipError_t iso_launch_attn_kv4_rows(const void *q, int q_stride, const iso_kv4 &cache, const kv4_batch &b, int most, void *out, int nq, int nkv,
                                    int d, void *ws, hipStream_t s) {
    const int G = nq / nkv, wgs = rows_wgs(nkv, iso_num_cu());
    rows_args a{(const bf16_t *)q, (bf16_t *)out, nullptr, (unsigned *)ws, kv4_view_of(cache), b, q_stride, nq, nkv, G, BM / G, most};
    a.part = (unsigned char *)ws + (((size_t)wgs * nkv * 4 + 255) & ~(size_t)255);
    const int lds = 2 * 2 * BN * 2 * d;
    static iso_dev_mask allowed[2];
    const void *kernel = d == 64 ? (const void *)attn_kv4_rows_kernel<64> : (const void *)attn_kv4_rows_kernel<128>;
    if (hipError_t e = iso_allow_lds(kernel, lds, &allowed[d == 64]); e != hipSuccess) return e;
    if (d == 64) hipLaunchKernelGGL(attn_kv4_rows_kernel<64>, dim3(nkv, wgs), dim3(THREADS), lds, s, a);
    else hipLaunchKernelGGL(attn_kv4_rows_kernel<128>, dim3(nkv, wgs), dim3(THREADS), lds, s, a);
    return hipGetLastError();
}
