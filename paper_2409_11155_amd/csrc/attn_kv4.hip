// Attention of a ragged batch over the paged 4-bit cache: decoding steps (bound by the cache's bytes) and chunks of prompts (bound by the
// instructions of the softmax and of unpacking, then by the matrix cores).
//
// A row tile is 16 * RT (row, query head) pairs of one key head.  Same mathematics as the other attention kernels: S^T = K Q^T, so that the
// softmax statistics are per-lane scalars and the probabilities feed O^T = V^T P^T from registers; v_mfma_f32_16x16x32_bf16.  A value of the
// cache is a bf16 number, so unpacking is exact: v_cvt_scalef32_pk_bf16_fp4 makes two elements an instruction, scale included.
//   * K goes from the page into the registers that the product wants: the four lanes of a key take a quarter of its head each, 16 (8)
//     bytes, and element order inside the head is free as long as q is read in the same one.  No LDS.
//   * V has to be transposed: a wave writes its 32 unpacked rows to LDS (its own 8 KB, no barrier) and reads them back with
//     ds_read_b64_tr_b16.  16-byte chunks are XOR-swizzled by the row (heads of 128: the LDS works in 23 % of the cycles, a fifth of that
//     on bank conflicts).
//   * RT = 2: what is unpacked once serves two blocks of 16 rows.  The second one is passed over where the tile does not reach it.
//   * T = float: q and the probabilities are cut into three bf16 terms that add up to all 24 bits (K and V have two): three products.
//
// Work: for each key head the row tiles of all requests lie on one line, which is cut into equal shares, a workgroup each, whatever the
// requests' lengths are.  Tile k of a request takes SETUP + max(0, kv_len - rows) + 1 + (k + 1) * ROWS / G keys there (G query heads a key
// head: a tile further down sees more keys; SETUP: its start and end), so a request's length is a closed form and a place's tile the root
// of a quadratic.  Places are counted in 1 / G of a key.  A workgroup's four waves take 32 keys of every 128 each and meet in LDS at the end
// of a tile.  A tile that crosses workgroups is parked in pieces (running maximum, sum, unnormalised output) with cache-bypassing stores;
// the workgroup that arrives last folds them in the order of the line, so the result does not depend on who that is, and puts the counter
// back to zero.  Nobody waits for anybody.  The shares are computed on the device from the lengths there: a captured step keeps its balance
// as the requests grow.
//
// Measured (bf16): 40 single tokens over 500 to 8192 keys, 13 heads of 128, 44.6 us, 4.1 TB/s of the cache (a large copy reaches 4.9);
// 48 x 2 rows over 300 to 8192 keys, 32 heads of 64 over 8, 21.7 us, 2.8 TB/s: shares of 600 to 1100 keys behind 4 to 5 us of start and end;
// one token over 131072 keys, 8 heads over 1, 16.9 us: 254 shares take 2 us to be found (some 600 dependent instructions and a trip to
// memory), 5 for their keys, 1 to be parked and 5 to be folded in two rounds.  32 rows a tile, 16 heads over 2: 64 rows over 32768 keys 46 us
// (370 TFLOP/s); 2 x 509 rows and 22 single tokens over 700 to 6000 keys 37 to 40 us (up to 330), vector instructions in 50 %, matrix
// instructions in 16 % of the cycles, and workgroups that end between 32 and 40 us: every tile unpacks its request's keys again, 128
// tiles of 32 rows those of a 509-row chunk.  fp32: 40 single tokens of 4000 keys, 13 heads, 63 to 76 us; 512 rows of 4096 keys, 8 heads over 1,
// 40; 512 of 2000, 13 heads, 34; heads of 64, 32 over 8, 2048 of 2048 91.
#include "kv4.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, TILE = 32, UNIT = WAVES * TILE;
constexpr int GROUP = 16;             // pieces that are folded at once, at most; a tile has up to GROUP * GROUP of them
constexpr int SETUP = 512;            // what a tile's start and end cost, in keys
constexpr int ROUND = 256;            // keys that cost what a second round of folding does: 18 rows, 7300 keys each, 22.4 us with two, 17.1 with one
constexpr int MIN_SHARE = 256;        // keys of a share, at least
constexpr int SPLITS = GROUP * GROUP - 2;  // shares that the longest tile is cut into, at most (a share may begin and end inside it)

// Workgroups on a compute unit, by the registers.
constexpr int wg_per_cu(int elt, int d, int rt) { return elt == 4 ? (d == 64 ? 3 : 2) : rt == 2 ? (d == 64 ? 3 : 2) : d == 64 ? 4 : 3; }
constexpr int slot_floats(int d, int rt) { return 16 * rt * (d + 2); }       // output rows, then maxima, then sums

struct line_args {
    const void *q;
    void *out;
    float *part;
    unsigned *cnt;
    kv4_view c;
    kv4_batch b;
    int q_stride, nq, nkv, G;            // G: query heads of a key head
    unsigned g_mul, g_bits;              // x / G = (x * g_mul / 2^32 + x) >> g_bits for x below 2^31
    int most;                            // requests of more (row, head) pairs than this belong to another launch
};

__device__ __forceinline__ bf16x4_v read_tr(unsigned addr) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4_v *)(uintptr_t)addr);
}

// x as a sum of NP bf16 terms: the nearest, and the nearest of what is left (NP = 1, 2), or cut off so that three terms are all of x.
template <int NP> __device__ __forceinline__ void split(float x, bf16_t (&t)[NP]) {
    if constexpr (NP < 3) {
        t[0] = (bf16_t)x;
        if constexpr (NP == 2) t[1] = (bf16_t)(x - (float)t[0]);
    } else {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float cut = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
            t[p] = (bf16_t)cut;
            x -= cut;
        }
    }
}

// x / d, with inv about 1 / d: the estimate is off by one at most (quotients below 2^20 in 32 bits, below 2^24 in 64) before it is set right.
template <typename F> __device__ __forceinline__ int quotient(u64 x, u64 d, F inv) {
    const int q = (int)((F)x * inv);
    const u64 p = (u64)(unsigned)q * d;
    return uniform(x < p ? q - 1 : x - p >= d ? q + 1 : q);
}

// Inclusive sum over the wave and its maximum, lane 63 holds all of it: row shifts, then the last lanes of the rows handed on (DPP, no LDS).
template <int CTRL, int ROW_MASK> __device__ __forceinline__ u64 moved(u64 x) {
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROW_MASK, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROW_MASK, 0xf, false);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_scan(u64 x) {
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);
    return x + moved<0x143, 0xc>(x);
}
template <int CTRL, int ROW_MASK> __device__ __forceinline__ float moved(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROW_MASK, 0xf, false));
}
__device__ __forceinline__ float wave_max(float x) {           // of numbers >= 0
    x = fmaxf(x, moved<0x111, 0xf>(x));
    x = fmaxf(x, moved<0x112, 0xf>(x));
    x = fmaxf(x, moved<0x114, 0xf>(x));
    x = fmaxf(x, moved<0x118, 0xf>(x));
    x = fmaxf(x, moved<0x142, 0xa>(x));
    x = fmaxf(x, moved<0x143, 0xc>(x));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ u64 lane_of(u64 x, int lane) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)x, lane) | (u64)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32;
}


template <typename T, int D, int RT>
__global__ __launch_bounds__(THREADS, wg_per_cu(sizeof(T), D, RT)) void attn_kv4_kernel(line_args a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;               // bf16 terms of a query element ...
    constexpr int NV = sizeof(T) == 4 ? 3 : kv4_terms(D, 16 * RT);    // ... and of a probability
    constexpr int ROWS = 16 * RT;
    constexpr int WPL = D / 32;              // code words (8 elements) a lane takes of a key
    constexpr int RB = 2 * D;                // bytes of an unpacked row
    constexpr int VG = D == 64 && RT == 1 ? 2 : 1;      // blocks of 16 dims of V that are read at a time (two would not fit the registers beside two row blocks)
    __shared__ __attribute__((aligned(1024))) unsigned char lds[WAVES * TILE * RB];
    __shared__ float ml[2][WAVES][16];
    __shared__ int last_arriver;

    const int tid = threadIdx.x, lane = tid & 63, n16 = lane & 15, g4 = lane >> 4;
    const int wave = uniform(tid >> 6);
    const kv4_batch &b = a.b;
    const int shift = a.c.page_shift, G = a.G, kvh = blockIdx.x, wg = blockIdx.y;
    auto by_g = [&](int x) { return (int)((__umulhi((unsigned)x, a.g_mul) + (unsigned)x) >> a.g_bits); };

    // ---- the line: places in front of every request, and in all.  Every wave does this for itself, 64 requests at a time: no barrier,
    // and for up to 64 of them one trip to memory.
    struct Req { int first, n, base, keys; unsigned tiles; u64 start; };       // start: places of a tile before the (k + 1) * ROWS
    auto request = [&](int i) {
        const kv4_rows r = kv4_rows_of(scalar(b.row_start), scalar(b.kv_len), b.total_rows, i);
        const int keys = kv4_keys_of(scalar(b.kv_len), b.max_pages, i, shift), base = min(r.base, keys);
        return Req{r.first, r.n, base, keys, r.n * G > a.most ? 0u : (unsigned)(r.n * G + ROWS - 1) / ROWS, (u64)(unsigned)G * ((unsigned)max(0, base) + 1u + SETUP)};
    };
    auto places = [](const Req &q, unsigned k) { return k * q.start + (u64)ROWS * ((u64)k * (k + 1) / 2); };      // of the first k tiles
    auto of_lane = [&](int i) { return i < b.n_seqs ? places(request(i), request(i).tiles) : 0; };
    u64 mine = 0;
    float longest = 0.f;
    Req here;                                    // of the lane, where there are no more than 64 requests
    for (int i0 = 0; i0 < b.n_seqs; i0 += 64) {
        const int i = min(i0 + lane, b.n_seqs - 1);
        here = request(i);
        if (i == i0 + lane) mine += places(here, here.tiles);
        if (here.tiles) longest = fmaxf(longest, (float)here.start + (float)ROWS * (float)here.tiles);
    }
    u64 incl = wave_scan(mine);
    const u64 all = lane_of(incl, 63);
    longest = wave_max(longest);
    // Any share does that covers the line (2^-17 more than its part, for the roundings); never less than MIN_SHARE keys, nor so little that
    // a tile has more pieces than can be folded.
    constexpr float MORE = 1.f + 0x1p-17f;
    float share = fmaxf(fmaxf((float)all * (MORE * __builtin_amdgcn_rcpf((float)gridDim.y)), longest * (MORE / SPLITS)), (float)(G * MIN_SHARE));
    // one round of folding instead of two where that lengthens a share by less than ROUND keys
    const float one_round = longest * (MORE / (GROUP - 1));
    if (one_round > share && one_round - share < (float)(G * ROUND)) share = one_round;
    u64 per = (u64)share + 1;
    per = uniform(per);
    u64 at = (u64)wg * per;
    const u64 end = min(all, at + per);
    if (at >= end) return;
    const float inv_per = __builtin_amdgcn_rcpf((float)per);
    const double inv_unit = __builtin_amdgcn_rcp((double)(UNIT * G));
    int seq = 0;
    u64 inside = at;                             // place inside the request
    for (int i0 = 0;; i0 += 64) {
        if (b.n_seqs > 64) incl = wave_scan(of_lane(i0 + lane));
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= inside));      // requests that end before it
        if (n < 64) {
            seq = i0 + n;
            if (n) inside -= lane_of(incl, n - 1);
            break;
        }
        inside -= lane_of(incl, 63);
    }

    const float sc = 1.4426950408889634f / sqrtf((float)D);
    const unsigned lds_w = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * TILE * RB;
    auto swz = [](int row) { return D == 128 ? (row & 15) : ((row >> 1 & 3) << 1 | (row >> 3 & 1)); };
    // V: the lane's row on the way in is n16 (+ 16), on the way out 4 g4 + n16 / 4 (+ 16)
    unsigned char *const v_in = lds + wave * TILE * RB + n16 * RB;
    const int in_swz = swz(n16);
    const unsigned code_at = n16 * (D / 2) + g4 * WPL * 4, scale_at = n16 * (D / KV4_BLOCK) + g4 * WPL / 4;
    const int out_row = 4 * g4 + (n16 >> 2);
    const unsigned v_out = lds_w + out_row * RB + ((((n16 & 3) >> 1) ^ swz(out_row)) << 4) + ((n16 & 1) << 3);

    // (what a lane has read already is not read again: a trip to memory)
    Req rq;
    if (b.n_seqs <= 64) {
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, seq); };
        rq = Req{of(here.first), of(here.n), of(here.base), of(here.keys), (unsigned)of((int)here.tiles), lane_of(here.start, seq)};
    } else {
        rq = request(seq);
    }
    for (;;) {
        // ---- the tile that place `inside` lies in: the largest k with places(k) <= inside
        unsigned tile = 0;
        if (rq.tiles > 1) {
            const float c = ((float)rq.start + 0.5f * ROWS) * (1.f / ROWS), x = (2.f / ROWS) * (float)inside;      // root of k^2 + 2 c k = x
            tile = min(rq.tiles - 1, (unsigned)(x * __builtin_amdgcn_rcpf(c + __builtin_amdgcn_sqrtf(c * c + x))));
            while (tile > 0 && places(rq, tile) > inside) --tile;
            while (tile + 1 < rq.tiles && places(rq, tile + 1) <= inside) ++tile;
            tile = (unsigned)uniform((int)tile);
        }
        const u64 begin = places(rq, tile), s0 = at - (inside - begin), s1 = s0 + rq.start + (u64)ROWS * (tile + 1);      // on the line
        const u64 stop = min(end, s1);
        const int pairs = rq.n * G, first_pair = (int)tile * ROWS;
        const bool two = RT == 2 && pairs - first_pair > 16;
        auto limit = [&](int tok) { return (int)max(0ll, min((long long)rq.keys, (long long)rq.base + tok + 1)); };      // keys that a token sees
        const int lim_lo = uniform(limit(by_g(first_pair))), lim_hi = uniform(limit(by_g(min(pairs, first_pair + ROWS) - 1)));
        // ---- the piece's keys (the share begins and ends at multiples of UNIT keys of the tile), and the workgroups that have pieces
        const u64 s_keys = s0 + (u64)G * SETUP;
        // (a tile's places may lie past its last key, and past 31 bits: the limit is beyond every key)
        auto key_at = [&](u64 place) { return place < s_keys ? 0 : min(quotient(place - s_keys, (u64)G * UNIT, inv_unit), KV4_MAX_KEYS / UNIT) * UNIT; };
        const int ka = at == s0 ? 0 : key_at(at), kb = stop == s1 ? lim_hi : min(lim_hi, key_at(stop));
        auto owner = [&](int u) { return quotient(min(s1, s_keys + (u64)G * UNIT * (unsigned)(u + 1)) - 1, per, inv_per); };
        const int w0 = lim_hi > 0 ? owner(0) : quotient(s0, per, inv_per), w1 = lim_hi > UNIT ? owner((lim_hi - 1) / UNIT) : w0;
        if (wg >= w0 && wg <= w1) {
            // ---- this tile's rows
            bool real[RT];
            int lim[RT];
            bf16x8_t qf[NP][RT][WPL];
            f32x4_t o[RT][D / 16];
            float m_run[RT], l_run[RT];                // maximum in units of the base-2 exponent
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const int r = first_pair + 16 * x + n16, t = by_g(r), head = kvh * G + (r - t * G);
                real[x] = r < pairs;
                lim[x] = real[x] ? limit(t) : lim_lo;
                const T *qp = (const T *)a.q + (size_t)(rq.first + (real[x] ? t : 0)) * a.q_stride + (size_t)(real[x] ? head : 0) * D + g4 * WPL * 8;
                typedef T row8 __attribute__((ext_vector_type(8)));
#pragma unroll
                for (int w = 0; w < WPL; ++w) {
                    const row8 v = *reinterpret_cast<const row8 *>(qp + w * 8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        bf16_t part[NP];
                        split<NP>(real[x] ? iso_to_f32((T)v[e]) : 0.f, part);
#pragma unroll
                        for (int p = 0; p < NP; ++p) qf[p][x][w][e] = part[p];
                    }
                }
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) o[x][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                m_run[x] = -INFINITY;
                l_run[x] = 0.f;
            }

            const scalar_ints table = scalar(b.table + (size_t)seq * b.max_pages);
            struct Pages { int p[2]; };
            auto pages_of = [&](int k0) {
                Pages x;
#pragma unroll
                for (int h = 0; h < 2; ++h) x.p[h] = k0 + 16 * h < kb ? table[(k0 + 16 * h) >> shift] : -1;
                return x;
            };
            struct Codes { unsigned k[2][WPL], v[2][WPL]; unsigned ks[2], vs[2]; int there; };
            // Codes and scales of the wave's 32 keys from k0 on.  Where there is no page the first one is read instead, and what lies behind
            // the last visible key is read too: multiply() leaves both out.
            auto fetch = [&](int k0, const Pages &pages, Codes &c) {
                c.there = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool there = (unsigned)pages.p[h] < (unsigned)a.c.n_pages;
                    c.there |= (int)there << h;
                    const u64 tok = (((u64)(unsigned)(there ? pages.p[h] : 0) * (unsigned)a.nkv + (unsigned)kvh) << shift) + ((k0 + 16 * h) & (a.c.page - 1));
                    const u64 at_c = tok * (D / 2), at_s = tok * (D / KV4_BLOCK);
                    const auto rk = beyond(a.c.k, at_c), rv = beyond(a.c.v, at_c), rks = beyond(a.c.ks, at_s), rvs = beyond(a.c.vs, at_s);
                    if constexpr (D == 128) {
                        const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(rk, code_at, 0, 0);
                        const u32x4_t y = __builtin_amdgcn_raw_buffer_load_b128(rv, code_at, 0, 0);
#pragma unroll
                        for (int w = 0; w < WPL; ++w) c.k[h][w] = x[w], c.v[h][w] = y[w];
                    } else {
                        const u32x2_v x = __builtin_amdgcn_raw_buffer_load_b64(rk, code_at, 0, 0);
                        const u32x2_v y = __builtin_amdgcn_raw_buffer_load_b64(rv, code_at, 0, 0);
#pragma unroll
                        for (int w = 0; w < WPL; ++w) c.k[h][w] = x[w], c.v[h][w] = y[w];
                    }
                    c.ks[h] = __builtin_amdgcn_raw_buffer_load_b8(rks, scale_at, 0, 0);
                    c.vs[h] = __builtin_amdgcn_raw_buffer_load_b8(rvs, scale_at, 0, 0);
                }
            };
            auto multiply = [&](int k0, Codes &c, auto second_c) {
                constexpr int N = decltype(second_c)::value ? RT : 1;          // blocks of 16 rows
                // rows of the tile that do not see all 32 keys: their probabilities are zero, and V must not be NaN there
                const bool masked = k0 + TILE > lim_lo || c.there != 3;
                uint64_t nan_v[2] = {0, 0};
                if (masked) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool seen = (c.there >> h & 1) && k0 + 16 * h + n16 < lim_hi;
                        nan_v[h] = __builtin_amdgcn_ballot_w64(seen && c.vs[h] == 255);
                        if (!seen || c.vs[h] == 255) {
                            c.vs[h] = 127;
#pragma unroll
                            for (int w = 0; w < WPL; ++w) c.v[h][w] = 0;
                        }
                    }
                }
                f32x4_t s[RT][2];
                // unpacking and scores go before the other workgroups' softmax: 64 rows x 16 heads over 32768 keys 49.6 -> 47.1 us
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int x = 0; x < N; ++x) s[x][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    const float f = kv4_scale(c.ks[h]);
#pragma unroll
                    for (int w = 0; w < WPL; ++w) {
                        const bf16x8_t kf = unpack8(c.k[h][w], f);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
#pragma unroll
                            for (int x = 0; x < N; ++x) s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][x][w], s[x][h], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float f = kv4_scale(c.vs[h]);
#pragma unroll
                    for (int w = 0; w < WPL; ++w)
                        *reinterpret_cast<bf16x8_t *>(v_in + h * 16 * RB + (((g4 * WPL + w) ^ in_swz) << 4)) = unpack8(c.v[h][w], f);
                }
                // V comes back VG blocks of 16 dims at a time: the first ones while the probabilities are computed, then one group ahead
                bf16x8_t vf[2][VG];
                auto read_v = [&](int buf, int dt0) {
#pragma unroll
                    for (int i = 0; i < VG; ++i) {
                        const unsigned from = v_out ^ (unsigned)((dt0 + i) << 5);
                        vf[buf][i] = __builtin_shufflevector(read_tr(from), read_tr(from + 16 * RB), 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                };
                read_v(0, 0);
                __builtin_amdgcn_s_setprio(0);
                __builtin_amdgcn_sched_barrier(0);
                float mx[RT];
                bool moves = false;
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    if (masked) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int vis = c.there >> h & 1 ? lim[x] - k0 - 16 * h - 4 * g4 : 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[x][h][e] = e < vis ? s[x][h][e] : -INFINITY;
                        }
                    }
                    mx[x] = -INFINITY;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) mx[x] = fmaxf(mx[x], s[x][h][e]);
                    mx[x] *= sc;
                    moves = moves || mx[x] > m_run[x];
                }
                // the running maximum moves rarely deep in a cache; the four lanes of a row agree on it
                if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
                    for (int x = 0; x < N; ++x) {
                        float top = fmaxf(mx[x], __shfl_xor(mx[x], 16, 64));
                        top = fmaxf(m_run[x], fmaxf(top, __shfl_xor(top, 32, 64)));
                        const float alpha = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[x] - top);
                        m_run[x] = top;
                        l_run[x] *= alpha;
#pragma unroll
                        for (int dt = 0; dt < D / 16; ++dt) o[x][dt] *= alpha;
                    }
                }
                bf16x8_t pb[RT][NV];
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float neg_m = m_run[x] == -INFINITY ? 0.f : -m_run[x];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = __builtin_amdgcn_exp2f(fmaf(s[x][h][e], sc, neg_m));
                            l_run[x] += p;
                            bf16_t part[NV];
                            split<NV>(p, part);
#pragma unroll
                            for (int y = 0; y < NV; ++y) pb[x][y][4 * h + e] = part[y];
                        }
                }
#pragma unroll
                for (int grp = 0; grp < D / 16 / VG; ++grp) {
                    if (grp + 1 < D / 16 / VG) read_v((grp + 1) & 1, VG * (grp + 1));
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < VG; ++i)
#pragma unroll
                        for (int p = 0; p < NV; ++p)
#pragma unroll
                            for (int x = 0; x < N; ++x)
                                o[x][VG * grp + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[grp & 1][i], pb[x][p], o[x][VG * grp + i], 0, 0, 0);
                }
                // a token whose V is NaN in some block: so is that block of the rows that see it, and of no others
                if ((nan_v[0] | nan_v[1]) != 0) {
#pragma unroll
                    for (int x = 0; x < N; ++x) {
                        unsigned blocks = 0;               // bit = 16 dims
                        for (int h = 0; h < 2; ++h)
                            for (uint64_t m = h ? nan_v[1] : nan_v[0]; m; m &= m - 1) {
                                const int bit = __builtin_ctzll(m);
                                if (k0 + 16 * h + (bit & 15) < lim[x]) blocks |= ((1u << D / 64) - 1) << (bit >> 4) * (D / 64);
                            }
#pragma unroll
                        for (int dt = 0; dt < D / 16; ++dt)
                            if (blocks >> dt & 1) o[x][dt] = f32x4_t{NAN, NAN, NAN, NAN};
                    }
                }
            };
            // Codes are requested a tile ahead and page numbers two, without a branch: behind the share's end there are no pages, and
            // what has none is not fetched.  (A branch around the requests would make every wait one for all of them.)
            auto keys = [&](auto second_c) {
                int k0 = ka + wave * TILE;
                Codes c0, c1;
                fetch(k0, pages_of(k0), c0);
                Pages pages = pages_of(k0 + UNIT);
                auto step = [&](Codes &now, Codes &later) {
                    fetch(k0 + UNIT, pages, later);
                    pages = pages_of(k0 + 2 * UNIT);
                    multiply(k0, now, second_c);
                    k0 += UNIT;
                };
                while (k0 < kb) {
                    step(c0, c1);
                    if (k0 >= kb) break;
                    step(c1, c0);
                }
            };
            if (RT == 2 && two) keys(std::true_type{});
            else keys(std::false_type{});

            // ---- the four waves' states, 16 rows at a time: thread = (row, 16th of the head)
            constexpr int CPT = D / 64;              // float4 of a row that a thread has
            const int row = tid >> 4, col = tid & 15;
            f32x4_t sum[RT][CPT];
            float m[RT], l[RT];
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                l_run[x] += __shfl_xor(l_run[x], 16, 64);
                l_run[x] += __shfl_xor(l_run[x], 32, 64);
                if (x) __syncthreads();
                float *mine_o = reinterpret_cast<float *>(lds + wave * TILE * RB) + n16 * D;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4_t *>(mine_o + (((4 * dt + g4) ^ n16) << 2)) = o[x][dt];
                if (g4 == 0) ml[0][wave][n16] = m_run[x], ml[1][wave][n16] = l_run[x];
                __syncthreads();
                m[x] = -INFINITY;
                l[x] = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) m[x] = fmaxf(m[x], ml[0][w][row]);
#pragma unroll
                for (int y = 0; y < CPT; ++y) sum[x][y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = m[x] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[0][w][row] - m[x]);      // no score but NaN: zeros and NaN add up
                    l[x] += ml[1][w][row] * f;
                    const float *po = reinterpret_cast<const float *>(lds + w * TILE * RB) + row * D;
#pragma unroll
                    for (int y = 0; y < CPT; ++y) sum[x][y] += *reinterpret_cast<const f32x4_t *>(po + (((col * CPT + y) ^ row) << 2)) * f;
                }
            }
            const int rows = min(ROWS, pairs - first_pair);
            bool writes = true;
            if (w1 > w0) {
                // ---- a piece of the tile: park it.  Up to GROUP pieces are folded by the workgroup that arrives last.  More of them go in
                // groups of about their number's root, 8 or 16: the last to arrive of a group folds it, the last of those the groups'.  (A
                // compute unit gets about 45 GB/s of pieces from memory: 126 of 4 KB took one workgroup 13 us.  16 rows, 16 heads over 2,
                // 8192 keys, pieces of 16 KB: 25.7 us with groups of 16, 22.4 with smaller ones.)
                constexpr int SLOT = slot_floats(D, RT) * 4;
                const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc((char *)a.part + (size_t)kvh * gridDim.y * 2 * SLOT, 0, (int)(gridDim.y * 2 * SLOT), 0x00020000);
                auto index = [&](int w) { return 2 * w + (w == w0 ? 1 : 0); };      // a workgroup's tile from before, or the one begun here
                auto park = [&](int w) {
                    const unsigned p = (unsigned)index(w) * SLOT;
#pragma unroll
                    for (int x = 0; x < RT; ++x)
                        if (16 * x + row < rows) {
#pragma unroll
                            for (int y = 0; y < CPT; ++y)
                                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, sum[x][y]), rp, p + (16 * x + row) * D * 4 + (col * CPT + y) * 16, 0, COHERENT);
                            if (col == 0) {
                                const u32x2_v v = {__float_as_uint(m[x]), __float_as_uint(l[x])};
                                __builtin_amdgcn_raw_buffer_store_b64(v, rp, p + ROWS * D * 4 + (16 * x + row) * 8, 0, COHERENT);
                            }
                        }
                };
                auto last_of = [&](unsigned *cnt, int n) {
                    __builtin_amdgcn_s_waitcnt(0);       // my stores have reached memory ...
                    __syncthreads();                     // ... and so have everybody's, before the arrival is counted
                    if (tid == 0) {
                        const unsigned before = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
                        last_arriver = before == (unsigned)(n - 1);
                        if (last_arriver) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
                    }
                    __syncthreads();
                    const bool last = last_arriver != 0;
                    __syncthreads();
                    return last;
                };
                // n <= GROUP pieces, `step` workgroups apart from w on, AT_ONCE of them requested at a time
                auto fold = [&](int w, int step, int n) {
                    constexpr int AT_ONCE = 8;
#pragma unroll
                    for (int x = 0; x < RT; ++x) {
                        m[x] = -INFINITY;
                        l[x] = 0.f;
#pragma unroll
                        for (int y = 0; y < CPT; ++y) sum[x][y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                        if (16 * x + row >= rows) continue;
#pragma nounroll
                        for (int k0 = 0; k0 < n; k0 += AT_ONCE) {
                            f32x4_t v[AT_ONCE][CPT];
                            u32x2_v s[AT_ONCE];
#pragma unroll
                            for (int k = 0; k < AT_ONCE; ++k) {
                                if (k0 + k >= n) continue;             // the same for all: no load without a use
                                const unsigned p = (unsigned)index(w + (k0 + k) * step) * SLOT;
                                s[k] = __builtin_amdgcn_raw_buffer_load_b64(rp, (16 * x + row) * 8, p + ROWS * D * 4, COHERENT);
#pragma unroll
                                for (int y = 0; y < CPT; ++y)
                                    v[k][y] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rp, (16 * x + row) * D * 4 + (col * CPT + y) * 16, p, COHERENT));
                            }
                            float top = m[x];
#pragma unroll
                            for (int k = 0; k < AT_ONCE; ++k)
                                if (k0 + k < n) top = fmaxf(top, __uint_as_float(s[k][0]));
                            const float fa = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - top);
                            m[x] = top;
                            l[x] *= fa;
#pragma unroll
                            for (int y = 0; y < CPT; ++y) sum[x][y] *= fa;
#pragma unroll
                            for (int k = 0; k < AT_ONCE; ++k)
                                if (k0 + k < n) {
                                    const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(__uint_as_float(s[k][0]) - top);
                                    l[x] += __uint_as_float(s[k][1]) * f;
#pragma unroll
                                    for (int y = 0; y < CPT; ++y) sum[x][y] += v[k][y] * f;
                                }
                        }
                    }
                };
                unsigned *const cnt = a.cnt + (size_t)kvh * gridDim.y * 3;     // two of pieces and one of groups a workgroup
                const int n = w1 - w0 + 1, bits = n <= GROUP || n > GROUP * GROUP / 4 ? 4 : 3, size = 1 << bits;
                const int group = (wg - w0) >> bits, head = w0 + (group << bits), groups = (n + size - 1) >> bits, members = min(size, n - (group << bits));
                park(wg);
                writes = last_of(cnt + index(head), members);
                if (writes) {
                    fold(head, 1, members);
                    if (groups > 1) {
                        park(head);                      // in the place of the group's first piece, which is read
                        writes = last_of(cnt + 2 * gridDim.y + w0, groups);
                        if (writes) fold(w0, size, groups);
                    }
                }
            }
            if (writes) {
#pragma unroll
                for (int x = 0; x < RT; ++x)
                    if (16 * x + row < rows) {
                        const int rr = first_pair + 16 * x + row, tok = by_g(rr);
                        const float inv = l[x] == 0.f ? 0.f : 1.0f / l[x];
                        T *op = (T *)a.out + ((size_t)(rq.first + tok) * a.nq + kvh * G + (rr - tok * G)) * D + col * CPT * 4;
#pragma unroll
                        for (int y = 0; y < CPT; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e) op[4 * y + e] = iso_from_f32<T>(sum[x][y][e] * inv);
                    }
            }
            __syncthreads();                         // the LDS is read; the next tile writes it
        }
        // ---- on along the line
        at = uniform(stop);
        if (at >= end) break;
        inside = uniform(inside + (stop - (s0 + (inside - begin))));
        if (tile + 1 == rq.tiles) {                  // stop was the end of this tile
            inside = 0;
            do {
                seq = uniform(seq + 1);
                rq = request(seq);
            } while (rq.tiles == 0);
        }
    }
}

int line_wgs(int per_cu, int nkv, int ncu) { return max(1, per_cu * min(ncu, 512) / nkv); }      // for a key head
// A workspace is one of counters, the same for every variant (they are zero between calls), and one of pieces.
size_t counters(int nkv, int ncu) { return ((size_t)line_wgs(4, nkv, ncu) * nkv * 3 * 4 + 255) & ~(size_t)255; }

template <typename T, int D, int RT> hipError_t launch(line_args a, void *ws, hipStream_t s) {
    const int wgs = line_wgs(wg_per_cu(sizeof(T), D, RT), a.nkv, iso_num_cu());
    a.cnt = (unsigned *)ws;
    a.part = (float *)((char *)ws + counters(a.nkv, iso_num_cu()));
    // The key heads run fastest: shares of the same number are alike in all heads, and where they are fewer than the workgroups, the ones
    // that have some are the first.  (Shares fastest: one compute unit got the same shares of several heads; 32 heads of 64 over 8, 2 rows
    // over 1616 keys 11.3 us, now 8.0, 7 x 4 rows over up to 2000 12.8 and 10.0.)
    hipLaunchKernelGGL((attn_kv4_kernel<T, D, RT>), dim3(a.nkv, wgs), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

size_t iso_attn_kv4_ws_bytes(int dtype, int nkv, int d, int ncu) {
    size_t most = 0;
    const int elt = dtype == ISO_F32 ? 4 : 2;
    for (int rt = 1; rt <= (elt == 4 ? 1 : 2); ++rt) {
        const int wgs = line_wgs(wg_per_cu(elt, d, rt), nkv, ncu) * nkv;
        most = std::max(most, counters(nkv, ncu) + (size_t)2 * wgs * slot_floats(d, rt) * 4);
    }
    return most;
}

hipError_t iso_launch_attn_kv4(int dtype, const void *q, int q_stride, const iso_kv4 &cache, const kv4_batch &b, int max_rows, int most, void *out,
                               int nq, int nkv, int d, void *ws, hipStream_t s) {
    const unsigned G = (unsigned)(nq / nkv), bits = G == 1 ? 0 : 32 - __builtin_clz(G - 1);        // 2^bits >= G
    const unsigned mul = (unsigned)(((((u64)1 << bits) - G) << 32) / G) + 1;
    const line_args a{q, out, nullptr, nullptr, kv4_view_of(cache), b, q_stride, nq, nkv, (int)G, mul, bits, most};
    // Two blocks of rows a tile where a request can have more than one, and, with heads of 128 (two workgroups on a compute unit then instead
    // of three, pieces twice as large), where a workgroup's share is about 900 keys or more by the room that the table has (not by the keys that
    // are there, which the host does not know: 8 x 5 rows of up to 4000 keys, 16 heads over 2, 15 us through a table of that width, 19 through
    // one of 131072).  16 and 32 rows a tile, 16 heads over 2: 5 rows for each of 8 requests of up to 4000 keys 14 and 22 us; 509 rows of
    // 700 / 2048 / 6000 17 / 30 / 62 and 19 / 28 / 54.  Heads of 64, 32 over 8: 256 rows of 512 / 2048 / 8192 15 / 25 / 58 and 17 / 24 / 52, 2048 of 2048 72 and
    // 62; 16 over 16: 256 of 512 / 32768 12 / 96 and 13 / 86.
    const long long keys = (long long)b.max_pages * cache.page, pairs = (long long)b.total_rows * nq;
    const bool two = std::min((long long)max_rows * a.G, (long long)most) > 16 && (d == 64 || pairs / 32 * keys >= 900ll * wg_per_cu(2, 128, 2) * iso_num_cu());
    if (dtype == ISO_F32) return d == 64 ? launch<float, 64, 1>(a, ws, s) : launch<float, 128, 1>(a, ws, s);
    if (d == 64) return two ? launch<bf16_t, 64, 2>(a, ws, s) : launch<bf16_t, 64, 1>(a, ws, s);
    return two ? launch<bf16_t, 128, 2>(a, ws, s) : launch<bf16_t, 128, 1>(a, ws, s);
}
