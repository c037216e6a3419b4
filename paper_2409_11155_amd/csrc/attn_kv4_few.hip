// Attention over the paged 4-bit cache for few rows: a row tile is 16 rows (token, query head of the key head), which a decoding
// step's tokens fill or less.  Bound by the cache's bytes.
//
// Same mathematics as the other attention kernels: S^T = K Q^T, so that the softmax statistics are per-lane scalars and the
// probabilities feed O^T = V^T P^T from registers; v_mfma_f32_16x16x32_bf16.  A value of the cache is a bf16 number, so unpacking is
// exact: v_cvt_scalef32_pk_bf16_fp4 makes two elements an instruction, scale included.
//   * K goes from the page into the registers that the product wants: the four lanes of a key take a quarter of its head each, 16 (8)
//     bytes, and element order inside the head is free as long as q is read in the same one.  No LDS.
//   * V has to be transposed: a wave writes its 32 unpacked rows to LDS (its own 8 KB, no barrier) and reads them back with
//     ds_read_b64_tr_b16.  16-byte chunks are XOR-swizzled by the row so that neither side has bank conflicts.
//   * T = float: q and the probabilities are cut into three bf16 terms that add up to all 24 bits (K and V have two): three products.
//
// Work: the (kv head, request, row tile) triples have ceil(keys / 128) units of 128 keys each; all units lie on one line which is cut
// into equal shares, a workgroup each, whatever the requests' lengths are.  A workgroup's four waves take 32 keys of a unit each and
// meet in LDS at the end of a triple.  A triple that crosses workgroups is parked in pieces (running maximum, sum, unnormalised output)
// with cache-bypassing stores; the workgroup that arrives last folds them in the order of the line, so the result does not depend on who
// that is, and puts the counter back to zero.  Nobody waits for anybody.  The shares are computed on the device from the lengths there:
// a captured step keeps its balance as the requests grow.
#include "kv4.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, TILE = 32, UNIT = WAVES * TILE, ROWS = 16;
constexpr int FOLD = 128, SPLITS = FOLD - 2;              // pieces of a triple, at most (two less than the fold takes: a share may start and end inside one)
constexpr int COHERENT = 1 | 16;         // buffer cache policy sc0 | sc1: system scope, bypasses the XCD-local L2

typedef __bf16 bf16x4_v __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_v __attribute__((ext_vector_type(2)));

// Workgroups on a compute unit, by the registers: float keeps three terms of q.
constexpr int wg_per_cu(int elt, int d) { return elt == 4 ? (d == 64 ? 3 : 2) : d == 64 ? 4 : 3; }
template <int D> constexpr int slot_floats() { return ROWS * (D + 2); }      // output rows, then maxima, then sums

struct few_args {
    const void *q;
    void *out;
    float *part;
    unsigned *cnt;
    kv4_view c;
    kv4_batch b;
    int q_stride, nq, nkv, G, wgs;       // G: query heads of a key head
    int most;                            // requests of more (row, head) pairs than this belong to another launch
    int unit_shift;                      // log2 of a unit's keys: UNIT, or a multiple that keeps the line's length in 32 bits
};

__device__ __forceinline__ bf16x4_v read_tr(unsigned addr) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4_v *)(uintptr_t)addr);
}

// x as a sum of NP bf16 terms: rounded to nearest (NP = 1), or cut off so that three terms are all of x.
template <int NP> __device__ __forceinline__ void split(float x, bf16_t (&t)[NP]) {
    if constexpr (NP == 1) {
        t[0] = (bf16_t)x;
    } else {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float cut = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
            t[p] = (bf16_t)cut;
            x -= cut;
        }
    }
}

__device__ __forceinline__ bf16x8_t unpack8(unsigned w, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Wave-uniform values are made scalar explicitly, and what is read at a uniform place is read by the scalar unit: vector loads come
// back in order, so a page number among them would have to wait for the codes requested before it.
typedef const __attribute__((address_space(4))) int *scalar_ints;
// Buffer over the 4 GB from p + (at & ~0xffffffff) on: with the low half of `at` as the scalar offset, a lane's address is p + at + its own
// offset without an addition in a vector register.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t beyond(unsigned char *p, uint64_t at) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)(p + (at & 0xffffffff00000000ull)), 0, -1, 0x00020000);
}
__device__ __forceinline__ scalar_ints scalar(const int *p) { return (scalar_ints)(uintptr_t)p; }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ unsigned uniform(unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); }

// Inclusive sum and maximum over the wave, lane 63 holds all of it: row shifts, then the last lanes of the rows handed on (DPP, no LDS).
template <typename F> __device__ __forceinline__ unsigned wave_scan(unsigned x, F f) {
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
    return x;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS, wg_per_cu(sizeof(T), D)) void attn_kv4_few_kernel(few_args a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;
    constexpr int WPL = D / 32;              // code words (8 elements) a lane takes of a key
    constexpr int RB = 2 * D;                // bytes of an unpacked row
    constexpr int VG = D == 64 ? 2 : 1;      // blocks of 16 dims of V that are read at a time
    __shared__ __attribute__((aligned(1024))) unsigned char lds[WAVES * TILE * RB];
    __shared__ float ml[2][WAVES][ROWS];
    __shared__ int last_arriver;

    const int tid = threadIdx.x, lane = tid & 63, n16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const kv4_batch &b = a.b;
    const int shift = a.c.page_shift, G = a.G, unit = 1 << a.unit_shift;

    // ---- units in front of every request, and in all
    struct Req { int first, n, base, keys; unsigned tiles, units; };
    auto request = [&](int i) {
        const kv4_rows r = kv4_rows_of(scalar(b.row_start), scalar(b.kv_len), b.total_rows, i);
        Req q{r.first, r.n, r.base, kv4_keys_of(scalar(b.kv_len), b.max_pages, i, shift), 0, 1};
        const unsigned pairs = (unsigned)(r.n * G);
        q.tiles = pairs > (unsigned)a.most ? 0 : (pairs + ROWS - 1) / ROWS;
        q.units = max(1u, ((unsigned)q.keys + unit - 1) >> a.unit_shift);
        return q;
    };
    // Every wave does this for itself, 64 requests at a time: no barrier, and for up to 64 of them one trip to memory.
    auto add = [](unsigned x, unsigned y) { return x + y; };
    unsigned mine = 0, longest = 0;
    for (int i0 = 0; i0 < b.n_seqs; i0 += 64) {
        const Req q = request(min(i0 + lane, b.n_seqs - 1));
        const unsigned u = i0 + lane < b.n_seqs ? q.tiles * q.units : 0;
        mine += u;
        if (u) longest = max(longest, q.units);
    }
    unsigned incl = wave_scan(mine, add);
    const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)incl, 63);
    longest = (unsigned)__builtin_amdgcn_readlane((int)wave_scan(longest, [](unsigned x, unsigned y) { return max(x, y); }), 63);
    if (all == 0) return;
    const unsigned total = all * (unsigned)a.nkv;
    const unsigned per = uniform(max((total + a.wgs - 1) / a.wgs, (longest + SPLITS - 1) / SPLITS));
    unsigned at = blockIdx.x * per;
    const unsigned end = min(total, at + per);
    if (at >= end) return;
    // ---- the request that holds the first unit
    int kvh = (int)uniform(at / all), seq = 0;
    unsigned inside = at - (unsigned)kvh * all;
    for (int i0 = 0;; i0 += 64) {
        if (b.n_seqs > 64) {
            const Req q = request(min(i0 + lane, b.n_seqs - 1));
            mine = i0 + lane < b.n_seqs ? q.tiles * q.units : 0;
            incl = wave_scan(mine, add);
        }
        const uint64_t in_front = __builtin_amdgcn_ballot_w64(incl <= inside);      // requests that end before it
        const int n = __builtin_popcountll(in_front);
        if (n < 64) {
            seq = i0 + n;
            inside -= n ? (unsigned)__builtin_amdgcn_readlane((int)incl, n - 1) : 0u;
            break;
        }
        inside -= (unsigned)__builtin_amdgcn_readlane((int)incl, 63);
    }

    const float sc = 1.4426950408889634f / sqrtf((float)D);
    const unsigned lds_w = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * TILE * RB;
    auto swz = [](int row) { return D == 128 ? ((row & 7) << 1 | (row >> 3 & 1)) : ((row >> 1 & 3) << 1 | (row >> 3 & 1)); };
    // V: the lane's row on the way in is n16 (+ 16), on the way out 4 g4 + n16 / 4 (+ 16)
    unsigned char *const v_in = lds + wave * TILE * RB + n16 * RB;
    const int in_swz = swz(n16);
    const unsigned code_at = n16 * (D / 2) + g4 * WPL * 4, scale_at = n16 * (D / KV4_BLOCK) + g4 * WPL / 4;
    const int out_row = 4 * g4 + (n16 >> 2);
    const unsigned v_out = lds_w + out_row * RB + ((((n16 & 3) >> 1) ^ swz(out_row)) << 4) + ((n16 & 1) << 3);

    for (;;) {
        const Req rq = request(seq);
        const unsigned tile = uniform(inside / rq.units), ua = inside - tile * rq.units;
        const unsigned ub = min(rq.units, ua + (end - at));
        const int pairs = rq.n * G;
        // ---- this tile's rows
        const int r = (int)tile * ROWS + n16, t = r / G, head = kvh * G + (r - t * G);
        const bool real = r < pairs;
        auto limit = [&](int tok) { return max(0, min(rq.keys, rq.base + tok + 1)); };      // keys that a token sees
        const int lim_lo = uniform(limit((int)tile * ROWS / G)), lim_hi = uniform(limit((min(pairs, (int)tile * ROWS + ROWS) - 1) / G));
        const int lim = real ? limit(t) : lim_lo;
        bf16x8_t qf[NP][WPL];
        {
            const T *qp = (const T *)a.q + (size_t)(rq.first + (real ? t : 0)) * a.q_stride + (size_t)(real ? head : 0) * D + g4 * WPL * 8;
            typedef T row8 __attribute__((ext_vector_type(8)));
#pragma unroll
            for (int w = 0; w < WPL; ++w) {
                const row8 x = *reinterpret_cast<const row8 *>(qp + w * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t part[NP];
                    split<NP>(real ? iso_to_f32((T)x[e]) : 0.f, part);
#pragma unroll
                    for (int p = 0; p < NP; ++p) qf[p][w][e] = part[p];
                }
            }
        }
        f32x4_t o[D / 16];
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        float m_run = -INFINITY, l_run = 0.f;          // maximum in units of the base-2 exponent

        const scalar_ints table = scalar(b.table + (size_t)seq * b.max_pages);
        int k0 = (int)min((long long)ua << a.unit_shift, (long long)lim_hi) + wave * TILE;
        const int k_end = (int)min((long long)ub << a.unit_shift, (long long)lim_hi);
        struct Pages { int p[2]; };
        auto pages_of = [&](int k0) {
            Pages x;
#pragma unroll
            for (int h = 0; h < 2; ++h) x.p[h] = k0 + 16 * h < k_end ? table[(k0 + 16 * h) >> shift] : -1;
            return x;
        };
        struct Codes { unsigned k[2][WPL], v[2][WPL]; unsigned ks[2], vs[2]; int there; };
        // Codes and scales of the wave's 32 keys from k0 on.  Where there is no page the first one is read instead, and what lies behind the
        // last visible key is read too: multiply() leaves both out.
        auto fetch = [&](int k0, const Pages &pages, Codes &c) {
            c.there = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool there = (unsigned)pages.p[h] < (unsigned)a.c.n_pages;
                c.there |= (int)there << h;
                const uint64_t tok = (((uint64_t)(unsigned)(there ? pages.p[h] : 0) * (unsigned)a.nkv + (unsigned)kvh) << shift) + ((k0 + 16 * h) & (a.c.page - 1));
                const uint64_t at_c = tok * (D / 2), at_s = tok * (D / KV4_BLOCK);
                const auto rk = beyond(a.c.k, at_c), rv = beyond(a.c.v, at_c), rks = beyond(a.c.ks, at_s), rvs = beyond(a.c.vs, at_s);
                if constexpr (D == 128) {
                    const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(rk, code_at, (unsigned)at_c, 0);
                    const u32x4_t y = __builtin_amdgcn_raw_buffer_load_b128(rv, code_at, (unsigned)at_c, 0);
#pragma unroll
                    for (int w = 0; w < WPL; ++w) c.k[h][w] = x[w], c.v[h][w] = y[w];
                } else {
                    const u32x2_v x = __builtin_amdgcn_raw_buffer_load_b64(rk, code_at, (unsigned)at_c, 0);
                    const u32x2_v y = __builtin_amdgcn_raw_buffer_load_b64(rv, code_at, (unsigned)at_c, 0);
#pragma unroll
                    for (int w = 0; w < WPL; ++w) c.k[h][w] = x[w], c.v[h][w] = y[w];
                }
                c.ks[h] = __builtin_amdgcn_raw_buffer_load_b8(rks, scale_at, (unsigned)at_s, 0);
                c.vs[h] = __builtin_amdgcn_raw_buffer_load_b8(rvs, scale_at, (unsigned)at_s, 0);
            }
        };
        auto multiply = [&](int k0, Codes &c) {
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
            f32x4_t s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                const float f = kv4_scale(c.ks[h]);
#pragma unroll
                for (int w = 0; w < WPL; ++w) {
                    const bf16x8_t kf = unpack8(c.k[h][w], f);
#pragma unroll
                    for (int p = 0; p < NP; ++p) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][w], s[h], 0, 0, 0);
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
                    const unsigned at = v_out ^ (unsigned)((dt0 + i) << 5);
                    vf[buf][i] = __builtin_shufflevector(read_tr(at), read_tr(at + 16 * RB), 0, 1, 2, 3, 4, 5, 6, 7);
                }
            };
            read_v(0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (masked) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (k0 + 16 * h + 4 * g4 + e >= lim || !(c.there >> h & 1)) s[h][e] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[h][e]);
            mx *= sc;
            // the running maximum moves rarely deep in a cache; the four lanes of a row agree on it
            if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float m_new = fmaxf(m_run, mx);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) o[dt] *= alpha;
            }
            const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
            bf16x8_t pb[NP];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[h][e], sc, neg_m));
                    l_run += p;
                    bf16_t part[NP];
                    split<NP>(p, part);
#pragma unroll
                    for (int x = 0; x < NP; ++x) pb[x][4 * h + e] = part[x];
                }
#pragma unroll
            for (int grp = 0; grp < D / 16 / VG; ++grp) {
                if (grp + 1 < D / 16 / VG) read_v((grp + 1) & 1, VG * (grp + 1));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < VG; ++i)
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        o[VG * grp + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[grp & 1][i], pb[p], o[VG * grp + i], 0, 0, 0);
            }
            // a token whose V is NaN in some block: so is that block of the rows that see it, and of no others
            if ((nan_v[0] | nan_v[1]) != 0) {
                unsigned blocks = 0;                       // bit = 16 dims
                for (int h = 0; h < 2; ++h)
                    for (uint64_t m = h ? nan_v[1] : nan_v[0]; m; m &= m - 1) {
                        const int bit = __builtin_ctzll(m);
                        if (k0 + 16 * h + (bit & 15) < lim) blocks |= ((1u << D / 64) - 1) << (bit >> 4) * (D / 64);
                    }
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt)
                    if (blocks >> dt & 1) o[dt] = f32x4_t{NAN, NAN, NAN, NAN};
            }
        };

        {
            // Codes are requested a tile ahead and page numbers two, without a branch: behind the share's end there are no pages,
            // and what has none is not fetched.  (A branch around the requests would make every wait one for all of them.)
            Codes c0, c1;
            fetch(k0, pages_of(k0), c0);
            Pages pages = pages_of(k0 + UNIT);
            auto step = [&](Codes &now, Codes &later) {
                fetch(k0 + UNIT, pages, later);
                pages = pages_of(k0 + 2 * UNIT);
                multiply(k0, now);
                k0 += UNIT;
            };
            while (k0 < k_end) {
                step(c0, c1);
                if (k0 >= k_end) break;
                step(c1, c0);
            }
        }
        // ---- the four waves' states
        l_run += __shfl_xor(l_run, 16, 64);
        l_run += __shfl_xor(l_run, 32, 64);
        {
            float *po = reinterpret_cast<float *>(lds + wave * TILE * RB) + n16 * D;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4_t *>(po + (((4 * dt + g4) ^ n16) << 2)) = o[dt];
            if (g4 == 0) ml[0][wave][n16] = m_run, ml[1][wave][n16] = l_run;
        }
        __syncthreads();
        constexpr int CPT = D / 64;              // float4 of a row that a thread has
        const int row = tid >> 4, col = tid & 15;
        float m = -INFINITY, l = 0.f;
        f32x4_t sum[CPT];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[0][w][row]);
#pragma unroll
        for (int x = 0; x < CPT; ++x) sum[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[0][w][row] - m);      // no score but NaN: zeros and NaN add up
            l += ml[1][w][row] * f;
            const float *po = reinterpret_cast<const float *>(lds + w * TILE * RB) + row * D;
#pragma unroll
            for (int x = 0; x < CPT; ++x) sum[x] += *reinterpret_cast<const f32x4_t *>(po + (((col * CPT + x) ^ row) << 2)) * f;
        }
        const bool real_row = (int)tile * ROWS + row < pairs;
        bool writes = true;
        if (ub - ua < rq.units) {
            // ---- a piece of the triple: park it, and fold all of them if this is the last to arrive
            const unsigned s0 = at - ua;                                        // the triple's first unit on the line
            const int w0 = (int)uniform(s0 / per), w1 = (int)uniform((s0 + rq.units - 1) / per);
            const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc((void *)a.part, 0, 2 * a.wgs * slot_floats<D>() * 4, 0x00020000);
            auto slot = [&](int w) { return (unsigned)(2 * w + (w == w0 ? 1 : 0)) * (slot_floats<D>() * 4); };
            if (real_row) {
                const unsigned p = slot(blockIdx.x);
#pragma unroll
                for (int x = 0; x < CPT; ++x)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, sum[x]), rp, p + (row * D + (col * CPT + x) * 4) * 4, 0, COHERENT);
                if (col == 0) {
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(m), rp, p + (ROWS * D + row) * 4, 0, COHERENT);
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(l), rp, p + (ROWS * D + ROWS + row) * 4, 0, COHERENT);
                }
            }
            __builtin_amdgcn_s_waitcnt(0);       // my stores have reached memory ...
            __syncthreads();                     // ... and so have everybody's, before the arrival is counted
            if (tid == 0) {
                const unsigned n = __hip_atomic_fetch_add(&a.cnt[w0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
                last_arriver = n == (unsigned)(w1 - w0);
                if (last_arriver) __hip_atomic_store(&a.cnt[w0], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
            }
            __syncthreads();
            writes = last_arriver != 0;
            if (writes) {
                // All maxima and sums at once, then the rows with their weights.  Sixteen threads take a row of a piece; where the tile
                // has fewer than 16 rows, the threads left over take every second (fourth, ...) piece.
                const int n = w1 - w0 + 1, frow = tid & 15;
                float mw[FOLD / 16], lw[FOLD / 16], top = -INFINITY, lsum = 0.f;
#pragma unroll
                for (int k = 0; k < FOLD / 16; ++k) {
                    const int w = (tid >> 4) + 16 * k;
                    mw[k] = -INFINITY;
                    lw[k] = 0.f;
                    if (w < n && (int)tile * ROWS + frow < pairs) {
                        mw[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, slot(w0 + w) + (ROWS * D + frow) * 4, 0, COHERENT));
                        lw[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, slot(w0 + w) + (ROWS * D + ROWS + frow) * 4, 0, COHERENT));
                    }
                }
                float *const wt = reinterpret_cast<float *>(lds), *const red = wt + FOLD * ROWS;      // weights [piece][row]; [16][16]
#pragma unroll
                for (int k = 0; k < FOLD / 16; ++k) top = fmaxf(top, mw[k]);
                red[tid] = top;
                __syncthreads();
#pragma unroll
                for (int k = 0; k < 16; ++k) top = fmaxf(top, red[16 * k + frow]);
#pragma unroll
                for (int k = 0; k < FOLD / 16; ++k) {
                    const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw[k] - top);
                    lsum += lw[k] * f;
                    wt[tid + 256 * k] = f;
                }
                __syncthreads();
                red[tid] = lsum;
                __syncthreads();
                const int rows = min(ROWS, pairs - (int)tile * ROWS), rs = rows > 8 ? 4 : rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0;
                const int my_row = (tid >> 4) & ((1 << rs) - 1), part = tid >> (4 + rs), parts = 16 >> rs;
#pragma unroll
                for (int x = 0; x < CPT; ++x) sum[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (my_row < rows) {
#pragma unroll 8
                    for (int w = part; w < n; w += parts) {
                        const float f = wt[w * ROWS + my_row];
#pragma unroll
                        for (int x = 0; x < CPT; ++x)
                            sum[x] += f * __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rp, slot(w0 + w) + (my_row * D + (col * CPT + x) * 4) * 4, 0, COHERENT));
                    }
                }
                l = 0.f;
#pragma unroll
                for (int k = 0; k < 16; ++k) l += red[16 * k + row];
                __syncthreads();
                f32x4_t *const rest = reinterpret_cast<f32x4_t *>(lds);        // [part][row][16 * CPT], over the weights
#pragma unroll
                for (int x = 0; x < CPT; ++x) rest[(tid >> 4) * 16 * CPT + col * CPT + x] = sum[x];
                __syncthreads();
#pragma unroll
                for (int x = 0; x < CPT; ++x) {
                    sum[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    if (real_row)
                        for (int k = 0; k < parts; ++k) sum[x] += rest[((k << rs) + row) * 16 * CPT + col * CPT + x];
                }
            }
        }
        if (writes && real_row) {
            const int rr = (int)tile * ROWS + row, tok = rr / G;
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            T *op = (T *)a.out + ((size_t)(rq.first + tok) * a.nq + kvh * G + (rr - tok * G)) * D + col * CPT * 4;
#pragma unroll
            for (int x = 0; x < CPT; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) op[4 * x + e] = iso_from_f32<T>(sum[x][e] * inv);
        }
        __syncthreads();                         // the LDS is read; the next triple writes it
        // ---- on along the line
        at = uniform(at + (ub - ua));
        if (at >= end) break;
        inside = uniform(inside + (ub - ua));
        if (inside == rq.tiles * rq.units) {
            inside = 0;
            do {
                if (++seq == b.n_seqs) seq = 0, ++kvh;
                seq = uniform(seq);
            } while (request(seq).tiles == 0);
            kvh = uniform(kvh);
        }
    }
}

}  // namespace

// Workgroups of the line, at most: as many as the chip holds at once.
namespace {
int few_wgs(int ncu, int elt, int d) { return wg_per_cu(elt, d) * min(ncu, 512); }
size_t few_bytes(int d, int wgs) { return (size_t)wgs * 4 + (size_t)2 * wgs * (d == 64 ? slot_floats<64>() : slot_floats<128>()) * 4; }
}  // namespace
size_t iso_attn_kv4_few_ws_bytes(int d, int ncu) { return few_bytes(d, few_wgs(ncu, 2, d)) + 256; }

hipError_t iso_launch_attn_kv4_few(int dtype, const void *q, int q_stride, const iso_kv4 &cache, const kv4_batch &b, int most, void *out,
                                   int nq, int nkv, int d, void *ws, hipStream_t s) {
    // a unit grows until the line's length stays below 2^31 whatever the lengths on the device are
    const long long tiles = ((long long)b.total_rows * (nq / nkv) / ROWS + b.n_seqs) * nkv, keys = (long long)b.max_pages * cache.page;
    int shift = __builtin_ctz(UNIT);
    auto units = [&]() { return tiles * ((keys + (1ll << shift) - 1) >> shift); };
    while (units() >= (1ll << 31) && shift < 30) ++shift;
    if (units() >= (1ll << 31)) return hipErrorInvalidValue;
    const int wgs = (int)min((long long)few_wgs(iso_num_cu(), dtype == ISO_F32 ? 4 : 2, d), units());    // no more workgroups than units
    few_args a{q, out, nullptr, (unsigned *)ws, kv4_view_of(cache), b, q_stride, nq, nkv, nq / nkv, wgs, most, shift};
    a.part = (float *)((char *)ws + (((size_t)few_wgs(iso_num_cu(), dtype == ISO_F32 ? 4 : 2, d) * 4 + 255) & ~(size_t)255));
    if (dtype == ISO_F32 && d == 64) hipLaunchKernelGGL((attn_kv4_few_kernel<float, 64>), dim3(wgs), dim3(THREADS), 0, s, a);
    else if (dtype == ISO_F32 && d == 128) hipLaunchKernelGGL((attn_kv4_few_kernel<float, 128>), dim3(wgs), dim3(THREADS), 0, s, a);
    else if (dtype == ISO_BF16 && d == 64) hipLaunchKernelGGL((attn_kv4_few_kernel<bf16_t, 64>), dim3(wgs), dim3(THREADS), 0, s, a);
    else if (dtype == ISO_BF16 && d == 128) hipLaunchKernelGGL((attn_kv4_few_kernel<bf16_t, 128>), dim3(wgs), dim3(THREADS), 0, s, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}
