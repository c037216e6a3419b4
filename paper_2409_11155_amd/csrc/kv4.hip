// Around the paged 4-bit key/value cache: block tables and slots from request lengths, and the writes into pages and reads back.
#include "kv4.h"

namespace {

// ---- block tables ------------------------------------------------------------------------------
// start_i = sum of the fresh tokens before request i, base_i = sum of the pages taken before it (both exclusive prefix sums);
// the rest is a lookup per row and per new page.  Latency is all there is to it (a full batch of prompts writes half a megabyte),
// so it is one launch: every workgroup computes the prefix sums for itself, which costs less than a second launch would.  256 single
// tokens 4.7 us, 100 000 rows of prompts 5.4: three trips to memory (lengths, table, rows) and the scan in between.
constexpr int BT_THREADS = 256;

struct bt_args {
    const int *cached, *fresh, *free_pages, *free_head;
    int *table, *row_start, *kv_len, *positions, *slots, *free_next;
    int n_seqs, page_shift, n_free, max_pages, max_rows;
};

// Pages that n tokens take, as far as the table's width goes.
__device__ __forceinline__ int bt_pages(int n, int shift, int most) {
    return min(most, (int)(((long long)max(0, n) + (1 << shift) - 1) >> shift));
}

// Largest i with prefix[i] <= x among 0 .. n-1 (prefix[0] = 0 <= x); of equal entries the last, so requests without any are passed over.
__device__ __forceinline__ int bt_find(const int *prefix, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(BT_THREADS) void block_tables_kernel(bt_args a) {
    __shared__ int start[KV4_MAX_SEQS + 1], base[KV4_MAX_SEQS + 1];
    __shared__ int wave_sum[2][BT_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.n_seqs + BT_THREADS - 1) / BT_THREADS;
    const int lo = min(a.n_seqs, tid * per), hi = min(a.n_seqs, lo + per);
    int rows = 0, pages = 0;
    for (int i = lo; i < hi; ++i) {
        const int c = max(0, a.cached[i]), f = max(0, a.fresh[i]);
        start[i] = rows;
        base[i] = pages;
        rows += f;
        pages += bt_pages(c + f, a.page_shift, a.max_pages) - bt_pages(c, a.page_shift, a.max_pages);
    }
    int r_in = rows, p_in = pages;                     // inclusive over the wave, then the waves before
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int r = __shfl_up(r_in, o, 64), p = __shfl_up(p_in, o, 64);
        if (lane >= o) r_in += r, p_in += p;
    }
    if (lane == 63) wave_sum[0][wave] = r_in, wave_sum[1][wave] = p_in;
    __syncthreads();
    int r_off = r_in - rows, p_off = p_in - pages, r_all = 0, p_all = 0;
#pragma unroll
    for (int w = 0; w < BT_THREADS / 64; ++w) {
        if (w < wave) r_off += wave_sum[0][w], p_off += wave_sum[1][w];
        r_all += wave_sum[0][w];
        p_all += wave_sum[1][w];
    }
    for (int i = lo; i < hi; ++i) {
        start[i] += r_off;
        base[i] += p_off;
        if (blockIdx.x == 0) {
            a.row_start[i] = start[i];
            a.kv_len[i] = max(0, a.cached[i]) + max(0, a.fresh[i]);
        }
    }
    const int head = a.free_head ? *a.free_head : 0;
    if (blockIdx.x == 0 && tid == 0) {
        a.row_start[a.n_seqs] = r_all;
        *a.free_next = head + p_all;
    }
    __syncthreads();
    auto free_page = [&](int k) {                      // k-th page that this call takes
        const long long at = (long long)head + k;
        return at >= 0 && at < a.n_free ? a.free_pages[at] : -1;
    };
    const unsigned first = blockIdx.x * BT_THREADS + tid, stride = gridDim.x * BT_THREADS;
    for (unsigned k = first; k < (unsigned)max(0, p_all); k += stride) {
        const int i = bt_find(base, a.n_seqs, (int)k);
        const int col = bt_pages(a.cached[i], a.page_shift, a.max_pages) + (int)k - base[i];
        if ((unsigned)col < (unsigned)a.max_pages) a.table[(size_t)i * a.max_pages + col] = free_page((int)k);
    }
    for (unsigned x = first; x < (unsigned)a.max_rows; x += stride) {
        const int r = (int)x;
        int pos = -1, slot = -1;
        if (r < r_all) {
            const int i = bt_find(start, a.n_seqs, r);
            const int c = max(0, a.cached[i]);
            pos = c + r - start[i];
            const int col = pos >> a.page_shift, have = bt_pages(c, a.page_shift, a.max_pages);
            if ((unsigned)col < (unsigned)a.max_pages) {       // (unsigned: lengths that add up to 2^31 or more stay in bounds too)
                const int pg = col < have ? a.table[(size_t)i * a.max_pages + col] : free_page(base[i] + col - have);
                if ((unsigned)pg < 0x80000000u >> a.page_shift) slot = (pg << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
            }
        }
        a.positions[r] = pos;
        a.slots[r] = slot;
    }
}

// ---- rows into pages, and back -----------------------------------------------------------------
// Eight elements a lane and half a head: a lane has elements 8 l .. 8 l + 7 of the low half and of the high half of one head (the
// two that a rotary step joins), four neighbouring lanes have a block of each.  Bound by memory: 16 bytes (bf16) a load, four bytes
// of codes a store.  bf16, 13 heads of 128: 16384 rows stored in 30 us (4.6 TB/s), loaded in 27; 2047 rows rotated and written
// in 9.8 (3.3 TB/s), loaded in 5.8 (2.9).  64 rows 4.0 and 2.5: launch and two dependent trips to memory.  A rotated head reads its position's
// cosines and sines again, 512 bytes for 256 of its own (26 times a row with 13 heads; from the caches, but through the same pipe).  fp32:
// 2047 rows rotated and written in 11.5, 16384 in 96 (4.9 TB/s), stored in 40, loaded in 44.
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&x)[8]) {
    const f32x4_t a = reinterpret_cast<const f32x4_t *>(p)[0], b = reinterpret_cast<const f32x4_t *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t *p, float (&x)[8]) {
    const bf16x8_t a = *reinterpret_cast<const bf16x8_t *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    reinterpret_cast<f32x4_t *>(p)[0] = f32x4_t{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4_t *>(p)[1] = f32x4_t{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8]) {
    bf16x8_t a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (bf16_t)x[i];
    *reinterpret_cast<bf16x8_t *>(p) = a;
}

// Rounds to fp32 so that no comparison with a number of fewer bits comes out otherwise than for x itself: toward zero, and the
// last bit set if something was cut off.  (Nearest would take a value just beside the border of two codes onto it.)
__device__ __forceinline__ float round_to_odd(double x) {
    const float f = (float)x;
    if (!(fabsf(f) < INFINITY)) return isfinite(x) ? copysignf(3.4e38f, f) : f;      // beyond it every code saturates alike
    const double cut = x - (double)f;                  // exact
    const unsigned away = (unsigned)(__double2hiint(cut) ^ __double2hiint(x)) >> 31;  // rounded away from zero
    return cut == 0.0 ? f : __uint_as_float((__float_as_uint(f) - away) | 1u);
}

// Codes and scale of the block that four neighbouring lanes hold: e = least integer with max|x| <= 7 * 2^e.  (7 and not 6: what lies
// above 6 * 2^e is then off by at most 2^e, no more than between 4 and 6.)  The least e is -125, for every value to be a normal bf16
// number, the largest 125, for none to be infinite; there smaller elements go to zero and larger ones to 6 * 2^125.  Ties go to the even code, what is above 6 * 2^e to 6: as the instruction does.
__device__ __forceinline__ unsigned encode8(const float (&x)[8], unsigned *scale) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
    top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1
    if (top >= 0x7f800000u) {                          // an infinity or a NaN: the block stands for NaN
        *scale = 255;
        return 0;
    }
    const int s = min(252, max(2, (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0)));
    *scale = (unsigned)s;
    const float f = kv4_scale((unsigned)s);
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], f, 3);
    return w;
}

// Bytes of token `slot` of kv head g, in the codes (D / 2 a token) and the scales (D / 32).
template <int D> __device__ __forceinline__ size_t token_at(const kv4_view &c, int nkv, int slot, int g) {
    return (((size_t)(slot >> c.page_shift) * nkv + g) << c.page_shift) + (slot & (c.page - 1));
}

// Both halves of a head that its lanes hold, to token `tok`: four bytes of codes a lane and half; the scales of all blocks go to the
// first lane, which stores them at once.
template <int D>
__device__ __forceinline__ void put(unsigned char *codes, unsigned char *scales, size_t tok, const float (&lo)[8], const float (&hi)[8], int l) {
    unsigned s_lo, s_hi;
    unsigned *const w = reinterpret_cast<unsigned *>(codes + tok * (D / 2));
    const unsigned c_lo = encode8(lo, &s_lo), c_hi = encode8(hi, &s_hi);
    w[l] = c_lo;
    w[D / 16 + l] = c_hi;
    if constexpr (D == 128) {                          // lanes 0 and 4: blocks 0 | 2 and 1 | 3
        const unsigned mine = s_lo | s_hi << 16;
        const unsigned next = (unsigned)__builtin_amdgcn_mov_dpp((int)mine, 0x104, 0xF, 0xF, true);      // from four lanes up
        if (l == 0) reinterpret_cast<unsigned *>(scales)[tok] = mine | next << 8;
    } else {
        if (l == 0) reinterpret_cast<unsigned short *>(scales)[tok] = (unsigned short)(s_lo | s_hi << 8);
    }
}

// ROPE: rows of the QKV projection, heads [q | k | v]; q is rotated into q_out (or in place), k rotated, both written at `slots`.
// Otherwise: separate k and v rows as a prefill's cache holds them.
// The key's rotation is computed in 64 bits from the fp32 table: its codes are then those of the exact product sum, whatever lies
// next to the border of two codes.  (q: as everywhere else in 32 bits.)
template <typename T, int D, bool ROPE>
__global__ __launch_bounds__(256) void kv4_write_kernel(T *qkv, T *q_out, const T *__restrict__ k_rows, const T *__restrict__ v_rows,
                                                        kv4_view c, const int *__restrict__ positions, const int *__restrict__ slots,
                                                        const float *__restrict__ cos_t, const float *__restrict__ sin_t, int max_pos,
                                                        int n_rows, int nq, int nkv) {
    constexpr int LPH = D / 16;                        // lanes per head
    const unsigned heads = ROPE ? nq + 2 * nkv : 2 * nkv;
    const unsigned th = blockIdx.x * (256u / LPH) + threadIdx.x / LPH;         // (row, head); fewer than 2^31 of them
    const int l = threadIdx.x % LPH;
    if (th >= (unsigned)n_rows * heads) return;        // a head's lanes leave together
    // All rows' k heads, then all q, then all v: a wave does one of them (key heads are rotated in 64 bits, and with heads in a row's order
    // nearly every wave had one: 2047 rows of 13 heads each 12.6 us, now 9.8; 2048 of 16 heads over 2 7.7 and 6.0).
    const unsigned k_all = (unsigned)n_rows * nkv, q_end = k_all + (ROPE ? (unsigned)n_rows * nq : 0);
    const bool is_k = th < k_all, is_q = ROPE && !is_k && th < q_end, is_v = !is_k && !is_q;
    const unsigned r = th - (is_k ? 0 : is_q ? k_all : q_end), per = is_q ? nq : nkv;
    const int t = (int)(r / per), g = (int)(r - (unsigned)t * per);
    const T *src = ROPE ? qkv + ((size_t)t * heads + (is_q ? 0 : is_v ? nq + nkv : nq) + g) * D : (is_v ? v_rows : k_rows) + (size_t)r * D;
    float lo[8], hi[8];
    load8<T>(src + 8 * l, lo);                         // on their way before it is known where they go
    load8<T>(src + D / 2 + 8 * l, hi);
    const int slot = slots[t];
    const bool kept = slot >= 0 && (slot >> c.page_shift) < c.n_pages;
    const int pos = ROPE ? positions[t] : 0;
    if (pos < 0 || pos >= max_pos) return;             // no row
    if (!is_q && !kept) return;
    if (ROPE && !is_v) {
        float cs[8], sn[8];
        load8<float>(cos_t + (size_t)pos * (D / 2) + 8 * l, cs);
        load8<float>(sin_t + (size_t)pos * (D / 2) + 8 * l, sn);
        if (is_q) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = lo[i], b = hi[i];
                lo[i] = fmaf(a, cs[i], -(b * sn[i]));
                hi[i] = fmaf(b, cs[i], a * sn[i]);
            }
            T *dst = q_out ? q_out + (size_t)r * D : const_cast<T *>(src);
            store8(dst + 8 * l, lo);
            store8(dst + D / 2 + 8 * l, hi);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double a = lo[i], b = hi[i];
            lo[i] = round_to_odd(a * (double)cs[i] - b * (double)sn[i]);
            hi[i] = round_to_odd(b * (double)cs[i] + a * (double)sn[i]);
        }
    }
    const size_t tok = token_at<D>(c, nkv, slot, g);
    put<D>(is_v ? c.v : c.k, is_v ? c.vs : c.ks, tok, lo, hi, l);
}

// The values that the slots hold, as rows: eight elements a lane.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_load_kernel(kv4_view c, const int *__restrict__ slots, T *__restrict__ k_rows,
                                                       T *__restrict__ v_rows, int n_rows, int nkv) {
    constexpr int LPH = D / 8;
    const unsigned th = blockIdx.x * (256u / LPH) + threadIdx.x / LPH;         // (row, head); fewer than 2^31 of them
    const int l = threadIdx.x % LPH;
    if (th >= (unsigned)n_rows * 2u * nkv) return;
    const unsigned k_all = (unsigned)n_rows * nkv;             // all rows' k heads, then all v
    const bool is_v = th >= k_all;
    const unsigned r = is_v ? th - k_all : th;
    const int t = (int)(r / (unsigned)nkv), g = (int)(r - (unsigned)t * nkv);
    const int slot = slots[t];
    if (slot < 0 || (slot >> c.page_shift) >= c.n_pages) return;
    const size_t tok = token_at<D>(c, nkv, slot, g);
    const unsigned w = *reinterpret_cast<const unsigned *>((is_v ? c.v : c.k) + tok * (D / 2) + 4 * l);
    const float f = kv4_scale((is_v ? c.vs : c.ks)[tok * (D / KV4_BLOCK) + l / 4]);
    const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1);
    const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3);
    const float x[8] = {(float)p0[0], (float)p0[1], (float)p1[0], (float)p1[1], (float)p2[0], (float)p2[1], (float)p3[0], (float)p3[1]};
    store8((is_v ? v_rows : k_rows) + (size_t)r * D + 8 * l, x);
}

template <typename T, int D>
hipError_t launch_write(bool rope, void *qkv, void *q_out, const void *k_rows, const void *v_rows, const kv4_view &c, const int *positions,
                        const int *slots, const float *cos_t, const float *sin_t, int max_pos, int n_rows, int nq, int nkv, hipStream_t s) {
    const long long lanes = (long long)n_rows * ((rope ? nq : 0) + 2 * nkv) * (D / 16);
    const dim3 grid((unsigned)((lanes + 255) / 256)), block(256);
    if (rope)
        hipLaunchKernelGGL((kv4_write_kernel<T, D, true>), grid, block, 0, s, (T *)qkv, (T *)q_out, nullptr, nullptr, c, positions, slots, cos_t,
                           sin_t, max_pos, n_rows, nq, nkv);
    else
        hipLaunchKernelGGL((kv4_write_kernel<T, D, false>), grid, block, 0, s, nullptr, nullptr, (const T *)k_rows, (const T *)v_rows, c,
                           nullptr, slots, nullptr, nullptr, 1, n_rows, 0, nkv);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_load(const kv4_view &c, const int *slots, void *k_rows, void *v_rows, int n_rows, int nkv, hipStream_t s) {
    const long long lanes = (long long)n_rows * 2 * nkv * (D / 8);
    hipLaunchKernelGGL((kv4_load_kernel<T, D>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, s, c, slots, (T *)k_rows, (T *)v_rows,
                       n_rows, nkv);
    return hipGetLastError();
}

}  // namespace

hipError_t iso_launch_block_tables(const int *cached, const int *fresh, int n_seqs, int page, const int *free_pages, int n_free,
                                   const int *free_head_or_null, int *table, int max_pages, int *row_start, int *kv_len, int *positions,
                                   int *slots, int max_rows, int *free_next, hipStream_t s) {
    const bt_args a{cached, fresh, free_pages, free_head_or_null, table, row_start, kv_len, positions, slots, free_next,
                    n_seqs, __builtin_ctz((unsigned)page), n_free, max_pages, max_rows};
    const int wgs = min(256, (max_rows - 1) / BT_THREADS + 1);
    hipLaunchKernelGGL(block_tables_kernel, dim3(wgs), dim3(BT_THREADS), 0, s, a);
    return hipGetLastError();
}

hipError_t iso_launch_kv4_write(int dtype, void *qkv, void *q_out_or_null, const iso_kv4 &cache, const int *positions, const int *slots,
                                const float *cos_t, const float *sin_t, int max_pos, int n_rows, int nq, int nkv, int d, hipStream_t s) {
    const kv4_view c = kv4_view_of(cache);
    auto go = dtype == ISO_F32 ? (d == 64 ? launch_write<float, 64> : launch_write<float, 128>)
                               : (d == 64 ? launch_write<bf16_t, 64> : launch_write<bf16_t, 128>);
    return go(true, qkv, q_out_or_null, nullptr, nullptr, c, positions, slots, cos_t, sin_t, max_pos, n_rows, nq, nkv, s);
}

hipError_t iso_launch_kv4_store(int dtype, const void *k_rows, const void *v_rows, const iso_kv4 &cache, const int *slots, int n_rows, int nkv,
                                int d, hipStream_t s) {
    const kv4_view c = kv4_view_of(cache);
    auto go = dtype == ISO_F32 ? (d == 64 ? launch_write<float, 64> : launch_write<float, 128>)
                               : (d == 64 ? launch_write<bf16_t, 64> : launch_write<bf16_t, 128>);
    return go(false, nullptr, nullptr, k_rows, v_rows, c, nullptr, slots, nullptr, nullptr, 1, n_rows, 0, nkv, s);
}

hipError_t iso_launch_kv4_load(int dtype, const iso_kv4 &cache, const int *slots, void *k_rows, void *v_rows, int n_rows, int nkv, int d,
                               hipStream_t s) {
    const kv4_view c = kv4_view_of(cache);
    auto go = dtype == ISO_F32 ? (d == 64 ? launch_load<float, 64> : launch_load<float, 128>)
                               : (d == 64 ? launch_load<bf16_t, 64> : launch_load<bf16_t, 128>);
    return go(c, slots, k_rows, v_rows, n_rows, nkv, s);
}
