// The 4-bit key/value cache: 32 neighbouring elements of a head (a block) share a scale 2^(byte - 127); an element is E2M1, a
// sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (the OCP microscaling format with 4-bit elements).  A value has at most two
// significant bits, so unpacking into bf16 rounds nothing.  Byte 255 is NaN for the whole block.
#pragma once
#include "iso_internal.h"

constexpr int KV4_BLOCK = 32;
constexpr int KV4_MAX_SEQS = 4096;      // requests in one call: their prefix sums are kept in LDS
constexpr int KV4_MAX_KEYS = 0x7fffffff - 1023;      // tokens that a request's table has room for: key counters run up to 300 past the last one

// bf16 terms of a probability in the product with V, in tiles of so many (row, head) pairs (bf16 contexts; the probabilities' sum keeps 24
// bits).  Two are the nearest and the nearest of what is left, 16 bits: results are then as far from 64 bits as the rounding of the output
// alone, 1.66e-3 of their size; with one term 2.1e-3.  Heads of 64: two, as in the attention over rows (attn_bf16_dtl.hip).  Heads of 128: there
// it is one; here two where they cost next to nothing, in tiles of 16 pairs, which wait for the cache's bytes.  Times of one and two (us):
//   heads of 64, 32 over 8:  48 x 2 rows over 300 to 8192 keys 20.6 and 21.6,  500 rows of 2500 27 and 31,  2048 of 2048 40 and 47
//   heads of 128, tiles of 16:  40 single tokens, 13 heads over 13, 500 to 8192 keys 44.3 and 44.7,  one of 131072, 8 over 1, 16.6 and 16.9
//     512 rows of 2000, 13 over 13, 26.0 and 27.5;
//   tiles of 32:  2 x 509 rows and 22 tokens, 16 over 2, 700 to 6000 keys 37.5 and 42.4;  of 128:  2048 of 32768, 8 over 1, 267 and 364 (spilled)
constexpr int kv4_terms(int d, int tile) { return d == 64 || tile == 16 ? 2 : 1; }

// Device view of an iso_kv4.  Strides in bytes; a page holds every kv head's tokens, a head's tokens are contiguous.
struct kv4_view {
    unsigned char *k, *v, *ks, *vs;
    int n_pages, page, page_shift;
};
inline kv4_view kv4_view_of(const iso_kv4 &c) {
    return kv4_view{(unsigned char *)c.k, (unsigned char *)c.v, (unsigned char *)c.k_scale, (unsigned char *)c.v_scale,
                    c.n_pages, c.page, __builtin_ctz((unsigned)c.page)};
}
// Ragged batch: request i has rows [row_start[i], row_start[i+1]) of the step's tensors and kv_len[i] tokens, the rows' own among
// them; token j is at offset j % page of page table[i * max_pages + j / page].
struct kv4_batch {
    const int *table, *row_start, *kv_len;
    int max_pages, n_seqs, total_rows;
};

// Value of a scale byte, as the conversion instructions take it (they read the exponent field: 0 is 2^-127, 255 is NaN).
__device__ __forceinline__ float kv4_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// Rows of request i that exist, and the position of its row t: base + t.
struct kv4_rows {
    int first, n, base;
};
template <typename P> __device__ __forceinline__ kv4_rows kv4_rows_of(P row_start, P kv_len, int total_rows, int i) {
    const int lo = row_start[i], hi = row_start[i + 1];
    const int base = kv_len[i] - (hi - lo);
    const int first = max(0, lo), last = min(total_rows, hi);
    return kv4_rows{first, max(0, last - first), base + (first - lo)};
}
// Keys of request i that its table can hold.
template <typename P> __device__ __forceinline__ int kv4_keys_of(P kv_len, int max_pages, int i, int page_shift) {
    const long long cap = (long long)max_pages << page_shift;
    return (int)min((long long)max(0, kv_len[i]), cap);
}

// ---- what both tiled attention kernels use
typedef unsigned long long u64;
typedef __bf16 bf16x4_v __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_v __attribute__((ext_vector_type(2)));
constexpr int COHERENT = 1 | 16;      // buffer cache policy sc0 | sc1: system scope, bypasses the XCD-local L2

// Eight elements of a code word (exact).
__device__ __forceinline__ bf16x8_t unpack8(unsigned w, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Wave-uniform values are made scalar explicitly, and what is read at a uniform place is read by the scalar unit: vector loads come
// back in order, so a page number among them would have to wait for the codes requested before it.
typedef const __attribute__((address_space(4))) int *scalar_ints;
__device__ __forceinline__ scalar_ints scalar(const int *p) { return (scalar_ints)(uintptr_t)p; }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ u64 uniform(u64 x) { return (u64)(unsigned)uniform((int)x) | (u64)(unsigned)uniform((int)(x >> 32)) << 32; }
// Buffer from p + at on: a lane's address needs no addition in a vector register.  (`at` is not taken as the scalar offset: that one counts
// in the comparison with the buffer's size, which cannot be more than 4 GB.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t beyond(unsigned char *p, u64 at) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)(p + at), 0, -1, 0x00020000);
}
