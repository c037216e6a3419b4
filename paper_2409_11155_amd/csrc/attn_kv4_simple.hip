// Attention of a ragged batch over the paged 4-bit cache, one wavefront per (query row, query head): online softmax over 64-key
// slices, fp32 throughout.  Row t of request i is the token at kv_len - rows + t and sees key j iff j is not behind it and j's page
// exists; a row that sees no key is zero.  ISO_FLAG_SIMPLE_ATTN forces it.
#include "kv4.h"

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void attn_kv4_simple_kernel(const T *__restrict__ q, int q_stride, kv4_view c, kv4_batch b,
                                                              T *__restrict__ out, int nq, int nkv) {
    constexpr int PER = D / 64;
    __shared__ float qs[4][D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row = blockIdx.x * 4 + wave, h = blockIdx.y, g = h / (nq / nkv);
    int i = 0;                                          // the row's request: the last one that starts at or before it
    for (int lo = 0, hi = b.n_seqs; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (b.row_start[mid] <= row) lo = mid;
        else hi = mid;
        i = lo;
    }
    const kv4_rows rw = kv4_rows_of(b.row_start, b.kv_len, b.total_rows, i);
    const bool active = row >= rw.first && row < rw.first + rw.n;
    const float scale = 1.0f / sqrtf((float)D);
    if (active)
        for (int e = lane; e < D; e += 64) qs[wave][e] = iso_to_f32(q[(size_t)row * q_stride + (size_t)h * D + e]) * scale;
    __syncthreads();
    if (!active) return;                                // rows in front of the first request or behind the last
    const int keys = kv4_keys_of(b.kv_len, b.max_pages, i, c.page_shift);
    const int n_vis = min(keys, rw.base + (row - rw.first) + 1);
    const int *table = b.table + (size_t)i * b.max_pages;
    float o[PER] = {};
    float m = -INFINITY, l = 0.f;
    for (int j0 = 0; j0 < n_vis; j0 += 64) {
        const int j = j0 + lane;
        const int pg = j < n_vis ? table[j >> c.page_shift] : -1;
        const bool seen = pg >= 0 && pg < c.n_pages;
        const size_t tok = seen ? (((size_t)pg * nkv + g) << c.page_shift) + (j & (c.page - 1)) : 0;
        float sc = -INFINITY;
        if (seen) {
            float acc = 0.f;
            for (int w = 0; w < D / 8; ++w) {
                const unsigned code = reinterpret_cast<const unsigned *>(c.k + tok * (D / 2))[w];
                const float f = kv4_scale(c.ks[tok * (D / KV4_BLOCK) + w / 4]);
                const bf16x2_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 1),
                                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 3)};
#pragma unroll
                for (int x = 0; x < 8; ++x) acc = fmaf(qs[wave][8 * w + x], (float)p[x / 2][x % 2], acc);
            }
            sc = acc;
        }
        const float m_new = fmaxf(m, iso_wave_max(sc));
        const float at = m_new == -INFINITY ? 0.f : m_new;          // nothing seen yet: every probability is exp(-inf)
        const float p = seen ? expf(sc - at) : 0.f;
        const float alpha = expf(m - at);
        l = l * alpha + iso_wave_sum(p);
#pragma unroll
        for (int r = 0; r < PER; ++r) o[r] *= alpha;
        const int cnt = min(64, n_vis - j0);
        for (int jj = 0; jj < cnt; ++jj) {
            if (!__shfl((int)seen, jj, 64)) continue;               // whatever a missing page's address holds stays out
            const float pj = __shfl(p, jj, 64);
            const size_t tv = (size_t)__shfl((long long)tok, jj, 64);
#pragma unroll
            for (int r = 0; r < PER; ++r) {
                const int e = lane + 64 * r;
                const unsigned byte = c.v[tv * (D / 2) + e / 2];
                const bf16x2_t x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(byte, kv4_scale(c.vs[tv * (D / KV4_BLOCK) + e / KV4_BLOCK]), 0);
                o[r] = fmaf(pj, (float)x[e & 1], o[r]);
            }
        }
        m = m_new;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int r = 0; r < PER; ++r) out[((size_t)row * nq + h) * D + lane + 64 * r] = iso_from_f32<T>(o[r] * inv);
}

}  // namespace

hipError_t iso_launch_attn_kv4_simple(int dtype, const void *q, int q_stride, const iso_kv4 &cache, const kv4_batch &b, void *out, int nq,
                                      int nkv, int d, hipStream_t s) {
    const kv4_view c = kv4_view_of(cache);
    const dim3 grid((b.total_rows - 1) / 4 + 1, nq), block(256);
#define ISO_KV4_SIMPLE(TT, DD) \
    hipLaunchKernelGGL((attn_kv4_simple_kernel<TT, DD>), grid, block, 0, s, (const TT *)q, q_stride, c, b, (TT *)out, nq, nkv)
    if (dtype == ISO_F32 && d == 64) ISO_KV4_SIMPLE(float, 64);
    else if (dtype == ISO_F32 && d == 128) ISO_KV4_SIMPLE(float, 128);
    else if (dtype == ISO_BF16 && d == 64) ISO_KV4_SIMPLE(bf16_t, 64);
    else if (dtype == ISO_BF16 && d == 128) ISO_KV4_SIMPLE(bf16_t, 128);
    else return hipErrorInvalidValue;
#undef ISO_KV4_SIMPLE
    return hipGetLastError();
}
