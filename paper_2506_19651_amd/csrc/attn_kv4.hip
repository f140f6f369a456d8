// Attention over the paged 4-bit KV cache (gfx950).
//
// One wavefront per (row, query head): 64 keys a step, one to a lane; scores, a running maximum and sum of the softmax, then every
// lane adds up D / 64 elements of the values.  All products and sums are in fp32.
#include "kv4.h"

namespace pevlm {

template <bool BF16>
__device__ __forceinline__ float attn_element(const void *p, int64_t i)
{
    return BF16 ? __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16) : ((const float *)p)[i];
}

__device__ __forceinline__ uint16_t bf16_nearest(float f)
{
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0;
    u += 0x7fffu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}

template <int D, bool BF16>
__global__ __launch_bounds__(64) void attn_kv4_kernel(Kv4Attn p)
{
    using C = Kv4Cfg<D>;
    __shared__ float query[D];
    const int32_t row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    int32_t s = -1, i = 0;
    for (int32_t s0 = 0; s0 < p.num_seqs && s < 0; s0 += 64) {
        const int32_t mine = s0 + lane;
        bool has = false;
        if (mine < p.num_seqs) {
            const int64_t first = p.row_start[mine], n = p.row_len[mine];
            has = first >= 0 && n > 0 && first + n <= p.num_rows && row >= first && row < first + n;
        }
        const uint64_t found = __ballot(has);
        if (found) s = s0 + __builtin_ctzll(found);
    }
    if (s < 0) return;
    i = row - p.row_start[s];
    const int64_t width = (int64_t)p.max_pages << p.pool.page_shift;
    const int32_t given = p.seq_len[s], held = given < 0 ? 0 : (given < width ? given : (int32_t)width);
    const int32_t pos = held - p.row_len[s] + i;
    const int32_t sink = p.sink_len ? p.sink_len[s] : 0, window = p.window ? p.window[s] : -1;
    const int64_t near = window < 0 ? 0 : (int64_t)pos - window + 1;  // first token inside the window
    const int32_t g = p.heads.kv_of_q[h];
    for (int32_t d = lane; d < D; d += 64) query[d] = attn_element<BF16>(p.q, ((int64_t)row * p.n_q_heads + h) * D + d);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[D / 64];
    for (int e = 0; e < D / 64; ++e) acc[e] = 0.f;
    for (int32_t j0 = 0; j0 <= pos; j0 += 64) {
        if (j0 >= sink && j0 + 63 < near) continue;
        const int32_t j = j0 + lane, column = j >> p.pool.page_shift, in_page = j & ((1 << p.pool.page_shift) - 1);
        bool seen = j <= pos && (j >= near || j < sink);
        int32_t page = 0;
        if (seen) {
            page = p.table[(int64_t)s * p.max_pages + column];
            seen = page >= 0 && page < p.pool.num_pages;
        }
        const int64_t rec = kv4_record<D>(p.pool, seen ? page : 0, g, in_page / kKv4Record);
        const int32_t t = in_page % kKv4Record;
        float score = -INFINITY;
        if (seen) {
            float sum = 0.f;
            for (int b = 0; b < C::NB; ++b) {
                const uint8_t *codes = p.pool.base + rec + (b * 16 + t) * 16;
                const float scale = kv4_scale(p.pool.base[rec + C::SCALES + (b * 16 + t) * 2]);
                for (int k = 0; k < 16; ++k) {
                    sum += kv4_value(codes[k]) * scale * query[b * 32 + 2 * k];
                    sum += kv4_value(codes[k] >> 4) * scale * query[b * 32 + 2 * k + 1];
                }
            }
            score = sum * p.scale;
        }
        float top = score;
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
        const float w = seen ? expf(score - base) : 0.f, alpha = expf(m - base);
        l *= alpha;
        for (int e = 0; e < D / 64; ++e) acc[e] *= alpha;
        m = m_new;
        float sum = w;
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        l += sum;
        const uint64_t keys = __ballot(seen);
        for (int k = 0; k < 64; ++k) {
            if (!(keys >> k & 1)) continue;
            const float wk = __shfl(w, k);
            const int64_t r = __shfl(rec, k);
            const int32_t tk = __shfl(t, k);
            for (int e = 0; e < D / 64; ++e) {
                const int32_t d = lane * (D / 64) + e, b = d / 32;
                const uint32_t byte = p.pool.base[r + C::CODES + (b * 16 + tk) * 16 + d % 32 / 2];
                const float scale = kv4_scale(p.pool.base[r + C::SCALES + (b * 16 + tk) * 2 + 1]);
                acc[e] += wk * (kv4_value(d & 1 ? byte >> 4 : byte) * scale);
            }
        }
    }
    const bool none = m == -INFINITY && l == 0.f;
    for (int e = 0; e < D / 64; ++e) {
        const float x = none ? 0.f : acc[e] / l;
        const int64_t o = ((int64_t)row * p.n_q_heads + h) * D + lane * (D / 64) + e;
        if (BF16) ((uint16_t *)p.out)[o] = bf16_nearest(x);
        else ((float *)p.out)[o] = x;
    }
    if (p.lse && lane == 0) p.lse[(int64_t)row * p.n_q_heads + h] = none ? -INFINITY : m + logf(l);
}

hipError_t launch_attn_kv4(const Kv4Attn &p, int32_t D, bool bf16, hipStream_t stream)
{
    const auto kernel = D == 128 ? (bf16 ? attn_kv4_kernel<128, true> : attn_kv4_kernel<128, false>)
                                 : (bf16 ? attn_kv4_kernel<64, true> : attn_kv4_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3(p.num_rows, p.n_q_heads), dim3(64), 0, stream, p);
    return hipGetLastError();
}

}  // namespace pevlm
