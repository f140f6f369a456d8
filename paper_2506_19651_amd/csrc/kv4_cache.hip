// The paged 4-bit KV cache's bookkeeping and its rows in and out (gfx950).
#include "kv4.h"
#include "wave_scan.h"

namespace pevlm {

// ------------------------------------------------------------------------------------------
// Slots.  What a request gets depends on those before it only through two running sums (rows, pages), so one workgroup
// takes the requests T at a time: inclusive scans of the new tokens, then of the pages that the requests which fit lack.  Sums stop
// at 2^32 - 1, which is more than any bound they are held to.  A step's few rows are filled in by the same workgroup from LDS; a prompt's by
// a launch of one row a lane.  Bound by latency: kernel 4.2 us for 64 requests of one token where two launches took 3.9 and 2.6.
// ------------------------------------------------------------------------------------------
constexpr int32_t kSmallRows = 2048, kSmallRequests = 1024;

// inclusive sum over the workgroup; `waves` holds the wavefronts' sums
template <int T>
__device__ __forceinline__ uint32_t scan_sum(uint32_t x, uint32_t *waves)
{
    const auto add = [](uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); };
    x = wave_scan(x, add);
    if constexpr (T > 64) {
        const int32_t wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 63) waves[wave] = x;
        __syncthreads();
        uint32_t before = 0;
        for (int w = 0; w < wave; ++w) before = add(before, waves[w]);
        x = add(x, before);
    }
    return x;
}

// What a row of a request gets, from the request's lengths and first new page
struct RowOf {
    int32_t start, rows, held, first_free;  // held: before the new tokens
};

__device__ __forceinline__ void fill_row(const Kv4Slots &p, int32_t row, int32_t s, const RowOf &r)
{
    const int32_t i = row - r.start, in_page = (1 << p.page_shift) - 1;
    int32_t slot = -1, pos = 0;
    if (i >= 0 && i < r.rows) {
        const int32_t at = r.held + i, column = at >> p.page_shift;
        const int32_t have = (int32_t)(((int64_t)r.held + in_page) >> p.page_shift);
        int32_t *entry = p.table + (int64_t)s * p.max_pages + column;
        int32_t page;
        if (column < have) {
            page = *entry;
        } else {
            page = p.free_pages[r.first_free - (column - have)];
            if ((at & in_page) == 0) *entry = page;
        }
        if (page >= 0 && page < p.num_pages) slot = (page << p.page_shift) + (at & in_page);
        pos = (int32_t)((uint32_t)at + (uint32_t)(p.pos_offset ? p.pos_offset[s] : 0));
    }
    p.slot_map[row] = slot;
    if (p.pos_ids)
        for (int a = 0; a < 3; ++a) p.pos_ids[(int64_t)a * p.num_rows + row] = pos;
}

// The last request that starts at or before the row
template <class Start>
__device__ __forceinline__ int32_t request_of(int32_t n, int32_t row, Start start)
{
    int32_t s = 0, hi = n;
    while (hi - s > 1) {
        const int32_t mid = (s + hi) / 2;
        if (start(mid) <= row) s = mid;
        else hi = mid;
    }
    return s;
}

// SMALL: at most kSmallRequests requests and kSmallRows rows, which are filled in here
template <int T, bool SMALL>
__global__ __launch_bounds__(T) void kv4_requests_kernel(Kv4Slots p)
{
    __shared__ uint32_t waves[2][T / 64];
    __shared__ uint32_t rows_before, need_before, taken;
    __shared__ RowOf of[SMALL ? kSmallRequests : 1];
    const int64_t width = (int64_t)p.max_pages << p.page_shift;
    const int32_t round = (1 << p.page_shift) - 1;
    int32_t free = *p.num_free;
    free = free < 0 ? 0 : (free < p.free_capacity ? free : p.free_capacity);
    if (threadIdx.x == 0) rows_before = need_before = taken = 0;
    for (int32_t s0 = 0; s0 < p.num_seqs; s0 += T) {
        const int32_t s = s0 + threadIdx.x;
        const bool real = s < p.num_seqs;
        const int32_t given = real ? p.seq_len[s] : 0;
        const int64_t held = given < 0 ? 0 : given;
        int32_t more = real ? (p.new_len ? p.new_len[s] : 1) : 0;
        more = more < 0 ? 0 : more;
        __syncthreads();  // the sums before these requests stand
        const uint32_t end = __builtin_elementwise_add_sat(scan_sum<T>(more, waves[0]), rows_before);
        const uint32_t start = end == UINT32_MAX ? UINT32_MAX : end - more;  // beyond any row either way
        const bool fits = held + more <= width && end <= (uint32_t)p.num_rows;
        const int64_t have = (held + round) >> p.page_shift;
        const uint32_t need = fits ? (uint32_t)(((held + more + round) >> p.page_shift) - have) : 0;
        const uint32_t all = __builtin_elementwise_add_sat(scan_sum<T>(need, waves[1]), need_before);
        const bool served = fits && (need == 0 || all <= (uint32_t)free);
        if (real) {
            RowOf r;
            r.start = (int32_t)(start < INT32_MAX ? start : INT32_MAX);
            r.rows = served ? more : 0;
            r.held = (int32_t)held;
            r.first_free = served ? (int32_t)(free - 1 - (all - need)) : 0;
            p.row_start[s] = r.start;
            p.row_len[s] = r.rows;
            p.seq_len_out[s] = served ? (int32_t)(held + more) : given;
            if constexpr (SMALL) of[s] = r;
            else p.first_free[s] = r.first_free;
        }
        if (served && need > 0) atomicMax(&taken, all);  // of whole numbers: any order
        __syncthreads();  // both sums have been read
        if (threadIdx.x == T - 1) {
            rows_before = end;
            need_before = all;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *p.num_free_out = free - (int32_t)taken;
    if constexpr (SMALL)
        for (int32_t row = threadIdx.x; row < p.num_rows; row += T) {
            const int32_t s = request_of(p.num_seqs, row, [&](int32_t i) { return of[i].start; });
            fill_row(p, row, s, of[s]);
        }
}

__global__ __launch_bounds__(256) void kv4_slots_kernel(Kv4Slots p)
{
    const int32_t row = blockIdx.x * 256 + threadIdx.x;
    if (row >= p.num_rows) return;
    const int32_t s = request_of(p.num_seqs, row, [&](int32_t i) { return p.row_start[i]; });
    RowOf r;
    r.start = p.row_start[s];
    r.rows = p.row_len[s];
    r.held = p.seq_len_out[s] - r.rows;
    r.first_free = p.first_free[s];
    fill_row(p, row, s, r);
}

hipError_t launch_kv4_slots(const Kv4Slots &p, hipStream_t stream)
{
    if (p.num_rows <= kSmallRows && p.num_seqs <= kSmallRequests) {
        const bool few = p.num_seqs <= 256 && p.num_rows <= 512;
        if (few) hipLaunchKernelGGL((kv4_requests_kernel<256, true>), dim3(1), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((kv4_requests_kernel<1024, true>), dim3(1), dim3(1024), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((kv4_requests_kernel<1024, false>), dim3(1), dim3(1024), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.num_rows == 0) return e;
    hipLaunchKernelGGL(kv4_slots_kernel, dim3((p.num_rows + 255) / 256), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Rows in: a lane encodes one block of 32 elements.
// ------------------------------------------------------------------------------------------
// Exponent of a block's scale from the bits of its largest magnitude a = 1.f * 2^(E - 127): the smallest e with a <= 6 * 2^e
__device__ __forceinline__ int32_t kv4_exponent(uint32_t a)
{
    if (a == 0) return 0;
    const int32_t e = (int32_t)(a >> 23) - 129 + ((a & 0x7fffffu) > 0x400000u);
    return e < kKv4MinExp ? kKv4MinExp : (e > kKv4MaxExp ? kKv4MaxExp : e);
}

// Code of y, to nearest, ties to the even code
__device__ __forceinline__ uint32_t kv4_code(float y)
{
    const float m = fabsf(y);
    const uint32_t c = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.f);
    return c | (__float_as_uint(y) >> 31) << 3;
}

template <bool BF16>
__device__ __forceinline__ float kv4_element(const void *row, int32_t i)
{
    return BF16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[i] << 16) : ((const float *)row)[i];
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv4_store_kernel(Kv4Rows p)
{
    constexpr int NB = Kv4Cfg<D>::NB;
    const int64_t per_row = (int64_t)p.pool.n_kv_heads * 2 * NB;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= p.num_rows * per_row) return;
    const int32_t row = (int32_t)(id / per_row), unit = (int32_t)(id % per_row);
    const int32_t b = unit % NB, which = unit / NB % 2, head = unit / (2 * NB);
    const int32_t slot = p.slot_map[row];
    if (slot < 0 || slot >> p.pool.page_shift >= p.pool.num_pages) return;
    const size_t e = BF16 ? 2 : 4;
    const void *src = (const char *)(which ? p.v : p.k) + ((int64_t)row * (which ? p.v_stride : p.k_stride) + head * D + b * 32) * e;
    float x[32];
    uint32_t amax = 0;
    for (int i = 0; i < 32; ++i) {
        x[i] = kv4_element<BF16>(src, i);
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    const bool fine = amax < 0x7f800000u;
    const int32_t exp = kv4_exponent(amax);
    const float f = exp2_int(-exp);
    uint32_t w[4] = {0, 0, 0, 0};
    if (fine)
        for (int i = 0; i < 32; ++i) w[i / 8] |= kv4_code(x[i] * f) << (i % 8 * 4);
    const int32_t in_page = slot & ((1 << p.pool.page_shift) - 1), t = in_page % kKv4Record;
    uint8_t *rec = p.pool.base + kv4_record<D>(p.pool, slot >> p.pool.page_shift, head, in_page / kKv4Record);
    *reinterpret_cast<uint4 *>(rec + which * Kv4Cfg<D>::CODES + (b * 16 + t) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    rec[Kv4Cfg<D>::SCALES + (b * 16 + t) * 2 + which] = (uint8_t)(fine ? exp + kKv4Bias : kKv4NanScale);
}

// Rows out: a lane decodes one block
template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv4_load_kernel(Kv4Rows p)
{
    constexpr int NB = Kv4Cfg<D>::NB;
    const int64_t per_row = (int64_t)p.pool.n_kv_heads * 2 * NB;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= p.num_rows * per_row) return;
    const int32_t row = (int32_t)(id / per_row), unit = (int32_t)(id % per_row);
    const int32_t b = unit % NB, which = unit / NB % 2, head = unit / (2 * NB);
    const int32_t slot = p.slot_map[row];
    if (slot < 0 || slot >> p.pool.page_shift >= p.pool.num_pages) return;
    const int32_t in_page = slot & ((1 << p.pool.page_shift) - 1), t = in_page % kKv4Record;
    const uint8_t *rec = p.pool.base + kv4_record<D>(p.pool, slot >> p.pool.page_shift, head, in_page / kKv4Record);
    const uint4 c = *reinterpret_cast<const uint4 *>(rec + which * Kv4Cfg<D>::CODES + (b * 16 + t) * 16);
    const float scale = kv4_scale(rec[Kv4Cfg<D>::SCALES + (b * 16 + t) * 2 + which]);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const int64_t to = (int64_t)row * (which ? p.v_stride : p.k_stride) + head * D + b * 32;
    void *dst = which ? p.v : p.k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2 x[4];
        kv4_decode8(w[i], scale, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t two = __builtin_bit_cast(uint32_t, x[j]);  // exact: a value has two significant bits
            const int64_t at = to + i * 8 + j * 2;
            if (BF16) *reinterpret_cast<uint32_t *>((uint16_t *)dst + at) = two;
            else *reinterpret_cast<float2 *>((float *)dst + at) = make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u));
        }
    }
}

static dim3 blocks_grid(const Kv4Rows &p, int32_t D)
{
    return dim3((uint32_t)(((int64_t)p.num_rows * p.pool.n_kv_heads * 2 * (D / 32) + 255) / 256));
}

hipError_t launch_kv4_store(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream)
{
    const auto kernel = D == 128 ? (bf16 ? kv4_store_kernel<128, true> : kv4_store_kernel<128, false>)
                                 : (bf16 ? kv4_store_kernel<64, true> : kv4_store_kernel<64, false>);
    hipLaunchKernelGGL(kernel, blocks_grid(p, D), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_kv4_load(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream)
{
    const auto kernel = D == 128 ? (bf16 ? kv4_load_kernel<128, true> : kv4_load_kernel<128, false>)
                                 : (bf16 ? kv4_load_kernel<64, true> : kv4_load_kernel<64, false>);
    hipLaunchKernelGGL(kernel, blocks_grid(p, D), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace pevlm
