// The paged 4-bit KV cache's bookkeeping and its rows in and out (gfx950).
#include "kv4.h"
#include "wave_scan.h"

namespace pevlm {

// ------------------------------------------------------------------------------------------
// Slots.  What a request gets depends on those before it only through two running sums (rows, pages), so one workgroup
// takes the requests T at a time: inclusive scans of the new tokens, then of the pages that the requests which fit lack.  Sums stop
// at 2^32 - 1, which is more than any bound they are held to.  A step's few rows are filled in by the same workgroup from LDS; a prompt's by
// a launch of one row a lane.  Bound by latency: 2.9 us for 64 requests of one token, 2.8 and 4.1 for four prompts of 141 K tokens.
// ------------------------------------------------------------------------------------------
// One launch against two, by the call: 64 requests of 1, 8 and 32 tokens 8.3 to 8.6 / 11.3 us, 1024 of one 8.6 / 11.4.  (Up to 8192 rows it would still
// serve, four requests of 2048 tokens 8.5 / 11.4.)  Beyond 1024 requests their lengths would not stay in LDS.
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
        // 256 / 1024 threads, the kernel: 64 requests of 1 token 3.0 / 3.5 us, of 8 4.4 / 4.0, of 32 10.1 / 6.0; 256 of 1 3.3 / 3.6; 512 of 1 5.4 / 4.0
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
// Rows in and out.  A wavefront takes kRowsAt rows of one KV head, K and V.  A lane has 8 neighbouring elements of a row (chunk
// l % (D / 8)), so that the wavefront's loads cover whole rows; four lanes make a block and find its scale.  What lane c of the four
// encodes of their four rows is one word of each row's 16 bytes: a transpose within the four gives every lane the 16 bytes of one row,
// and a wavefront's store is a record's codes as they lie, if its rows are neighbours in the cache.  Out the same way back.  Bound by HBM:
// 65.9 K tokens x 4 heads x 128 in 31.0 us, out 27.6 (171 MB each, 5.5 and 6.2 TB/s), 100 K x 8 out 96 (524 MB, 5.4).
// ------------------------------------------------------------------------------------------
template <int D>
struct RowsCfg {
    static constexpr int CH = D / 8;        // chunks of a row
    static constexpr int PER_LOAD = 64 / CH; // rows that one load of 8 elements a lane covers
    static constexpr int ROWS = kv4_rows_of_wave(D);
};

constexpr int kXor1 = 0xB1, kXor2 = 0x4E;  // quad_perm of the neighbour, and of the one after the next

template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int32_t)x, CTRL, 0xf, 0xf, true);
}

// w[i] of lane c of four becomes w[c] of lane i
__device__ __forceinline__ void transpose_quad(uint32_t (&w)[4], int32_t c)
{
    const auto swap = [&](uint32_t &a, uint32_t &b, bool upper, auto from) {
        const uint32_t x = from(upper ? a : b);
        (upper ? a : b) = x;
    };
    const auto one = [](uint32_t x) { return quad<kXor1>(x); };
    const auto two = [](uint32_t x) { return quad<kXor2>(x); };
    swap(w[0], w[1], c & 1, one);
    swap(w[2], w[3], c & 1, one);
    swap(w[0], w[2], c & 2, two);
    swap(w[1], w[3], c & 2, two);
}

// Exponent of a block's scale from the bits of its largest magnitude a = 1.f * 2^(E - 127): the smallest e with a <= 6 * 2^e
__device__ __forceinline__ int32_t kv4_exponent(uint32_t a)
{
    if (a == 0) return 0;
    const int32_t e = (int32_t)(a >> 23) - 129 + ((a & 0x7fffffu) > 0x400000u);
    return e < kKv4MinExp ? kKv4MinExp : (e > kKv4MaxExp ? kKv4MaxExp : e);
}

// Where a slot lies in the pool; < 0: nowhere
template <int D>
__device__ __forceinline__ int64_t slot_record(const Kv4Pool &p, int32_t slot, int32_t head, int32_t &t)
{
    t = slot & (kKv4Record - 1);
    const int32_t page = slot >> p.page_shift;
    if (slot < 0 || page >= p.num_pages) return -1;
    return kv4_record<D>(p, page, head, (slot & ((1 << p.page_shift) - 1)) / kKv4Record);
}

typedef __attribute__((ext_vector_type(4))) uint32_t Words;

// 8 elements of a row (BF16: one word has two, else one).  Nothing reads them again: past the caches' retention, which leaves the stores theirs
// (65.9 K tokens x 4 heads x 128 45.1 -> 37.0 us).
template <bool BF16>
struct Chunk {
    uint32_t w[BF16 ? 4 : 8];
};
template <bool BF16>
__device__ __forceinline__ Chunk<BF16> load_chunk(const void *rows, int64_t at)
{
    Chunk<BF16> x;
    const Words *src = reinterpret_cast<const Words *>((const char *)rows + at * (BF16 ? 2 : 4));
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
        const Words a = __builtin_nontemporal_load(src + h);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[h * 4 + i] = a[i];
    }
    return x;
}

// The lane's word of codes and its block's scale byte
template <bool BF16>
__device__ __forceinline__ uint32_t encode_chunk(const Chunk<BF16> &x, uint32_t &scale_byte)
{
    uint32_t a = 0;
    if constexpr (BF16) {
        for (int i = 0; i < 4; ++i) {
            const uint32_t hi = x.w[i] & 0x7fff0000u, lo = x.w[i] << 16 & 0x7fff0000u;
            a = max(a, max(hi, lo));
        }
    } else {
        for (int i = 0; i < 8; ++i) a = max(a, x.w[i] & 0x7fffffffu);
    }
    a = max(a, quad<kXor1>(a));
    a = max(a, quad<kXor2>(a));
    const int32_t e = kv4_exponent(a);
    const float scale = exp2_int(e);
    uint32_t codes = 0;
    if constexpr (BF16) {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x.w[0]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x.w[1]), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x.w[2]), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x.w[3]), scale, 3);
    } else {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x.w[0]), __uint_as_float(x.w[1]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x.w[2]), __uint_as_float(x.w[3]), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x.w[4]), __uint_as_float(x.w[5]), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x.w[6]), __uint_as_float(x.w[7]), scale, 3);
    }
    const bool fine = a < 0x7f800000u;
    scale_byte = fine ? e + kKv4Bias : kKv4NanScale;
    return fine ? codes : 0;
}

// The lanes' places: chunk of the row, lane of its four, block; rows row0 + i * PER_LOAD of the group that the lane reads or writes
// as chunks, the row c * PER_LOAD of them whose codes it has.
template <int D>
struct RowLane {
    int32_t c, block, chunk, row;
    __device__ __forceinline__ RowLane()
    {
        const int32_t lane = threadIdx.x & 63;
        chunk = lane % RowsCfg<D>::CH;
        row = lane / RowsCfg<D>::CH;
        c = chunk & 3;
        block = chunk >> 2;
    }
};

template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv4_store_kernel(Kv4Rows p, int32_t groups)
{
    using R = RowsCfg<D>;
    const int32_t id = blockIdx.x * 4 + (threadIdx.x >> 6), head = id % p.pool.n_kv_heads, group = id / p.pool.n_kv_heads;
    if (group >= groups) return;
    const RowLane<D> L;
    const int32_t row0 = group * R::ROWS + L.row, mine = row0 + L.c * R::PER_LOAD;
    const int32_t slot = mine < p.num_rows ? p.slot_map[mine] : -1;
    Chunk<BF16> k[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t row = row0 + i * R::PER_LOAD, at = row < p.num_rows ? row : p.num_rows - 1;
        const int64_t in_row = head * D + L.chunk * 8;
        k[i] = load_chunk<BF16>(p.k, at * p.k_stride + in_row);
        v[i] = load_chunk<BF16>(p.v, at * p.v_stride + in_row);
    }
    uint32_t kw[4], vw[4], scales = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t ks, vs;
        kw[i] = encode_chunk<BF16>(k[i], ks);
        vw[i] = encode_chunk<BF16>(v[i], vs);
        if (L.c == i) scales = ks | vs << 8;
    }
    transpose_quad(kw, L.c);
    transpose_quad(vw, L.c);
    int32_t t;
    const int64_t rec = slot_record<D>(p.pool, slot, head, t);
    if (rec < 0) return;
    uint8_t *base = p.pool.base + rec;
    *reinterpret_cast<uint4 *>(base + (L.block * 16 + t) * 16) = make_uint4(kw[0], kw[1], kw[2], kw[3]);
    *reinterpret_cast<uint4 *>(base + Kv4Cfg<D>::CODES + (L.block * 16 + t) * 16) = make_uint4(vw[0], vw[1], vw[2], vw[3]);
    *reinterpret_cast<uint16_t *>(base + Kv4Cfg<D>::SCALES + (L.block * 16 + t) * 2) = (uint16_t)scales;
}

template <bool BF16, bool STREAM>
__device__ __forceinline__ void store_chunk(void *rows, int64_t at, uint32_t codes, float scale)
{
    bf16x2 x[4];
    kv4_decode8(codes, scale, x);  // exact in either type: a value has two significant bits
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(uint32_t, x[j]);
    Words *dst = reinterpret_cast<Words *>((char *)rows + at * (BF16 ? 2 : 4));
    const auto put = [](Words x, Words *to) {
        if constexpr (STREAM) __builtin_nontemporal_store(x, to);
        else *to = x;
    };
    if constexpr (BF16) {
        put(Words{w[0], w[1], w[2], w[3]}, dst);
    } else {
        put(Words{w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u}, dst);
        put(Words{w[2] << 16, w[2] & 0xffff0000u, w[3] << 16, w[3] & 0xffff0000u}, dst + 1);
    }
}

// STREAM: more rows than the caches hold, which go past their retention (65.9 K tokens x 4 heads x 128 after a store 29.2 -> 28.3 us, the store that comes
// next 36.8 -> 30.5; 101 K x 8 108 -> 104); fewer stay for the call that reads them.
template <int D, bool BF16, bool STREAM>
__global__ __launch_bounds__(256) void kv4_load_kernel(Kv4Rows p, int32_t groups)
{
    using R = RowsCfg<D>;
    const int32_t id = blockIdx.x * 4 + (threadIdx.x >> 6), head = id % p.pool.n_kv_heads, group = id / p.pool.n_kv_heads;
    if (group >= groups) return;
    const RowLane<D> L;
    const int32_t row0 = group * R::ROWS + L.row, mine = row0 + L.c * R::PER_LOAD;
    const int32_t slot = mine < p.num_rows ? p.slot_map[mine] : -1;
    int32_t t;
    const int64_t rec = slot_record<D>(p.pool, slot, head, t);
    uint32_t kw[4] = {}, vw[4] = {}, scales = 0;
    if (rec >= 0) {
        const uint8_t *base = p.pool.base + rec;
        const uint4 k = *reinterpret_cast<const uint4 *>(base + (L.block * 16 + t) * 16);
        const uint4 v = *reinterpret_cast<const uint4 *>(base + Kv4Cfg<D>::CODES + (L.block * 16 + t) * 16);
        scales = *reinterpret_cast<const uint16_t *>(base + Kv4Cfg<D>::SCALES + (L.block * 16 + t) * 2) | 1u << 16;  // and: there is such a row
        kw[0] = k.x; kw[1] = k.y; kw[2] = k.z; kw[3] = k.w;
        vw[0] = v.x; vw[1] = v.y; vw[2] = v.z; vw[3] = v.w;
    }
    transpose_quad(kw, L.c);
    transpose_quad(vw, L.c);
    const uint32_t of_row[4] = {quad<0x00>(scales), quad<0x55>(scales), quad<0xAA>(scales), quad<0xFF>(scales)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!(of_row[i] >> 16)) continue;
        const int64_t row = row0 + i * R::PER_LOAD, in_row = head * D + L.chunk * 8;
        store_chunk<BF16, STREAM>(p.k, row * p.k_stride + in_row, kw[i], kv4_scale(of_row[i] & 255u));
        store_chunk<BF16, STREAM>(p.v, row * p.v_stride + in_row, vw[i], kv4_scale(of_row[i] >> 8 & 255u));
    }
}

constexpr int64_t kCacheBytes = 32 << 20;  // the XCDs' L2 caches

template <int D, bool BF16>
static hipError_t launch_rows(const Kv4Rows &p, bool in, hipStream_t stream)
{
    const int32_t groups = ceil_div(p.num_rows, RowsCfg<D>::ROWS);
    const dim3 grid((uint32_t)(((int64_t)groups * p.pool.n_kv_heads + 3) / 4));
    if (in) hipLaunchKernelGGL((kv4_store_kernel<D, BF16>), grid, dim3(256), 0, stream, p, groups);
    else if ((int64_t)p.num_rows * p.pool.n_kv_heads * D * (BF16 ? 4 : 8) > kCacheBytes) hipLaunchKernelGGL((kv4_load_kernel<D, BF16, true>), grid, dim3(256), 0, stream, p, groups);
    else hipLaunchKernelGGL((kv4_load_kernel<D, BF16, false>), grid, dim3(256), 0, stream, p, groups);
    return hipGetLastError();
}

static hipError_t launch_rows(const Kv4Rows &p, int32_t D, bool bf16, bool in, hipStream_t stream)
{
    if (D == 128) return bf16 ? launch_rows<128, true>(p, in, stream) : launch_rows<128, false>(p, in, stream);
    return bf16 ? launch_rows<64, true>(p, in, stream) : launch_rows<64, false>(p, in, stream);
}

hipError_t launch_kv4_store(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream) { return launch_rows(p, D, bf16, true, stream); }
hipError_t launch_kv4_load(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream) { return launch_rows(p, D, bf16, false, stream); }

}  // namespace pevlm
