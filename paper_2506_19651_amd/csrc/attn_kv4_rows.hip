// Attention over the paged 4-bit KV cache for many rows (gfx950): the (row, query head) pairs of a KV head fill tiles of 128.
//
// Tile arithmetic of the bf16 kernels (attn_bf16_tile.h), 32 pairs a wavefront, 64 keys a tile, four wavefronts that share the keys.  The codes of a
// tile are fetched two tiles ahead into registers, a record a wavefront, and go as bf16 numbers, exactly, into one of two LDS stages while
// the other is worked on: 16 conversions and 4 LDS writes a wavefront and tensor, next to 32 matrix instructions of 32 cycles.
//
// Weights are rounded to bf16 once (2^-8); their sum is taken before that, in fp32, so that lse has none of it.
#include "attn_bf16_tile.h"
#include "attn_kv4.h"

namespace pevlm {

namespace {

constexpr int NW = 4;
constexpr int kPairs = 1 << kKv4RowsTileShift;
static_assert(kPairs == NW * 32 && kKeyTile == kKv4Record << kKv4RowsStepShift, "a wavefront has 32 pairs and stages a record");

// What the wavefronts say of the records that they staged
struct StageNote {
    uint64_t nan[NW];     // lanes whose block of V is NaN, and some row sees it
    int32_t tok[NW];      // first token; -1: not there
    int32_t special[NW];  // whether some row does not see some key of it, or some value is NaN
};

struct NoLoads {
    __device__ __forceinline__ void issue(int) const {}
};

// Weights of a tile against reference m as bf16 pairs, and their sum over the lane's 32 keys before they are rounded
__device__ __forceinline__ float tile_weights(const f32x16 (&s)[2], float c_log2, float m, u32x4 (&pf)[4])
{
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int kc = j >> 1, i = (j & 1) * 8 + w * 2;
            const float a = weight(s[kc][i], c_log2, m), b = weight(s[kc][i + 1], c_log2, m);
            sum[w] += a + b;
            pf[j][w] = weight_pair(a, b);
        }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

}  // namespace

template <int D>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv4_rows_kernel(Kv4Attn p)
{
    using C = TileCfg<D>;
    using F = Kv4Cfg<D>;
    constexpr int KSTEPS = C::KSTEPS, DBLK = C::DBLK, ROWB = C::ROWB, CH = C::CH, TILEB = C::TILEB;
    constexpr int WORDS = D / 32;  // words of codes that a lane stages of a tensor
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][TILEB];
    __shared__ StageNote notes[2];

    const Place at = find_place<false>(p, blockIdx.x);
    if (at.s < 0) return;
    const Request r = at.r;
    int32_t tile, split;
    const int32_t g = divide(divide(at.rest, at.tiles, tile), at.splits, split);
    const int32_t item = at.first_item + at.rest;
    const int32_t head0 = first_head(p, g), G = heads_of(p, g);
    const int32_t pair0 = tile * kPairs, n_pairs = min(r.rows * G - pair0, kPairs);
    if (n_pairs <= 0) return;
    const Span span = span_of(r);
    const int32_t steps = steps_of(p, span), per = divide_up(steps, at.splits);
    const int32_t tile0 = split * per, n_tiles = max(0, min(per, steps - tile0));

    const int32_t tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kg = lane >> 4, l32 = lane & 31, g32 = lane >> 5;
    const int32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    LaneOff L;
    L.g32 = g32;
    L.k_row_off = l32 * ROWB;
    L.k_swz = l32 & (CH - 1);
    L.v_row_off = (g32 * 4 + (l16 >> 2)) * ROWB + (lane & 1) * 8;
    L.v_ch_lo = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    L.v_swz = (lane >> 2) & C::VSW;

    // ---- staging: the wavefront's record of a tile
    const int32_t *const table = p.table + (int64_t)at.s * p.max_pages;
    const int32_t rec_shift = p.pool.page_shift - 4;
    const uint32_t head_bytes = (uint32_t)F::BYTES << rec_shift, page_bytes = head_bytes * p.pool.n_kv_heads, head_off = head_bytes * g;
    const int32_t pos_lo = r.held - r.rows + divide(pair0, G), pos_hi = r.held - r.rows + divide(pair0 + n_pairs - 1, G);
    const int32_t near_lo = near_of(r, pos_lo), near_hi = near_of(r, pos_hi);
    const auto record_of = [&](int32_t t) {  // -1: none
        const int32_t v = (tile0 + t) * NW + wave;
        return t < n_tiles && v < span.records ? (v < span.n_sink ? v : v - span.n_sink + span.near) : -1;
    };
    const auto page_of = [&](int32_t t) {
        const int32_t rec = record_of(t);
        return table[(rec < 0 ? 0 : rec) >> rec_shift];
    };
    const uint32_t code_off = D == 128 ? lane * 16 : (kg >> 1) * 256 + l16 * 16 + (kg & 1) * 8;
    const uint32_t scale_off = F::SCALES + ((D == 128 ? kg : kg >> 1) * 16 + (l16 & 14)) * 2, scale_bit = (l16 & 1) * 16;
    struct Codes {
        uint32_t k[WORDS], v[WORDS], scales;
        int32_t tok;
    };
    const auto fetch = [&](Codes &c, int32_t t, int32_t page_loaded) {
        const int32_t rec = record_of(t), page = __builtin_amdgcn_readfirstlane(page_loaded);
        const bool there = rec >= 0 && page >= 0 && page < p.pool.num_pages;
        c.tok = there ? rec * kKv4Record : -1;
        const uint64_t off = there ? (uint64_t)(uint32_t)page * page_bytes + head_off + (uint32_t)(rec & ((1 << rec_shift) - 1)) * F::BYTES : 0;
        const uint8_t *base = p.pool.base + off;
        if constexpr (D == 128) {
            const uint4 k = *reinterpret_cast<const uint4 *>(base + code_off), v = *reinterpret_cast<const uint4 *>(base + F::CODES + code_off);
            c.k[0] = k.x; c.k[1] = k.y; c.k[2] = k.z; c.k[3] = k.w;
            c.v[0] = v.x; c.v[1] = v.y; c.v[2] = v.z; c.v[3] = v.w;
        } else {
            const uint2 k = *reinterpret_cast<const uint2 *>(base + code_off), v = *reinterpret_cast<const uint2 *>(base + F::CODES + code_off);
            c.k[0] = k.x; c.k[1] = k.y;
            c.v[0] = v.x; c.v[1] = v.y;
        }
        c.scales = *reinterpret_cast<const uint32_t *>(base + scale_off);
    };
    const auto stage = [&](Codes &c, int32_t st) {
        uint32_t v_scale = c.scales >> (scale_bit + 8) & 255u;
        // the values of a key that no row sees, and NaN blocks, count as 0
        const int32_t j = c.tok + l16;
        const bool seen = c.tok >= 0 && j <= pos_hi && (j >= near_lo || j < r.sink);
        const uint64_t nan = __ballot(seen && v_scale == kKv4NanScale);
        const bool whole = c.tok >= 0 && c.tok + 15 <= pos_lo && (c.tok >= near_hi || c.tok + 15 < r.sink);
        if (!seen || v_scale == kKv4NanScale) {
            v_scale = kKv4Bias;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) c.v[w] = 0;
        }
        const float ks = kv4_scale(c.scales >> scale_bit & 255u), vs = kv4_scale(v_scale);
        const int32_t row = wave * kKv4Record + l16;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const int32_t ch = kg * WORDS + w;
            bf16x2 x[4];
            kv4_decode8(c.k[w], ks, x);
            *reinterpret_cast<uint4 *>(lds[st][0] + row * ROWB + ((ch ^ (row & (CH - 1))) << 4)) =
                make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]), __builtin_bit_cast(uint32_t, x[3]));
            kv4_decode8(c.v[w], vs, x);
            *reinterpret_cast<uint4 *>(lds[st][1] + row * ROWB + ((ch ^ ((row & C::VSW) << 2)) << 4)) =
                make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]), __builtin_bit_cast(uint32_t, x[3]));
        }
        if (lane == 0) {
            notes[st].nan[wave] = nan;
            notes[st].tok[wave] = c.tok;
            notes[st].special[wave] = !whole || nan != 0;
        }
    };

    Codes codes;
    int32_t page = page_of(0);
    const int32_t page1 = page_of(1), page2 = page_of(2);

    // ---- queries: the lane's pair, elements kk * 16 + g32 * 8 .. + 8 of k-step kk
    const int32_t my_pair = pair0 + min(wave * 32 + l32, n_pairs - 1);
    int32_t in_row;
    const int32_t row = divide(my_pair, G, in_row), head = query_head(p, head0 + in_row);
    const int32_t pos = r.held - r.rows + row, near = near_of(r, pos);
    const int64_t to = (int64_t)(r.row0 + row) * p.n_q_heads + head;
    bf16x8 qf[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>((const uint16_t *)p.q + to * D + kk * 16 + g32 * 8);
    const bool active = wave * 32 < n_pairs;
    const int32_t wave_pos_hi = r.held - r.rows + divide(pair0 + min(wave * 32 + 31, n_pairs - 1), G);  // keys behind it are not for this wavefront

    float m_ref = -INFINITY, l_run = 0.f;
    uint32_t lost = 0;
    f32x16 o[DBLK], s[2];
#pragma unroll
    for (int b = 0; b < DBLK; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    u32x4 pf[4];

    if (n_tiles > 0) {
        fetch(codes, 0, page);
        stage(codes, 0);
        fetch(codes, 1, page1);
        page = page2;
    }
    const NoLoads none;
    for (int32_t t = 0; t < n_tiles; ++t) {
        const int32_t st = t & 1;
        __syncthreads();  // tile t stands, and nobody reads the other stage any more
        stage(codes, st ^ 1);  // behind the last tile: one that is not there
        const int32_t page_next = page_of(t + 3);
        fetch(codes, t + 2, page);
        page = page_next;
        const StageNote &note = notes[st];
        const int32_t first_tok = __builtin_amdgcn_readfirstlane(note.tok[0]);
        if (!active || first_tok > wave_pos_hi) continue;
        qk_tile<D, false, 1>(lds[st][0], L, qf, s, none, [] {}, [] {});
        if (__builtin_amdgcn_readfirstlane(note.special[0] | note.special[1] | note.special[2] | note.special[3])) {
#pragma unroll
            for (int e = 0; e < NW; ++e) {
                const int32_t tok = note.tok[e];
                const auto sees = [&](int32_t j) { return tok >= 0 && j <= pos && (j >= near || j < r.sink); };
#pragma unroll
                for (int i = 0; i < 8; ++i) {  // entries of keys e * 16 .. + 16 of the tile
                    const int32_t c = (i >> 2) * 8 + (i & 3) + 4 * g32;
                    if (!sees(tok + c)) s[e >> 1][(e & 1) * 8 + i] = -INFINITY;
                }
                for (uint64_t bad = note.nan[e]; bad; bad &= bad - 1) {
                    const int32_t from = __builtin_ctzll(bad);
                    if (sees(tok + (from & 15))) lost |= 1u << (D == 128 ? from >> 4 : from >> 5);
                }
            }
        }
        float psum = tile_weights(s, p.c_log2, reference_of(m_ref), pf);
        const bool up = sum_reached_step(psum) || m_ref == -INFINITY;
        if (__any(up)) {
            const float mx = row_max(s) * p.c_log2;
            const bool has = m_ref != -INFINITY;
            const float m_new = (int)up | __shfl_xor((int)up, 32) ? fmaxf(m_ref, mx) : m_ref;
            const float alpha = has ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
            m_ref = m_new;
            psum = tile_weights(s, p.c_log2, reference_of(m_ref), pf);
            l_run *= alpha;
#pragma unroll
            for (int b = 0; b < DBLK; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
        }
        l_run += psum;
        pv_tile<D>(lds[st][1], L, pf, o);
    }

    // ---- the lane's pair: elements b * 32 + i4 * 8 + g32 * 4 .. + 4
    const float l = l_run + __shfl_xor(l_run, 32);
    if (wave * 32 + l32 >= n_pairs) return;
    const int64_t slot = (int64_t)item * p.tile_pairs + wave * 32 + l32;
#pragma unroll
    for (int b = 0; b < DBLK; ++b)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            f32x4 x = {o[b][i4 * 4], o[b][i4 * 4 + 1], o[b][i4 * 4 + 2], o[b][i4 * 4 + 3]};
            if (lost >> b & 1u) x = f32x4{NAN, NAN, NAN, NAN};
            const int32_t d4 = b * 32 + i4 * 8 + g32 * 4;
            if (at.splits > 1) store_part<D>(p, slot, d4, x, m_ref, l);
            else store_pair<D, true>(p, to, d4, x, m_ref, l);
        }
}

void launch_attn_kv4_rows(const Kv4Attn &p, int32_t D, hipStream_t stream)
{
    const dim3 grid((p.grid + 7) / 8 * 8), block(NW * 64);
    if (D == 128) hipLaunchKernelGGL(attn_kv4_rows_kernel<128>, grid, block, 0, stream, p);
    else hipLaunchKernelGGL(attn_kv4_rows_kernel<64>, grid, block, 0, stream, p);
}

}  // namespace pevlm
