// Attention over the paged 4-bit KV cache for many rows (gfx950): the (row, query head) pairs of a KV head fill tiles of 128.
//
// Four wavefronts of 32 pairs share tiles of 64 keys.  The records of a tile go from the cache straight into LDS, as they lie, three tiles
// ahead, a record a wavefront.  K is read from there: a lane's 16 bytes are one block of one key, and its 32 elements, converted (exactly)
// a word at a time between the matrix instructions, are its share of four of them, if the k index runs over the blocks first.  So a tile of K is
// 4 KB of LDS reads a wavefront; as bf16 rows it would be 16, and with V's 16 four wavefronts would need all of what LDS delivers.  V goes on to a second
// place in LDS as bf16 rows (each wavefront its record), and comes back transposed.  The value products of a tile are issued among the
// next one's weights.
//
// (The scaled matrix instructions take 4-bit K as it is, against Q in two E4M3 parts: they lose what is below 2^-17 of a block's
// largest product, 9e-5 of a score of 5.)
//
// Bound by the matrix and vector instructions of its loop together: 128 rows x 28/4 heads x 128 over 65.9 K tokens (121 GFLOP) 129 us, 0.94 PFLOP/s where a
// large library product reaches 1.22; matrix cores are busy 46 % and vector instructions issue 60 % of the time, which a SIMD's two
// wavefronts overlap little.  Joining the parts (33 MB each way) takes 9 us of it.
//
// Weights are rounded to bf16 once (2^-8); their sum is taken before that, in fp32, so that lse has none of it.
//
// Waits.  Loads into LDS complete in issue order per wavefront, and every wavefront issues the same number in every tile (behind the last tile
// the pool's first record again, into a stage that nobody reads); nothing else in the loop is counted with them: the places of 64 tiles'
// records are held in a wavefront's lanes.  The top of a tile waits until only those of the two tiles after it are outstanding.  (Page numbers by
// scalar loads, one a tile, cost their latency on every tile: LDS reads and scalar loads share a counter.)
#include "attn_bf16_tile.h"
#include "attn_kv4.h"

namespace pevlm {

namespace {

constexpr int NW = 4;
constexpr int kPairs = 1 << kKv4RowsTileShift;
static_assert(kPairs == NW * 32 && kKeyTile == kKv4Record << kKv4RowsStepShift, "a wavefront has 32 pairs and stages a record");

// What the wavefronts say of the records that they staged
constexpr int32_t kSpecial = 1;  // beside a record's first token: some row does not see some key of it
struct ValueNote {
    uint64_t nan[NW];  // lanes whose block is NaN, and some row sees it
    int32_t tok[NW];
    int32_t tile;      // the last tile in which there were any
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

constexpr int kStages = 4;  // tiles of records in LDS

// 4 bytes a lane from global memory into LDS, as load_lds_16_base
__device__ __forceinline__ void load_lds_4_base(const void *sbase, uint32_t voff, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n" ::"s"(lds_addr), "v"(voff), "s"(sbase) : "memory");
}

// V^T fragment n (k-step n / DBLK, block n % DBLK) from rows that lie as value_chunk says; `at`: the lane's place in a block's 64 bytes
template <int D>
__device__ __forceinline__ bf16x8 read_values(const uint8_t *tv, const uint32_t (&at)[D / 32], int n)
{
    using C = TileCfg<D>;
    const int ks = n / C::DBLK, b = n % C::DBLK;
    bf16x8 dst;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
        const uint8_t *ptr = tv + (ks * 16 + tt * 8) * C::ROWB + at[b];
        const bf16x4 rb = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, ptr)));
        dst[tt * 4 + 0] = rb[0]; dst[tt * 4 + 1] = rb[1];
        dst[tt * 4 + 2] = rb[2]; dst[tt * 4 + 3] = rb[3];
    }
    return dst;
}

// O^T += V^T P^T, and WEIGHTS: the next tile's weights against reference m meanwhile, their sum before they are rounded
template <int D, bool WEIGHTS>
__device__ __forceinline__ float values(const uint8_t *tv, const uint32_t (&at)[D / 32], u32x4 (&pf)[4], f32x16 (&o)[D / 32], const f32x16 (&s)[2],
                                        float c_log2, float m, const bf16x8 (&vfirst)[kValuesAhead])
{
    using C = TileCfg<D>;
    constexpr int PF = kValuesAhead, NM = 4 * C::DBLK, PPM = 16 / NM;
    float sum[2] = {0.f, 0.f};
    bf16x8 vf[NM];
    float e[8];
#pragma unroll
    for (int n = 0; n < PF; ++n) vf[n] = vfirst[n];
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        const int ks = n / C::DBLK, b = n % C::DBLK;
        if (n + PF < NM) vf[n + PF] = read_values<D>(tv, at, n + PF);
        o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n], __builtin_bit_cast(bf16x8, pf[ks]), o[b], 0, 0, 0);
        if constexpr (WEIGHTS) {
#pragma unroll
            for (int x = 0; x < PPM; ++x) {
                const int pi = n * PPM + x, kc = pi >> 3, i = (pi & 7) * 2;
                float &e0 = e[(pi & 3) * 2], &e1 = e[(pi & 3) * 2 + 1];
                e0 = weight(s[kc][i], c_log2, m);
                e1 = weight(s[kc][i + 1], c_log2, m);
                asm volatile("" : "+v"(e0), "+v"(e1));  // here, not after the last MFMA
                sum[0] += e0;
                sum[1] += e1;
            }
            if (b == C::DBLK - 1) {
#pragma unroll
                for (int w = 0; w < 4; ++w) pf[ks][w] = weight_pair(e[w * 2], e[w * 2 + 1]);
                asm volatile("" : "+v"(pf[ks]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    return sum[0] + sum[1];
}

}  // namespace

template <int D, bool FEW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv4_rows_kernel(Kv4Attn p)
{
    using C = TileCfg<D>;
    using F = Kv4Cfg<D>;
    constexpr int DBLK = C::DBLK, ROWB = C::ROWB, TILEB = C::TILEB;
    constexpr int KK = D / 64;               // pairs of blocks
    constexpr int RAW = F::SCALES + 256;     // a record in LDS: 16 D bytes of codes, 64 words of which half are scales
    constexpr int NLD = D / 64 + 1;          // loads of a record
    __shared__ __attribute__((aligned(1024))) uint8_t lds_v[2][TILEB];  // bf16 rows
    __shared__ __attribute__((aligned(1024))) uint8_t lds_raw[kStages][NW][RAW];
    __shared__ __attribute__((aligned(16))) int32_t key_notes[kStages][NW];  // first token (-1: not there) and kSpecial
    __shared__ ValueNote value_notes[2];

    have_fields(p);
    const Place at = find_place<false, FEW, true>(p, blockIdx.x);
    if (at.s < 0) return;
    const Request r = at.r;
    int32_t tile, split;
    const int32_t g = divide(divide(at.rest, at.tiles, tile), at.splits, split);
    const int32_t part = at.first_part + at.rest;
    const int32_t head0 = first_head(p, g), G = heads_of(p, g);
    const int32_t pair0 = tile * kPairs, n_pairs = min(r.rows * G - pair0, kPairs);
    if (n_pairs <= 0) return;
    const Span span = span_of(r);
    const int32_t steps = steps_of(p, span), per = divide_up(steps, at.splits);
    const int32_t tile0 = split * per, n_tiles = max(0, min(per, steps - tile0));

    const int32_t tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kg = lane >> 4, l32 = lane & 31, g32 = lane >> 5;
    const int32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t v_at[DBLK];
#pragma unroll
    for (int b = 0; b < DBLK; ++b) {
        const int32_t row = g32 * 4 + (l16 >> 2);
        v_at[b] = row * ROWB + value_chunk<D>(row, b * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
    }

    // ---- staging: the wavefront's record of a tile
    const int32_t *const table = p.table + (int64_t)at.s * p.max_pages;
    const int32_t rec_shift = p.pool.page_shift - 4;
    const uint32_t head_bytes = (uint32_t)F::BYTES << rec_shift, page_bytes = head_bytes * p.pool.n_kv_heads, head_off = head_bytes * g;
    const int32_t pos_lo = r.held - r.rows + divide(pair0, G), pos_hi = r.held - r.rows + divide(pair0 + n_pairs - 1, G);
    const int32_t near_lo = near_of(r, pos_lo), near_hi = near_of(r, pos_hi);
    uint64_t rec_off;  // of lane i: the wavefront's record of the i-th of 64 tiles
    int32_t rec_tok;
    const auto read_records = [&](int32_t first) {
        const int32_t t = first + lane, v = (tile0 + t) * NW + wave;
        const int32_t rec = t < n_tiles && v < span.records ? (v < span.n_sink ? v : v - span.n_sink + span.near) : -1;
        const int32_t page = table[(rec < 0 ? 0 : rec) >> rec_shift], tok = rec * kKv4Record;
        const bool there = rec >= 0 && page >= 0 && page < p.pool.num_pages;
        const bool whole = tok + 15 <= pos_lo && (tok >= near_hi || tok + 15 < r.sink);
        rec_off = there ? (uint64_t)(uint32_t)page * page_bytes + head_off + (uint32_t)(rec & ((1 << rec_shift) - 1)) * F::BYTES : 0;
        rec_tok = there ? (whole ? tok : tok | kSpecial) : -1;
    };
    const uint32_t raw_addr = (uint32_t)(size_t)LDS_PTR(void, lds_raw) + wave * RAW;
    const auto load = [&](int32_t t) {  // the wavefront's record of tile t
        if ((t & 63) == 0) {
            read_records(t);
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), said to the compiler, which would wait for it on every tile
        }
        const int32_t l = t & 63, st = t % kStages;
        const uint64_t off = (uint64_t)(uint32_t)lane_value((int32_t)(rec_off >> 32), l) << 32 | (uint32_t)lane_value((int32_t)rec_off, l);
        const int32_t note = lane_value(rec_tok, l);
        const uint8_t *base = p.pool.base + off;
        const uint32_t to = raw_addr + st * (NW * RAW);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) load_lds_16_base(base + i * 1024, lane * 16, to + i * 1024);
        load_lds_4_base(base + F::SCALES, (lane & (D / 4 - 1)) * 4, to + F::SCALES);
        if (lane == 0) key_notes[st][wave] = note;
        return note;
    };
    // V of the wavefront's record as bf16 rows.  The values of a key that no row sees, and NaN blocks, count as 0.
    const int32_t block = D == 128 ? kg : kg >> 1;  // D = 64: half kg & 1 of it
    const auto stage_v = [&](int32_t t, int32_t noted_tok) {
        const uint8_t *raw = lds_raw[t % kStages][wave];
        uint32_t w[D / 32];
        if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4 *>(raw + F::CODES + lane * 16);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(raw + F::CODES + (block * 16 + l16) * 16 + (kg & 1) * 8);
            w[0] = x.x; w[1] = x.y;
        }
        uint32_t scale = raw[F::SCALES + (block * 16 + l16) * 2 + 1];
        const int32_t tok = noted_tok < 0 ? -1 : noted_tok & ~kSpecial, j = tok + l16;
        const bool seen = tok >= 0 && j <= pos_hi && (j >= near_lo || j < r.sink);
        const uint64_t nan = __ballot(seen && scale == kKv4NanScale);
        const uint32_t keep = seen && scale != kKv4NanScale ? 0xffffffffu : 0u;
        scale = keep ? scale : kKv4Bias;
        const int32_t row = wave * kKv4Record + l16;
        uint8_t *dst = lds_v[t & 1] + row * ROWB;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            bf16x2 x[4];
            kv4_decode8(w[i] & keep, kv4_scale(scale), x);
            *reinterpret_cast<uint4 *>(dst + value_chunk<D>(l16, kg * (D / 32) + i) * 16) =
                make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]), __builtin_bit_cast(uint32_t, x[3]));
        }
        if (lane == 0) {
            value_notes[t & 1].nan[wave] = nan;
            value_notes[t & 1].tok[wave] = tok;
            if (nan != 0) value_notes[t & 1].tile = t;
        }
    };

    if (tid < 2) value_notes[tid].tile = -1;
    int32_t note0 = -1, note1 = -1, note2 = -1;  // of the next three tiles
    if (n_tiles > 0) {
        note0 = load(0);
        note1 = load(1);
        note2 = load(2);
    }

    // ---- queries: the lane's pair, elements m * 8 .. + 8 of block kk * 2 + g32 for the m-th instruction of pair kk
    const int32_t my_pair = pair0 + min(wave * 32 + l32, n_pairs - 1);
    int32_t in_row;
    const int32_t row = divide(my_pair, G, in_row), head = query_head(p, head0 + in_row);
    const int32_t pos = r.held - r.rows + row, near = near_of(r, pos);
    const int64_t to = (int64_t)(r.row0 + row) * p.n_q_heads + head;
    bf16x8 qf[KK][4];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int m = 0; m < 4; ++m) qf[kk][m] = *reinterpret_cast<const bf16x8 *>((const uint16_t *)p.q + to * D + (kk * 2 + g32) * 32 + m * 8);
    // tiles with a key that some row of the wavefront may see: the others come last
    int32_t n_w = 0;
    const int32_t wave_pos_hi = r.held - r.rows + divide(pair0 + min(wave * 32 + 31, n_pairs - 1), G);
    if (wave * 32 < n_pairs && wave_pos_hi >= 0) {
        const int32_t rec = wave_pos_hi / kKv4Record;
        const int32_t v = rec < span.n_sink ? rec : (rec < span.near ? span.n_sink - 1 : rec - span.near + span.n_sink);
        n_w = max(0, min(n_tiles, (v >> kKv4RowsStepShift) - tile0 + 1));
    }

    float m_ref = -INFINITY, l_run = 0.f;
    uint32_t lost = 0;
    f32x16 o[DBLK], s[2];
#pragma unroll
    for (int b = 0; b < DBLK; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    u32x4 pf[4];

    // K(t) and V(t - 1) stand behind the barrier of tile t
    const auto scores = [&](int32_t t) {
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        uint32_t w[KK][2][4];
        float scale[KK][2];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
                const uint8_t *raw = lds_raw[t % kStages][kc * 2] + (l32 >> 4) * RAW;
                const int32_t unit = (kk * 2 + g32) * 16 + l16;
                const uint4 x = *reinterpret_cast<const uint4 *>(raw + unit * 16);
                w[kk][kc][0] = x.x; w[kk][kc][1] = x.y; w[kk][kc][2] = x.z; w[kk][kc][3] = x.w;
                scale[kk][kc] = kv4_scale(raw[F::SCALES + unit * 2]);
            }
        s[0] = s[1] = zero;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int kc = 0; kc < 2; ++kc) {
                    bf16x2 x[4];
                    kv4_decode8(w[kk][kc][m], scale[kk][kc], x);
                    const bf16x8 a = {x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
                    s[kc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kk][m], s[kc], 0, 0, 0);
                }
    };
    // the 16 keys of a record that the lane's pair sees, as bits
    const auto seen_keys = [&](int32_t tok) {
        const auto below = [](int32_t n) { return (1u << max(0, min(n, 16))) - 1u; };
        return tok < 0 ? 0u : below(pos - tok + 1) & (~below(near - tok) | below(r.sink - tok));
    };
    const auto mask = [&](int32_t st) {
        const int4 note = *reinterpret_cast<const int4 *>(key_notes[st]);
        if (__builtin_amdgcn_readfirstlane(note.x | note.y | note.z | note.w) & kSpecial) {
            const int32_t noted[NW] = {note.x, note.y, note.z, note.w};
#pragma unroll
            for (int e = 0; e < NW; ++e) {
                const uint32_t seen = seen_keys(noted[e] < 0 ? -1 : noted[e] & ~kSpecial) >> (4 * g32);
#pragma unroll
                for (int i = 0; i < 8; ++i)  // entries of keys e * 16 .. + 16 of the tile
                    s[e >> 1][(e & 1) * 8 + i] = seen >> ((i >> 2) * 8 + (i & 3)) & 1u ? s[e >> 1][(e & 1) * 8 + i] : -INFINITY;
            }
        }
    };
    const auto note_lost = [&](int32_t t) {  // of tile t, whose values stand
        const ValueNote &note = value_notes[t & 1];
        if (__builtin_amdgcn_readfirstlane(note.tile) != t) return;
        for (int e = 0; e < NW; ++e)
            for (uint64_t bad = note.nan[e]; bad; bad &= bad - 1) {
                const int32_t from = __builtin_ctzll(bad);
                if (seen_keys(note.tok[e]) >> (from & 15) & 1u) lost |= 1u << (D == 128 ? from >> 4 : from >> 5);
            }
    };
    const auto raise = [&](float psum) {
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
    };

    const auto advance = [&](int32_t t) {  // K(t) and V(t - 1) stand, V(t) goes on, tile t + 3 is on its way
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NLD) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int32_t note3 = load(t + 3);
        stage_v(t, note0);
        note0 = note1;
        note1 = note2;
        note2 = note3;
    };
    bf16x8 first[kValuesAhead];
    const auto first_values = [&](int32_t t) {
#pragma unroll
        for (int n = 0; n < kValuesAhead; ++n) first[n] = read_values<D>(lds_v[t & 1], v_at, n);
    };
    const auto last_values = [&](int32_t t) {
        first_values(t);
        note_lost(t);
        values<D, false>(lds_v[t & 1], v_at, pf, o, s, 0.f, 0.f, first);
    };
    __builtin_amdgcn_s_waitcnt(0x0F70);  // for the queries, likewise
    if (n_tiles > 0) {
        advance(0);
        if (n_w > 0) {
            scores(0);
            mask(0);
            raise(tile_weights(s, p.c_log2, reference_of(m_ref), pf));
        }
        int32_t t = 1;
        for (; t < n_w; ++t) {
            advance(t);
            scores(t);
            // of a SIMD's two wavefronts the one at its value products goes first (128 rows of 65.9 K tokens 139 -> 134.5 us, 400 of 30 K 203 -> 191.5)
            __builtin_amdgcn_s_setprio(1);
            first_values(t - 1);
            mask(t % kStages);
            note_lost(t - 1);
            raise(values<D, true>(lds_v[(t - 1) & 1], v_at, pf, o, s, p.c_log2, reference_of(m_ref), first));
            __builtin_amdgcn_s_setprio(0);
        }
        for (; t < n_tiles; ++t) {
            advance(t);
            if (t == n_w) last_values(t - 1);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (n_w == n_tiles) last_values(n_tiles - 1);
    }

    // ---- the lane's pair: elements b * 32 + i4 * 8 + g32 * 4 .. + 4
    const float l = l_run + __shfl_xor(l_run, 32);
    if (wave * 32 + l32 >= n_pairs) return;
    const int64_t slot = (int64_t)part * p.tile_pairs + wave * 32 + l32;
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
    const dim3 grid(p.grid), block(NW * 64);
    const bool few = p.num_seqs <= 64;
    if (D == 128 && few) hipLaunchKernelGGL((attn_kv4_rows_kernel<128, true>), grid, block, 0, stream, p);
    else if (D == 128) hipLaunchKernelGGL((attn_kv4_rows_kernel<128, false>), grid, block, 0, stream, p);
    else if (few) hipLaunchKernelGGL((attn_kv4_rows_kernel<64, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((attn_kv4_rows_kernel<64, false>), grid, block, 0, stream, p);
}

}  // namespace pevlm
