// Attention over the paged 4-bit KV cache (gfx950).
//
// Products run on the bf16 matrix cores: a code times its block's scale is a bf16 number exactly (v_cvt_scalef32_pk_bf16_fp4, two
// values an instruction).  Scores are formed transposed, S^T = K Q^T (v_mfma_f32_16x16x32_bf16): the wavefront-wide 16-byte load of
// a record's K codes gives a lane one block of 32 elements of one key under one scale, which is its share of the A operand if
// the k index runs over the blocks first; a lane then has four keys of one (row, head) pair in its accumulators, and the weights
// of two records are its share of the B operand of O^T += V^T P^T.  V comes by the same load, goes as bf16 through a slice of LDS of
// the wavefront's own and back transposed (ds_read_b64_tr_b16).
//
// Roundings: Q of fp32 tensors is cut into three bf16 parts that add up to it (of numbers below 2^-103 what lies under 2^-126 may be
// lost), weights are split into two (bf16 tensors, 2^-16) or three parts (fp32); products of parts are exact in fp32, sums are fp32
// throughout.  (Weights of one part save 2 %: 101 -> 99 us for 16 requests of 65.9 K tokens.)
//
// A workgroup of four wavefronts takes an item, a run of steps of 32 tokens, the wavefronts in turn; what they have is joined in LDS.  Bound by HBM
// where there are many items: 16 requests of 65.9 K tokens x 28/4 heads x 128 (577 MB) 98 us, 5.9 TB/s with both launches, 6.3 inside the kernel;
// with all codes in the caches its arithmetic takes 60 of them (vector instructions issue 61 %, matrix cores are busy 27 % of the time).  One request of 65.9 K tokens
// (36 MB) is a chain of round trips, 19.8 us with stamps in it: place (1.1), records and queries (1.7), three steps (6.2), the join (1.3), the last workgroup's
// lag (1.7), from there to the merge's start (1.9), the merge (4.4), and from its end to the next call's start (1.5).  Three workgroups a compute unit are
// enough (four 101.6 against 100.9 us, two 111), and two steps ahead are no faster than one.
#include "attn_kv4.h"

namespace pevlm {

namespace {

constexpr int NW = 4;  // wavefronts of a workgroup

// N bf16 parts of two numbers; each takes the upper 8 bits of what the parts before it leave
template <int N>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bf16x2 two = {(__bf16)a, (__bf16)b};
        part[i] = __builtin_bit_cast(uint32_t, two);
        if (i + 1 < N) {
            a -= __uint_as_float(part[i] << 16);
            b -= __uint_as_float(part[i] & 0xffff0000u);
        }
    }
}

// The same with parts cut off instead of rounded, 8 bits each: three hold all 24, numbers above bf16's largest stay finite (rounded, the first part would
// be an infinity and the second its negative), and an infinity is its own first part.
template <int N>
__device__ __forceinline__ void cut_pair(float a, float b, uint32_t (&part)[N])
{
    const auto rest = [](float x) {
        const float top = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        return top == x ? 0.f : x - top;
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u);
        a = rest(a);
        b = rest(b);
    }
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Codes that one workgroup alone reads pass by the caches: 16 requests of 65.9 K tokens 118 -> 110 us, 64 of 16 K 120 -> 109.  (Where tiles share them
// that costs 3 %.)
template <typename T, bool SHARED>
__device__ __forceinline__ T read_codes(const uint8_t *from)
{
    if constexpr (SHARED) return *reinterpret_cast<const T *>(from);
    else return __builtin_nontemporal_load(reinterpret_cast<const T *>(from));
}

constexpr float kStep = 8.f;  // base-2 units that a row's maximum may outgrow its reference by

}  // namespace

// PT: tiles of 16 pairs that share the decoded records; SHARED: whether other workgroups read the same codes; FEW: up to 64 requests
template <int D, bool BF16, int PT, bool SHARED, bool FEW>
__global__ __launch_bounds__(NW * 64, PT == 1 ? 3 : 2) void attn_kv4_kernel(Kv4Attn p)
{
    using C = Kv4Cfg<D>;
    constexpr int KS = D / 32;         // k-steps of a score
    constexpr int DT = D / 16;         // tiles of 16 elements of an output row
    constexpr int NQ = BF16 ? 1 : 3, NP = BF16 ? 2 : 3;
    constexpr int ROWB = 2 * D;        // bytes of a V row in LDS
    constexpr int WORDS = D / 32;      // words of codes of a lane: 32 (16) elements of D = 128 (64)
    static_assert(WORDS == KS, "a lane's word is its share of a k-step");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NW * 32 * ROWB];
    constexpr int PAIRS = 16 * PT;
    __shared__ float lds_ml[NW][PAIRS][2];

    have_fields(p);
    const Place at = find_place<false, FEW, SHARED>(p, blockIdx.x);
    if (at.s < 0) return;
    const Request r = at.r;
    int32_t tile, split;
    const int32_t g = divide(divide(at.rest, at.tiles, tile), at.splits, split);
    const int32_t part = at.first_part + at.rest;
    const int32_t head0 = first_head(p, g), G = heads_of(p, g);
    const int32_t pair0 = tile * PAIRS, n_pairs_all = r.rows * G;
    const int32_t n_pairs = n_pairs_all - pair0 < PAIRS ? n_pairs_all - pair0 : PAIRS;
    if (n_pairs <= 0) return;
    const Span span = span_of(r);
    const int32_t steps = steps_of(p, span), per = divide_up(steps, at.splits);
    const int32_t step0 = split * per, step1 = step0 + per < steps ? step0 + per : steps;

    const int32_t tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kg = lane >> 4;
    const int32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint8_t *const slice = lds + wave * 32 * ROWB;

    // this lane's pairs (columns of S^T)
    int32_t row[PT], head[PT], pos[PT], near[PT];
#pragma unroll
    for (int u = 0; u < PT; ++u) {
        int32_t in_row;
        row[u] = divide(pair0 + min(u * 16 + l16, n_pairs - 1), G, in_row);
        head[u] = query_head(p, head0 + in_row);
        pos[u] = r.held - r.rows + row[u];
        near[u] = near_of(r, pos[u]);
    }
    // the tile's first and last rows: positions and windows rise with the row
    const int32_t pos_lo = lane_value(pos[0], 0), pos_hi = lane_value(pos[PT - 1], 15);
    const int32_t near_lo = near_of(r, pos_lo), near_hi = near_of(r, pos_hi);

    // ---- the wavefront's records, 64 steps at a time: lane i holds those of step i of them
    uint64_t rec_off[2];
    int32_t rec_tok[2];  // first token; -1: a record that is not there
    const int32_t *const table = p.table + (int64_t)at.s * p.max_pages;
    const int32_t rec_shift = p.pool.page_shift - 4;
    const uint32_t head_bytes = (uint32_t)C::BYTES << rec_shift, page_bytes = head_bytes * p.pool.n_kv_heads, head_off = head_bytes * g;
    const auto read_records = [&](int32_t first) {  // first: the wavefront's steps before these
        const int32_t st = step0 + wave + (first + lane) * NW;
        int32_t rec[2], page[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int32_t v = st * 2 + e;
            rec[e] = st < step1 && v < span.records ? (v < span.n_sink ? v : v - span.n_sink + span.near) : -1;
            page[e] = table[(rec[e] < 0 ? 0 : rec[e]) >> rec_shift];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool there = rec[e] >= 0 && page[e] >= 0 && page[e] < p.pool.num_pages;
            rec_tok[e] = there ? rec[e] * kKv4Record : -1;
            rec_off[e] = there ? (uint64_t)(uint32_t)page[e] * page_bytes + head_off + (uint32_t)(rec[e] & ((1 << rec_shift) - 1)) * C::BYTES : 0;
        }
    };

    // The step at hand; a word's place is filled with the next step's as soon as it is used
    uint32_t k[2][WORDS], v[2][WORDS], scales[2];
    int32_t tok[2];
    // D = 128: a lane takes block kg of token l16, 16 bytes.  D = 64: half kg & 1 of block kg / 2, 8 bytes
    const uint32_t code_off = D == 128 ? lane * 16 : (kg >> 1) * 256 + l16 * 16 + (kg & 1) * 8;
    // the two scale bytes lie in one half of a word (loads of two bytes are widened where they arrive, in front of their use)
    const uint32_t scale_off = C::SCALES + ((D == 128 ? kg : kg >> 1) * 16 + (l16 & 14)) * 2, scale_bit = (l16 & 1) * 16;
    const auto codes = [&](uint32_t (&to)[WORDS], const uint8_t *from) {
        if constexpr (D == 128) {
            const u32x4 x = read_codes<u32x4, SHARED>(from);
            to[0] = x[0]; to[1] = x[1]; to[2] = x[2]; to[3] = x[3];
        } else {
            const u32x2 x = read_codes<u32x2, SHARED>(from);
            to[0] = x[0]; to[1] = x[1];
        }
    };
    const auto record = [&](int32_t e, int32_t i) {  // of the i-th of those steps
        return p.pool.base + ((uint64_t)(uint32_t)lane_value((int32_t)(rec_off[e] >> 32), i) << 32 | (uint32_t)lane_value((int32_t)rec_off[e], i));
    };
    const auto fetch_k = [&](int32_t i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint8_t *base = record(e, i);
            tok[e] = lane_value(rec_tok[e], i);
            codes(k[e], base + code_off);
            scales[e] = *reinterpret_cast<const uint32_t *>(base + scale_off);
        }
    };
    const auto fetch_v = [&](int32_t i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) codes(v[e], record(e, i) + C::CODES + code_off);
    };

    // The order of the loop, for the waits at its head: K, then V
    const auto begin = [&](int32_t first, auto between) {
        read_records(first);
        fetch_k(0);
        asm volatile("" ::: "memory");
        between();
        fetch_v(0);
    };
    bf16x8 qf[PT][NQ][KS];
    begin(0, [&] {  // the queries on the way: the lane's pair, elements kg * (D / 4) + 8 m .. + 8 of k-step m
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int64_t at_q = ((int64_t)(r.row0 + row[u]) * p.n_q_heads + head[u]) * D + kg * (D / 4);
#pragma unroll
            for (int m = 0; m < KS; ++m) {
                if constexpr (BF16) {
                    qf[u][0][m] = *reinterpret_cast<const bf16x8 *>((const uint16_t *)p.q + at_q + m * 8);
                } else {
                    const float *q = (const float *)p.q + at_q + m * 8;
                    uint32_t w[NQ][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t part[NQ];
                        cut_pair<NQ>(q[2 * i], q[2 * i + 1], part);
                        for (int n = 0; n < NQ; ++n) w[n][i] = part[n];
                    }
                    for (int n = 0; n < NQ; ++n) {
                        const uint4 v = make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]);
                        qf[u][n][m] = __builtin_bit_cast(bf16x8, v);
                    }
                }
            }
        }
    });

    float m_ref[PT], l_run[PT];
    uint32_t lost[PT];  // 32-element blocks of the pair's output that a NaN block of V reaches
    f32x4 o[PT][DT];
#pragma unroll
    for (int u = 0; u < PT; ++u) {
        m_ref[u] = -INFINITY;
        l_run[u] = 0.f;
        lost[u] = 0;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const auto compute = [&](int32_t next) {
        f32x4 s[PT][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int u = 0; u < PT; ++u) s[u][e] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float scale = kv4_scale(scales[e] >> scale_bit & 255u);
#pragma unroll
            for (int m = 0; m < KS; ++m) {
                bf16x2 x[4];
                kv4_decode8(k[e][m], scale, x);
                const bf16x8 a = {x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
#pragma unroll
                for (int u = 0; u < PT; ++u)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[u][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[u][n][m], s[u][e], 0, 0, 0);
            }
        }
        const int32_t first[2] = {tok[0], tok[1]};
        uint32_t v_scale[2] = {scales[0] >> (scale_bit + 8) & 255u, scales[1] >> (scale_bit + 8) & 255u};
        fetch_k(next);
        // ---- masks: only where some row does not see some key, or some value is NaN
        bool whole = true;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            whole = whole && first[e] >= 0 && first[e] + 15 <= pos_lo && (first[e] >= near_hi || first[e] + 15 < r.sink);
        if (!whole || __any(v_scale[0] == kKv4NanScale || v_scale[1] == kKv4NanScale)) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t tok = first[e];
                const auto sees = [&](int u, int32_t j) { return tok >= 0 && j <= pos[u] && (j >= near[u] || j < r.sink); };
#pragma unroll
                for (int u = 0; u < PT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!sees(u, tok + kg * 4 + i)) s[u][e][i] = -INFINITY;
                // the values of a key that no row sees, and NaN blocks, count as 0
                const int32_t mine = tok + l16;
                const bool seen = tok >= 0 && mine <= pos_hi && (mine >= near_lo || mine < r.sink);
                for (uint64_t bad = __ballot(seen && v_scale[e] == kKv4NanScale); bad; bad &= bad - 1) {
                    const int32_t from = __builtin_ctzll(bad);
#pragma unroll
                    for (int u = 0; u < PT; ++u)
                        if (sees(u, tok + (from & 15))) lost[u] |= 1u << (D == 128 ? from >> 4 : from >> 5);
                }
                if (!seen || v_scale[e] == kKv4NanScale) {
                    v_scale[e] = kKv4Bias;
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) v[e][w] = 0;
                }
            }
        }
        // ---- V rows to LDS
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float scale = kv4_scale(v_scale[e]);
            const int32_t t = e * 16 + l16;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                bf16x2 x[4];
                kv4_decode8(v[e][w], scale, x);
                const uint4 four = make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]),
                                              __builtin_bit_cast(uint32_t, x[3]));
                *reinterpret_cast<uint4 *>(slice + t * ROWB + value_chunk<D>(l16, kg * WORDS + w) * 16) = four;
            }
        }
        fetch_v(next);
        // ---- weights against the pair's reference, which is raised where a score outgrows it
        uint32_t pw[PT][NP][4];
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const f32x4 a = s[u][0], b = s[u][1];
            float top = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
            if (__any(top * p.c_log2 > m_ref[u] + kStep)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32)) * p.c_log2;
                if (top > m_ref[u] + kStep) {
                    const float alpha = m_ref[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref[u] - top);
                    m_ref[u] = top;
                    l_run[u] *= alpha;
#pragma unroll
                    for (int t = 0; t < DT; ++t) o[u][t] *= alpha;
                }
            }
            const float ref = m_ref[u] == -INFINITY ? 0.f : m_ref[u];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = i >> 1, j = (i & 1) * 2;
                const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e][j], p.c_log2, -ref));
                const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e][j + 1], p.c_log2, -ref));
                l_run[u] += w0 + w1;
                uint32_t part[NP];
                split_pair<NP>(w0, w1, part);
#pragma unroll
                for (int n = 0; n < NP; ++n) pw[u][n][i] = part[n];
            }
        }
        // ---- O^T += V^T P^T: k index kg * 8 + j is token kg * 4 + j of the first record, j < 4, or + j - 4 of the second
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            bf16x8 a;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t tr = kg * 4 + (l16 >> 2);
                const uint8_t *src = slice + (e * 16 + tr) * ROWB + value_chunk<D>(tr, t * 2 + ((l16 & 3) >> 1)) * 16 + (l16 & 1) * 8;
                const bf16x4 four = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, src)));
                a[e * 4] = four[0]; a[e * 4 + 1] = four[1]; a[e * 4 + 2] = four[2]; a[e * 4 + 3] = four[3];
            }
#pragma unroll
            for (int u = 0; u < PT; ++u)
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    const uint4 b = make_uint4(pw[u][n][0], pw[u][n][1], pw[u][n][2], pw[u][n][3]);
                    o[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b), o[u][t], 0, 0, 0);
                }
        }
    };

    // Loads go out on every step (behind the last the last one's again): a load under a condition makes the compiler wait for all of them where
    // the paths meet.
    const int32_t mine = step1 - step0 > wave ? (step1 - step0 - wave + NW - 1) / NW : 0;  // the wavefront's steps
    // Of the wavefronts of a SIMD the oldest is served first, and the workgroups that came last would end last, 15 % behind the first: those that are behind
    // go first (one request of 65.9 K tokens 20.3 -> 19.5 us, 64 ragged ones 65.3 -> 64.0).
    const int32_t quarter = (mine + 3) / 4;
    __builtin_amdgcn_s_setprio(3);
    for (int32_t first = 0; first < mine;) {
        const int32_t n = mine - first < 64 ? mine - first : 64;
        for (int32_t i = 0; i < n; ++i) {
            const int32_t done = first + i;
            if (done == quarter) __builtin_amdgcn_s_setprio(2);
            else if (done == 2 * quarter) __builtin_amdgcn_s_setprio(1);
            else if (done == 3 * quarter) __builtin_amdgcn_s_setprio(0);
            compute(i + 1 < n ? i + 1 : i);
        }
        first += n;
        if (first < mine) begin(first, [] {});
    }

    // ---- the wavefronts' parts of a pair: O^T to the wavefronts' slices as [pair][D] (each has 16 * D * 4 bytes), joined by all
    float *const mine_o = reinterpret_cast<float *>(slice);
    const float *const all_o = reinterpret_cast<const float *>(lds);
#pragma unroll
    for (int u = 0; u < PT; ++u) {
        if (u > 0) __syncthreads();
        l_run[u] += __shfl_xor(l_run[u], 16);
        l_run[u] += __shfl_xor(l_run[u], 32);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            if (lost[u] >> (t >> 1) & 1u) o[u][t] = f32x4{NAN, NAN, NAN, NAN};
            *reinterpret_cast<f32x4 *>(mine_o + l16 * D + t * 16 + kg * 4) = o[u][t];
        }
        if (kg == 0) {
            lds_ml[wave][u * 16 + l16][0] = m_ref[u];
            lds_ml[wave][u * 16 + l16][1] = l_run[u];
        }
        __syncthreads();
        const int32_t n = min(n_pairs - u * 16, 16);
        for (int32_t i = tid; i < n * (D / 4); i += NW * 64) {
            const int32_t at_o = i / (D / 4), pr = u * 16 + at_o, d4 = i % (D / 4) * 4;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, lds_ml[w][pr][0]);
            const float ref = M == -INFINITY ? 0.f : M;
            float l = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = __builtin_amdgcn_exp2f(lds_ml[w][pr][0] - ref);
                l += f * lds_ml[w][pr][1];
                acc += f * *reinterpret_cast<const f32x4 *>(all_o + (w * 16 + at_o) * D + d4);
            }
            if (at.splits > 1) {
                store_part<D>(p, (int64_t)part * p.tile_pairs + pr, d4, acc, M, l);
            } else {
                int32_t hh;
                const int32_t rr = divide(pair0 + pr, G, hh);
                hh = query_head(p, head0 + hh);
                store_pair<D, BF16>(p, (int64_t)(r.row0 + rr) * p.n_q_heads + hh, d4, acc, M, l);
            }
        }
    }
}

// Joins the items of the units that were cut.  WAVES wavefronts take a pair, a workgroup one (16) or two (2) pairs of a unit: D / 4 lanes cover a row of
// values and the groups of them take the items in turn, kTurn at once with their maxima and sums, against a running maximum of their own; then
// the groups are joined.  Bound by latency, 4 to 6 us: the lengths, then the parts, in one memory round trip each.  (Lanes that walk all items take a
// trip for each, 23 us for 128 items of 28 pairs, and to fetch all maxima before the first values is one trip more.)
constexpr int kTurn = 6;

template <int D, bool BF16, int WAVES, bool FEW>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void merge_kv4_kernel(Kv4Attn p)
{
    constexpr int LPR = D / 4, NSUB = WAVES * 64 / LPR, PAIRS = WAVES == 16 ? 1 : 4 / WAVES;
    __shared__ float parts[PAIRS][WAVES][D], ml[PAIRS][WAVES][2];
    have_fields(p);
    int32_t pr;
    const int32_t unit = divide(blockIdx.x, (p.tile_pairs + PAIRS - 1) / PAIRS, pr);
    const Place at = find_place<true, FEW>(p, unit);
    if (at.s < 0 || at.splits < 2) return;
    int32_t tile;
    const int32_t g = divide(at.rest, at.tiles, tile);
    const int32_t head0 = first_head(p, g), G = heads_of(p, g);
    const int32_t pair0 = tile << p.tile_shift, n_pairs = min(at.r.rows * G - pair0, 1 << p.tile_shift);
    if (pr * PAIRS >= n_pairs) return;
    const int64_t part0 = at.first_part + ((int64_t)g * at.splits) * at.tiles + tile;
    if (part0 + (int64_t)(at.splits - 1) * at.tiles >= p.max_parts) return;
    const int32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x / (WAVES * 64)), tid = threadIdx.x % (WAVES * 64);
    const int32_t in_tile = pr * PAIRS + mine, pair = pair0 + in_tile;
    const int64_t slot0 = part0 * p.tile_pairs + (in_tile < p.tile_pairs ? in_tile : p.tile_pairs - 1), stride = (int64_t)at.tiles * p.tile_pairs;
    const int32_t sub = tid / LPR, d4 = tid % LPR * 4;
    float M = -INFINITY, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int32_t s0 = sub; s0 < at.splits; s0 += NSUB * kTurn) {
        f32x4 a[kTurn];
        float2 v[kTurn];
#pragma unroll
        for (int u = 0; u < kTurn; ++u) {
            const int32_t s = s0 + u * NSUB;
            const int64_t slot = slot0 + (s < at.splits ? s : s0) * stride;
            a[u] = *reinterpret_cast<const f32x4 *>(p.part_acc + slot * D + d4);
            v[u] = *reinterpret_cast<const float2 *>(p.part_ml + slot * 2);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < kTurn; ++u) top = fmaxf(top, v[u].x);
        const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(M - ref);
        l *= old;
        acc *= old;
        M = top;
#pragma unroll
        for (int u = 0; u < kTurn; ++u)
            if (s0 + u * NSUB < at.splits) {
                const float f = __builtin_amdgcn_exp2f(v[u].x - ref);
                l += f * v[u].y;
                acc += f * a[u];
            }
    }
    // the groups of a wavefront in registers, the wavefronts through LDS
    const auto join = [&](float M2, float l2, f32x4 acc2) {
        const float top = fmaxf(M, M2), ref = top == -INFINITY ? 0.f : top;
        const float f = __builtin_amdgcn_exp2f(M - ref), f2 = __builtin_amdgcn_exp2f(M2 - ref);
        l = f * l + f2 * l2;
        acc = f * acc + f2 * acc2;
        M = top;
    };
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
        const f32x4 other = {__shfl_xor(acc[0], o), __shfl_xor(acc[1], o), __shfl_xor(acc[2], o), __shfl_xor(acc[3], o)};
        join(__shfl_xor(M, o), __shfl_xor(l, o), other);
    }
    const int32_t wave = tid >> 6;
    if ((tid & 63) < LPR) {
        *reinterpret_cast<f32x4 *>(&parts[mine][wave][d4]) = acc;
        if (d4 == 0) {
            ml[mine][wave][0] = M;
            ml[mine][wave][1] = l;
        }
    }
    __syncthreads();
    if (tid >= LPR || in_tile >= n_pairs) return;
    float Ms[WAVES], ls[WAVES];
    f32x4 as[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        Ms[w] = ml[mine][w][0];
        ls[w] = ml[mine][w][1];
        as[w] = *reinterpret_cast<const f32x4 *>(&parts[mine][w][d4]);
    }
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) M = fmaxf(M, Ms[w]);
    const float ref = M == -INFINITY ? 0.f : M;
    l = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(Ms[w] - ref);
        l += f * ls[w];
        acc += f * as[w];
    }
    int32_t in_row;
    const int32_t row = divide(pair, G, in_row), head = query_head(p, head0 + in_row);
    store_pair<D, BF16>(p, (int64_t)(at.r.row0 + row) * p.n_q_heads + head, d4, acc, M, l);
}

template <int D, bool BF16, bool FEW>
static void launch(const Kv4Attn &p, hipStream_t stream)
{
    const dim3 grid(p.grid), block(NW * 64);
    if (p.tile_shift == kKv4RowsTileShift) launch_attn_kv4_rows(p, D, stream);
    else if (p.tile_shift == kKv4TileShift && !p.shared) hipLaunchKernelGGL((attn_kv4_kernel<D, BF16, 1, false, FEW>), grid, block, 0, stream, p);
    else if (p.tile_shift == kKv4TileShift) hipLaunchKernelGGL((attn_kv4_kernel<D, BF16, 1, true, FEW>), grid, block, 0, stream, p);
    else if (!p.shared) hipLaunchKernelGGL((attn_kv4_kernel<D, BF16, 2, false, FEW>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((attn_kv4_kernel<D, BF16, 2, true, FEW>), grid, block, 0, stream, p);
    if (p.merge_grid == 0) return;
    if (p.merge_waves == 2) hipLaunchKernelGGL((merge_kv4_kernel<D, BF16, 2, FEW>), dim3(p.merge_grid), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((merge_kv4_kernel<D, BF16, 16, FEW>), dim3(p.merge_grid), dim3(1024), 0, stream, p);
}

// Up to 64 requests the lanes hold all lengths, which are read once, and the items' length is chosen among three.  With / without, 1 row of 28/4 heads x
// 128: 64 requests of 200 tokens 15.9 / 17.4 us, of 1000 24.2 / 25.3, of 16 K 106 / 120; 24 ragged ones of 32/8 heads 58.0 / 61.3; 4 rows of 64
// ragged ones 132 / 168; 100 rows of 8 240 / 263.  Without, every wavefront reads the lengths of 64 requests at a time, two or three times: 65 requests of
// 1000 tokens 27.3 us, 256 85, 1024 835.
template <int D, bool BF16>
static void launch(const Kv4Attn &p, hipStream_t stream)
{
    p.num_seqs <= 64 ? launch<D, BF16, true>(p, stream) : launch<D, BF16, false>(p, stream);
}

hipError_t launch_attn_kv4(const Kv4Attn &p, int32_t D, bool bf16, hipStream_t stream)
{
    if (D == 128) bf16 ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
    else bf16 ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
    return hipGetLastError();
}

}  // namespace pevlm
