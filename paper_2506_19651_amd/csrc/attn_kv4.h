// Where a workgroup's item of the cache attention lies, and what it writes: shared by the kernels over the 4-bit cache.
#pragma once
#include "bf16_device.h"
#include "kv4.h"
#include "wave_scan.h"

namespace pevlm {

constexpr int32_t kMany = 0x3fffffff;  // two of them fit 31 bits

// What a request's rows see: records (16 tokens) [0, n_sink) and [near, near + n_near), which do not overlap
struct Span {
    int32_t n_sink, near, records;
};

struct Request {
    int32_t row0, rows, held, sink;  // rows: 0 if it has none (to write)
    int32_t window;                  // < 0: none
};

__device__ __forceinline__ Request read_request(const Kv4Attn &p, int32_t s)
{
    Request r;
    const int32_t width = p.max_pages << p.pool.page_shift;  // at most 2^30
    r.row0 = p.row_start[s];
    r.rows = p.row_len[s];
    const int32_t len = p.seq_len[s];
    r.window = p.window ? p.window[s] : -1;
    r.sink = p.window && p.sink_len ? p.sink_len[s] : 0;
    r.held = len < 0 ? 0 : (len < width ? len : width);
    if (r.window < 0) r.sink = 0;
    r.sink = r.sink < 0 ? 0 : (r.sink < r.held ? r.sink : r.held);
    if (r.row0 < 0 || r.rows < 0 || r.rows > p.num_rows - r.row0) r.rows = 0;
    return r;
}

// First token inside the window of the token at position `pos`.  A row before the first token (pos < 0) sees nothing, but a tile's or a request's first
// row sets the edge for those behind it: there it is token 0's, which no later row's lies before and whose difference fits 32 bits.
__device__ __forceinline__ int32_t near_of(const Request &r, int32_t pos)
{
    const int32_t n = (int32_t)((uint32_t)max(pos, 0) - (uint32_t)r.window + 1u);
    return r.window < 0 || n < 0 ? 0 : (n < r.held ? n : r.held);
}

__device__ __forceinline__ Span span_of(const Request &r)
{
    Span s;
    const int32_t first = near_of(r, r.held - r.rows);  // of the earliest row; a row before the first token sees nothing
    s.n_sink = ceil_div(r.sink, kKv4Record);
    s.near = first / kKv4Record;
    if (s.near < s.n_sink) s.near = s.n_sink;
    const int32_t end = ceil_div(r.held, kKv4Record);
    s.records = s.n_sink + (first < r.held && end > s.near ? end - s.near : 0);
    return s;
}

__device__ __forceinline__ int32_t steps_of(const Kv4Attn &p, const Span &s) { return (s.records + (1 << p.step_shift) - 1) >> p.step_shift; }

__device__ __forceinline__ int32_t lane_value(int32_t x, int32_t lane) { return __builtin_amdgcn_readlane(x, lane); }
// a value that is the same in every lane, where the compiler is to know it
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// x / d and the rest of it, 0 <= x < 2^30, 0 < d < 2^30, without a branch: an estimate that is within 2^8 (x / d to 2^-22 of it), what that leaves by
// the same factor, to within one.  (The compiler's division is twice as long, in a chain of integer products, and a workgroup makes several
// before its first load.)
__device__ __forceinline__ int32_t divide(int32_t x, int32_t d, int32_t &rest)
{
    const float f = __builtin_amdgcn_rcpf((float)d);
    int32_t n = (int32_t)((float)x * f);
    rest = x - n * d;
    const int32_t more = (int32_t)__builtin_floorf((float)rest * f);
    n += more;
    rest -= more * d;
    const int32_t under = rest < 0, over = rest >= d;
    rest += under ? d : (over ? -d : 0);
    return n + over - under;
}
__device__ __forceinline__ int32_t divide(int32_t x, int32_t d)
{
    int32_t rest;
    return divide(x, d, rest);
}
__device__ __forceinline__ int32_t divide_up(int32_t x, int32_t d) { return divide(x + d - 1, d); }  // x + d below 2^30

// The call's fields, asked for together when a kernel begins.  The compiler asks for each where it is used, and waits there: ten waits in a row
// before the first load of a record.
__device__ __forceinline__ void have_fields(const Kv4Attn &p)
{
    asm volatile("" ::"s"(p.q), "s"(p.out), "s"(p.lse), "s"(p.pool.base), "s"(p.pool.num_pages), "s"(p.pool.page_shift), "s"(p.pool.n_kv_heads), "s"(p.table),
                 "s"(p.row_start), "s"(p.row_len), "s"(p.seq_len), "s"(p.sink_len), "s"(p.window), "s"(p.part_acc), "s"(p.part_ml), "s"(p.num_seqs),
                 "s"(p.max_pages), "s"(p.num_rows), "s"(p.n_q_heads), "s"(p.tile_pairs), "s"(p.group), "s"(p.mapped), "s"(p.target),
                 "s"(p.min_steps), "s"(p.max_items), "s"(p.max_parts), "s"(p.c_log2));
}

// Where the idx-th item (or unit) of a call lies.  Every wavefront finds its own by itself: lane by lane over 64 requests at a
// time, once for the whole work, which sets the items' length, and once for the place.  FEW: up to 64 requests, which the lanes keep; SHARED:
// contiguous eighths of the items go to the XCDs, as tiles of the same keys are neighbours.
struct Place {
    int32_t s, first_part, splits, tiles, rest;  // first_part: parts of the requests before; rest: the item's (unit's) place within the request
    Request r;
};

template <bool UNITS, bool FEW, bool SHARED = false>
__device__ __forceinline__ Place find_place(const Kv4Attn &p, int32_t idx)
{
#pragma clang fp contract(off)
    // The attention and the merge find the items' length each for itself, and must agree: every product below is rounded before it is added, which the
    // compiler would otherwise choose kernel by kernel.
    const int32_t lane = threadIdx.x & 63;
    Request r;
    int32_t steps = 0, tiles = 0;
    const auto look = [&](int32_t s) {
        steps = tiles = 0;
        if (s < p.num_seqs) {
            r = read_request(p, s);
            if (r.rows > 0) {
                tiles = (r.rows * p.group + (1 << p.tile_shift) - 1) >> p.tile_shift;  // below 2^30: the host has looked at num_rows * group
                steps = steps_of(p, span_of(r));
            }
        }
    };
    // Counts stop at kMany: with row ranges that overlap they can pass any bound, and no item or unit lies there
    const auto count = [&](int32_t n) {
        const float x = (float)n * (float)tiles * (float)p.pool.n_kv_heads;
        return x < (float)kMany ? n * tiles * p.pool.n_kv_heads : kMany;
    };
    const auto sum = [](int32_t a, int32_t b) { return min(a + b, kMany); };
    const auto total = [](auto x) { return __builtin_bit_cast(decltype(x), lane_value(__builtin_bit_cast(int32_t, x), 63)); };
    // An item's steps.  The items of all units are to be p.target: at least work / target steps; with work / (target - units) it cannot be
    // passed, whatever is lost to rounding up.  The shortest of those two and the length between them that keeps to it is taken (up to 64 requests, which
    // the lanes hold; others take the last).  What the sums round off is less than one part in 2^18, and max_items has room for that.
    float work = 0.f, units = 0.f;
    const auto plus = [](float a, float b) { return a + b; };
    for (int32_t s0 = 0; s0 < (FEW ? 1 : p.num_seqs); s0 += 64) {
        look(s0 + lane);
        work += total(wave_scan((float)steps * (float)tiles, plus));
        units += total(wave_scan((float)tiles, plus));
    }
    const float heads = (float)p.pool.n_kv_heads, target = (float)p.target, room = target - units * heads;
    const auto length = [&](float items) {
        const float x = work * heads * __builtin_amdgcn_rcpf(items);
        return max(p.min_steps, x < 1e9f ? (int32_t)x + 1 : 1000000000);
    };
    int32_t per = length(room > 0.5f * target ? room : 0.5f * target);
    if (FEW) {
        const int32_t least = length(target);
        const auto keeps = [&](int32_t n) {
            const float all = total(wave_scan((float)(steps > n ? divide_up(steps, n) : 1) * (float)tiles, plus));
            return all * heads <= target;
        };
        if (per > least) per = keeps(least) ? least : (keeps((least + per) / 2) ? (least + per) / 2 : per);
    }
    const auto splits_of = [&] { return steps > per ? divide_up(steps, per) : 1; };  // rows that see nothing are an item, too

    Place at;
    at.s = -1;
    at.first_part = 0;
    if (SHARED) {
        int32_t all = 0;
        for (int32_t s0 = 0; s0 < (FEW ? 1 : p.num_seqs); s0 += 64) {
            if (!FEW) look(s0 + lane);
            all = sum(all, total(wave_scan(count(splits_of()), sum)));
        }
        all = all < p.max_items ? all : p.max_items;
        const int32_t per_xcd = (all + 7) / 8, j = idx >> 3;
        idx = (idx & 7) * per_xcd + j;
        if (j >= per_xcd || idx >= all) return at;
    }
    int32_t before = 0;
    for (int32_t s0 = 0; s0 < (FEW ? 1 : p.num_seqs); s0 += 64) {
        if (!FEW) look(s0 + lane);
        const int32_t splits = splits_of(), items = count(splits), mine = UNITS ? count(1) : items;
        const int32_t parts = splits > 1 ? items : 0, end = wave_scan(mine, sum), part_end = wave_scan(parts, sum);
        const uint64_t found = __ballot(sum(before, end) > idx);
        if (found) {
            const int32_t f = __builtin_ctzll(found);
            at.s = s0 + f;
            at.rest = idx - before - (lane_value(end, f) - lane_value(mine, f));
            at.splits = lane_value(splits, f);
            at.tiles = lane_value(tiles, f);
            at.first_part = sum(at.first_part, lane_value(part_end, f) - lane_value(parts, f));
            // row ranges that overlap can make more parts than there is room for
            if (!UNITS && at.splits > 1 && sum(at.first_part, at.rest) >= p.max_parts) at.s = -1;
            at.r.row0 = lane_value(r.row0, f);
            at.r.rows = lane_value(r.rows, f);
            at.r.held = lane_value(r.held, f);
            at.r.sink = lane_value(r.sink, f);
            at.r.window = lane_value(r.window, f);
            return at;
        }
        before = sum(before, total(end));
        at.first_part = sum(at.first_part, total(part_end));
    }
    return at;
}

// A KV head's query heads: as a map sorts them, or equal groups in order
__device__ __forceinline__ int32_t first_head(const Kv4Attn &p, int32_t g) { return p.mapped ? p.heads.first[g] : g * p.group; }
__device__ __forceinline__ int32_t heads_of(const Kv4Attn &p, int32_t g) { return p.mapped ? p.heads.first[g + 1] - p.heads.first[g] : p.group; }
__device__ __forceinline__ int32_t query_head(const Kv4Attn &p, int32_t i) { return p.mapped ? p.heads.order[i] : i; }

__device__ __forceinline__ uint16_t bf16_nearest(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// Four elements of a pair's row, from the values and sum of its weights against reference M
template <int D, bool BF16>
__device__ __forceinline__ void store_pair(const Kv4Attn &p, int64_t to, int32_t d4, f32x4 acc, float M, float l)
{
    const bool none = M == -INFINITY && l == 0.f;  // a row that sees nothing
    acc = none ? f32x4{0.f, 0.f, 0.f, 0.f} : acc * (1.f / l);
    if constexpr (BF16) {
        const ushort4 x = make_ushort4(bf16_nearest(acc[0]), bf16_nearest(acc[1]), bf16_nearest(acc[2]), bf16_nearest(acc[3]));
        *reinterpret_cast<ushort4 *>((uint16_t *)p.out + to * D + d4) = x;
    } else {
        *reinterpret_cast<f32x4 *>((float *)p.out + to * D + d4) = acc;
    }
    if (p.lse && d4 == 0) p.lse[to] = none ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Where the 16-byte chunk c of a row of V lies in LDS.  Neighbouring rows lie in other banks both for the lanes that write a chunk of 8 rows
// each and for those that read 32 bytes of 4 rows to transpose them.
template <int D>
__device__ __forceinline__ int32_t value_chunk(int32_t row, int32_t c)
{
    return c ^ ((row & (D / 16 - 1)) << 1);
}

// A pair's part of a unit that was cut
template <int D>
__device__ __forceinline__ void store_part(const Kv4Attn &p, int64_t slot, int32_t d4, f32x4 acc, float M, float l)
{
    *reinterpret_cast<f32x4 *>(p.part_acc + slot * D + d4) = acc;
    if (d4 == 0) {
        p.part_ml[slot * 2] = M;
        p.part_ml[slot * 2 + 1] = l;
    }
}

}  // namespace pevlm
