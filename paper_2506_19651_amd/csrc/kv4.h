// The paged 4-bit KV cache: its format as the kernels see it, and what the entry points hand to them.
#pragma once
#include "common.h"

namespace pevlm {

constexpr int32_t kKv4Record = 16;                 // tokens of a record
constexpr int32_t kKv4MinExp = -100, kKv4MaxExp = 125;
constexpr int32_t kKv4Bias = 127, kKv4NanScale = 255;

template <int D>
struct Kv4Cfg {
    static constexpr int NB = D / 32;              // blocks of a token's row
    static constexpr int CODES = 8 * D;            // bytes of a record's K (or V) codes
    static constexpr int SCALES = 16 * D;          // where its scales begin
    static constexpr int BYTES = 17 * D;
};

struct Kv4Pool {
    uint8_t *base;
    int32_t num_pages, page_shift, n_kv_heads;
};

// Record of the given page, KV head and record of the page.  A pool passes 2^32 bytes.
template <int D>
__host__ __device__ inline int64_t kv4_record(const Kv4Pool &p, int32_t page, int32_t head, int32_t r)
{
    return ((((int64_t)page * p.n_kv_heads + head) << (p.page_shift - 4)) + r) * Kv4Cfg<D>::BYTES;
}

// 2^e as a float, -126 <= e <= 127
__device__ __forceinline__ float exp2_int(int32_t e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// A block's scale from its byte, as the conversion instructions take it: they read the exponent only, and make NaN of 255
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// The eight values of a word of codes, in order, as bf16: exact
__device__ __forceinline__ void kv4_decode8(uint32_t codes, float scale, bf16x2 (&x)[4])
{
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
}

struct Kv4Slots {
    const int32_t *seq_len, *new_len, *free_pages, *num_free, *pos_offset;
    int32_t *seq_len_out, *num_free_out, *row_start, *row_len, *slot_map, *pos_ids, *table;
    int32_t *first_free;  // [num_seqs] scratch: where in the list the request's first new page stands (the others before it)
    int32_t num_seqs, num_rows, max_pages, page_shift, num_pages, free_capacity;
};

struct Kv4Rows {  // rows of K and V that go into slots, or come out of them
    void *k, *v;
    int64_t k_stride, v_stride;  // elements
    const int32_t *slot_map;
    int32_t num_rows;
    Kv4Pool pool;
};

// Rows of one KV head that a wavefront takes in or out: four loads of 8 elements a lane
constexpr int32_t kv4_rows_of_wave(int32_t D) { return 4 * 64 / (D / 8); }

// Attention.  A KV head's (row, query head) pairs of a request, head fastest, are cut into tiles; a unit is one tile against all keys that
// the request's rows see, in steps of a few records.  Units are cut into items of about equal length: a workgroup takes an item.
constexpr int32_t kKv4TileShift = 4, kKv4StepShift = 1;          // 16 pairs (or twice that), 2 records: the kernel of few rows
constexpr int32_t kKv4RowsTileShift = 7, kKv4RowsStepShift = 2;  // 128 pairs, 4 records: of many

struct Kv4Heads {
    uint8_t order[kMaxHeads];         // query heads sorted by KV head
    uint16_t first[kMaxHeads + 1];    // KV head g's are order[first[g] .. first[g + 1])
};

struct Kv4Attn {
    const void *q;
    void *out;
    float *lse;
    Kv4Pool pool;
    const int32_t *table, *row_start, *row_len, *seq_len, *sink_len, *window;
    float *part_acc, *part_ml;        // [part][tile_pairs][D], [part][tile_pairs][2]: the items of units that are cut, in their order
    int32_t num_seqs, max_pages, num_rows, n_q_heads;
    int32_t tile_shift, step_shift;   // pairs of a tile, records of a step
    int32_t tile_pairs;               // pairs that a tile can have: all of a tile, or all that the rows make
    int32_t group;                    // query heads of the KV head that has most
    int32_t mapped;                   // whether a head map is given
    int32_t shared;                   // whether there may be several tiles of the same keys
    int32_t target, min_steps;        // items that a call is cut into, if they are not shorter than this
    int32_t max_items, max_units;     // bounds that no lengths pass
    int32_t max_parts;                // likewise, for which the workspace has room
    int32_t grid;                     // and one for the items that the table's width allows
    int32_t merge_waves, merge_grid;  // of the kernel that joins items: wavefronts of a pair, workgroups (0: no unit is cut)
    float c_log2;                     // softmax scale * log2(e)
    Kv4Heads heads;
};

hipError_t launch_kv4_slots(const Kv4Slots &p, hipStream_t stream);
hipError_t launch_kv4_store(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream);
hipError_t launch_kv4_load(const Kv4Rows &p, int32_t D, bool bf16, hipStream_t stream);
void launch_attn_kv4_rows(const Kv4Attn &p, int32_t D, hipStream_t stream);  // bf16 tensors
hipError_t launch_attn_kv4(const Kv4Attn &p, int32_t D, bool bf16, hipStream_t stream);

}  // namespace pevlm
