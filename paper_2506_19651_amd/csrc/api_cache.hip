// Host side of the paged KV cache: argument validation and launches.  Entry points are documented in include/pevlm.h.
#include <string.h>

#include <algorithm>

#include "host.h"
#include "kv4.h"

namespace pevlm {

constexpr int64_t kMaxThreads = (int64_t)1 << 32;  // of a launch: fewer
constexpr int32_t kMaxRows = 1 << 30;              // a row's number and a few more fit 32 bits

constexpr int32_t kMinPage = 16, kMaxPage = 4096;
constexpr int32_t kMaxTokens = 1 << 30;  // of a request: a token's place and a tile's length add up in 32 bits

static bool page_size_ok(int32_t n) { return n >= kMinPage && n <= kMaxPage && (n & (n - 1)) == 0; }

static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

static pevlm_status check_pool(const pevlm_cache *c, Kv4Pool *pool, int32_t n_kv_heads)
{
    if (!c) return fail(PEVLM_ERR_INVALID_ARG, "cache is NULL");
    if (!page_size_ok(c->page_size)) return fail(PEVLM_ERR_INVALID_ARG, "page_size %d is not a power of two in [%d, %d]", c->page_size, kMinPage, kMaxPage);
    if (c->num_pages < 1 || (int64_t)c->num_pages * c->page_size > INT32_MAX)
        return fail(PEVLM_ERR_INVALID_ARG, "num_pages %d of %d tokens: need >= 1 page and fewer than 2^31 tokens", c->num_pages, c->page_size);
    pool->base = (uint8_t *)c->pool;
    pool->num_pages = c->num_pages;
    pool->page_shift = __builtin_ctz(c->page_size);
    pool->n_kv_heads = n_kv_heads;
    return PEVLM_OK;
}

static pevlm_status check_pool_memory(const pevlm_cache *c)
{
    if (!c->pool || !aligned16(c->pool)) return fail(PEVLM_ERR_INVALID_ARG, "the pool must be a 16-byte aligned device pointer");
    return PEVLM_OK;
}

static pevlm_status check_table(const pevlm_cache *c)
{
    if (c->num_seqs < 1 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > kMaxTokens)
        return fail(PEVLM_ERR_INVALID_ARG, "block table [%d][%d] of pages of %d tokens: need >= 1 request, >= 1 column and at most 2^30 tokens a request",
                    c->num_seqs, c->max_pages, c->page_size);
    if (!c->block_table || !aligned4(c->block_table)) return fail(PEVLM_ERR_INVALID_ARG, "block_table must be a 4-byte aligned device pointer");
    return PEVLM_OK;
}

static pevlm_status check_rows(const void *k, const void *v, int64_t k_stride, int64_t v_stride, const int32_t *slot_map, int32_t num_rows,
                               const pevlm_cache *cache, const pevlm_heads *heads, Kv4Rows *p)
{
    pevlm_status st = check_heads(heads, nullptr);
    if (st != PEVLM_OK) return st;
    st = check_pool(cache, &p->pool, heads->n_kv_heads);
    if (st != PEVLM_OK) return st;
    if (num_rows < 0) return fail(PEVLM_ERR_INVALID_ARG, "num_rows must not be negative");
    if (num_rows > kMaxRows || ((int64_t)num_rows / kv4_rows_of_wave(heads->head_dim) + 1) * heads->n_kv_heads * 64 + 256 > kMaxThreads)
        return fail(PEVLM_ERR_UNSUPPORTED, "too many rows: %d of %d heads", num_rows, heads->n_kv_heads);
    const int64_t row = (int64_t)heads->n_kv_heads * heads->head_dim;
    for (int64_t stride : {k_stride, v_stride})
        if (stride != 0 && (stride < row || stride % 8 != 0 || stride > INT32_MAX))
            return fail(PEVLM_ERR_INVALID_ARG, "row stride %lld: need 0 or a multiple of 8 of at least %lld, below 2^31", (long long)stride, (long long)row);
    if (num_rows == 0) return PEVLM_OK;
    st = check_pool_memory(cache);
    if (st != PEVLM_OK) return st;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(PEVLM_ERR_INVALID_ARG, "k and v must be 16-byte aligned device pointers");
    if (!slot_map || !aligned4(slot_map)) return fail(PEVLM_ERR_INVALID_ARG, "slot_map must be a 4-byte aligned device pointer");
    p->k = (void *)k;
    p->v = (void *)v;
    p->k_stride = k_stride ? k_stride : row;
    p->v_stride = v_stride ? v_stride : row;
    p->slot_map = slot_map;
    p->num_rows = num_rows;
    return PEVLM_OK;
}

// Query heads by KV head; returns the largest group
static int32_t group_heads(const HeadTable &tab, const pevlm_heads *h, Kv4Heads *out)
{
    int32_t most = 0, n = 0;
    for (int32_t g = 0; g < h->n_kv_heads; ++g) {
        out->first[g] = (uint16_t)n;
        while (n < h->n_q_heads && tab.kv_of_q[tab.head_order[n]] == g) ++n;
        most = std::max(most, n - out->first[g]);
    }
    out->first[h->n_kv_heads] = (uint16_t)n;
    memcpy(out->order, tab.head_order, sizeof out->order);
    return most;
}

// How a call is cut.  A request with r rows has ceil(r * group / tile) tiles of (row, query head) pairs of a KV head; tiles are of 16 pairs, of 32 in the
// same kernel, or of 128 in the kernel of many rows.  How long a request is stands on the GPU: the table's width is looked at.
enum class Cut { kTiles16, kTiles32, kTiles128 };

static int32_t asking_of(int32_t num_seqs, int32_t num_rows) { return std::max(1, std::min(num_seqs, num_rows)); }

// Workgroups of 16 pairs that a compute unit holds at a time, by registers
static int32_t resident16(const pevlm_heads *h) { return h->head_dim == 64 ? 4 : 3; }

// Tiles of 128: by the tiles of 16 and of 128 that a request's pairs fill, on average.  A tile of 128 takes the time of four of 16, of 64-wide heads of
// seven.  One request of 65.9 K tokens, 16 / 128: 28/4 heads x 128, 7 rows 33.8 / 34.6 us, 14 rows 47.1 / 41.0, 20 rows 55.1 / 55.7, 40 rows 96 / 72, 128
// rows 282 / 145; 32/8 heads 14 rows 49.6 / 50.4, 28 rows 78 / 59; 14/2 heads x 64, 18 rows 26.8 / 28.5, 128 rows 92 / 66.  Up to a few thousand
// tokens its start and longer steps do not pay (2000 tokens x 28/4, 14 rows 14.8 / 17.9, 60 rows 21.0 / 24.4, 128 rows 28.3 / 28.1).
//
// Tiles of 32 decode a record for two tiles of 16, and a unit has half as many workgroups: they pay by the steps that a workgroup of 16 would have.
// 16 / 32: 64 requests of 16 K tokens x 28/4, 4 rows (333 steps) 190 / 153 us; 16 of 65.9 K x 14/2 x 64, 4 rows (129) 62 / 53; fp32 32 rows of one of
// 65.9 K (150) 96 / 88; fp32 16 of 16 K, 4 rows (83) 65 / 64; 8 rows of one (43) 32.5 / 32.0; 4 rows of one (21) 25.0 / 26.7; 64 of 1000, 3
// rows (21) 25.8 / 32.3.
constexpr int64_t kManyRowsTokens = 4096, kTiles32Steps = 64;
static Cut cut_of(const pevlm_heads *h, int32_t group, int32_t num_seqs, int32_t num_rows, int64_t width)
{
    const int64_t asking = asking_of(num_seqs, num_rows), pairs = ((int64_t)num_rows * group + asking - 1) / asking;
    const int64_t tiles16 = (pairs + 15) / 16, tiles128 = (pairs + 127) / 128;
    if (h->dtype == PEVLM_BF16 && width >= kManyRowsTokens && tiles16 > (h->head_dim == 128 ? 4 : 7) * tiles128) return Cut::kTiles128;
    const double steps = (double)asking * tiles16 * h->n_kv_heads * (double)(width >> (4 + kKv4StepShift)) / (resident16(h) * compute_units());
    return tiles16 > 1 && steps >= kTiles32Steps ? Cut::kTiles32 : Cut::kTiles16;
}

// What bounds a call's items
static void size_attn(const pevlm_heads *h, const HeadTable &tab, int32_t num_seqs, int32_t num_rows, Cut cut, Kv4Attn *p)
{
    p->group = group_heads(tab, h, &p->heads);
    p->mapped = h->kv_head_of_q != nullptr;
    const int64_t asking = asking_of(num_seqs, num_rows), pairs = (int64_t)num_rows * p->group;
    const bool many = cut == Cut::kTiles128;
    p->tile_shift = many ? kKv4RowsTileShift : (cut == Cut::kTiles32 ? kKv4TileShift + 1 : kKv4TileShift);
    p->step_shift = many ? kKv4RowsStepShift : kKv4StepShift;
    p->tile_pairs = (int32_t)std::min<int64_t>(1 << p->tile_shift, pairs);
    // A call is one round of the workgroups that the compute units hold: a tile of 32 takes the registers of one more.  (Two rounds of shorter items are
    // 3 % slower, 16 requests of 65.9 K tokens 116.5 -> 119.4 us, four 8 %: an item's start and end, some 6 us, come twice.)
    p->target = (many ? 2 : resident16(h) - (cut == Cut::kTiles32 ? 1 : 0)) * compute_units();
    p->min_steps = many ? 4 : 8;  // 8 / 12: one request of 8000 tokens 12.5 / 13.1 us, of 30 K 15.8 / 16.7
    p->shared = pairs > asking << p->tile_shift;
    const int64_t units = h->n_kv_heads * (asking + (pairs >> p->tile_shift));
    p->max_units = (int32_t)std::min<int64_t>(units, INT32_MAX);
    p->max_items = (int32_t)std::min<int64_t>(units + p->target + 8, INT32_MAX);
    // An item's length is at least work / target, so a unit that is cut, longer than that, has at most twice its share of the target in items (and 64: what
    // sums round off).  Whole units need no room: 32768 rows of 28/4 heads x 128 in one request are 7168 of them, 480 MiB if they had.
    p->max_parts = std::min(p->max_items, 2 * p->target + 64);
}

static size_t ml_bytes(const Kv4Attn &p) { return align256((size_t)p.max_parts * p.tile_pairs * 2 * sizeof(float)); }
static size_t attn_bytes(const Kv4Attn &p, int32_t D) { return ml_bytes(p) + align256((size_t)p.max_parts * p.tile_pairs * D * sizeof(float)); }

}  // namespace pevlm

using namespace pevlm;

extern "C" {

size_t pevlm_cache_pool_bytes(const pevlm_heads *heads, int32_t num_pages, int32_t page_size)
{
    Kv4Pool pool;
    pevlm_cache c = {};
    c.num_pages = num_pages;
    c.page_size = page_size;
    if (check_heads(heads, nullptr) != PEVLM_OK || check_pool(&c, &pool, heads->n_kv_heads) != PEVLM_OK) return 0;
    return (size_t)num_pages * heads->n_kv_heads * (page_size / kKv4Record) * 17 * heads->head_dim;
}

size_t pevlm_cache_slots_workspace_bytes(int32_t num_seqs)
{
    if (num_seqs < 1) {
        fail(PEVLM_ERR_INVALID_ARG, "num_seqs must be >= 1");
        return 0;
    }
    return align256((size_t)num_seqs * sizeof(int32_t)) + 256;
}

pevlm_status pevlm_cache_slots(const pevlm_cache *cache, const int32_t *seq_len, const int32_t *new_len, const int32_t *free_pages,
                               int32_t free_capacity, const int32_t *num_free, int32_t num_rows, const int32_t *pos_offset, int32_t *seq_len_out,
                               int32_t *num_free_out, int32_t *row_start, int32_t *row_len, int32_t *slot_map, int32_t *pos_ids,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    Kv4Pool pool;
    pevlm_status st = check_pool(cache, &pool, 1);
    if (st == PEVLM_OK) st = check_table(cache);
    if (st != PEVLM_OK) return st;
    if (num_rows < 0 || free_capacity < 0) return fail(PEVLM_ERR_INVALID_ARG, "num_rows and free_capacity must not be negative");
    if (num_rows > kMaxRows) return fail(PEVLM_ERR_UNSUPPORTED, "too many rows: %d", num_rows);
    if (!seq_len || !num_free || !seq_len_out || !num_free_out || !row_start || !row_len || (!free_pages && free_capacity > 0) || (!slot_map && num_rows > 0))
        return fail(PEVLM_ERR_INVALID_ARG, "only new_len, pos_offset and pos_ids (and arrays without an entry) may be NULL");
    for (const int32_t *a : {seq_len, new_len, free_pages, num_free, pos_offset, (const int32_t *)seq_len_out, (const int32_t *)num_free_out,
                             (const int32_t *)row_start, (const int32_t *)row_len, (const int32_t *)slot_map, (const int32_t *)pos_ids})
        if (!aligned4(a)) return fail(PEVLM_ERR_INVALID_ARG, "arrays must be 4-byte aligned");
    const size_t need = (size_t)cache->num_seqs * sizeof(int32_t);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))
        return fail(PEVLM_ERR_WORKSPACE_TOO_SMALL, "slots workspace needs %zu bytes, 256-byte aligned (got %zu)",
                    pevlm_cache_slots_workspace_bytes(cache->num_seqs), workspace ? workspace_bytes : (size_t)0);
    Kv4Slots p;
    p.seq_len = seq_len; p.new_len = new_len; p.free_pages = free_pages; p.num_free = num_free; p.pos_offset = pos_offset;
    p.seq_len_out = seq_len_out; p.num_free_out = num_free_out; p.row_start = row_start; p.row_len = row_len;
    p.slot_map = slot_map; p.pos_ids = pos_ids; p.table = cache->block_table;
    p.first_free = (int32_t *)workspace;
    p.num_seqs = cache->num_seqs;
    p.num_rows = num_rows;
    p.max_pages = cache->max_pages;
    p.page_shift = pool.page_shift;
    p.num_pages = cache->num_pages;
    p.free_capacity = free_capacity;
    const hipError_t e = launch_kv4_slots(p, (hipStream_t)stream);
    return e == hipSuccess ? PEVLM_OK : hip_fail(e, "slots launch");
}

pevlm_status pevlm_cache_store_kv4(const void *k, const void *v, int64_t k_stride, int64_t v_stride, const int32_t *slot_map, int32_t num_rows,
                                   const pevlm_cache *cache, const pevlm_heads *heads, void *stream)
{
    Kv4Rows p;
    const pevlm_status st = check_rows(k, v, k_stride, v_stride, slot_map, num_rows, cache, heads, &p);
    if (st != PEVLM_OK || num_rows == 0) return st;
    const hipError_t e = launch_kv4_store(p, heads->head_dim, heads->dtype == PEVLM_BF16, (hipStream_t)stream);
    return e == hipSuccess ? PEVLM_OK : hip_fail(e, "cache store launch");
}

pevlm_status pevlm_cache_load_kv4(void *k, void *v, int64_t k_stride, int64_t v_stride, const int32_t *slot_map, int32_t num_rows,
                                  const pevlm_cache *cache, const pevlm_heads *heads, void *stream)
{
    Kv4Rows p;
    const pevlm_status st = check_rows(k, v, k_stride, v_stride, slot_map, num_rows, cache, heads, &p);
    if (st != PEVLM_OK || num_rows == 0) return st;
    const hipError_t e = launch_kv4_load(p, heads->head_dim, heads->dtype == PEVLM_BF16, (hipStream_t)stream);
    return e == hipSuccess ? PEVLM_OK : hip_fail(e, "cache load launch");
}

size_t pevlm_cache_attn_workspace_bytes(const pevlm_heads *heads, int32_t num_seqs, int32_t num_rows)
{
    if (check_heads(heads, nullptr) != PEVLM_OK) return 0;
    if (num_seqs < 1 || num_rows < 0) {
        fail(PEVLM_ERR_INVALID_ARG, "need num_seqs >= 1 and num_rows >= 0");
        return 0;
    }
    HeadTable tab;
    check_heads(heads, &tab);
    Kv4Attn p;
    size_t bytes = 0;
    // A call's cut depends on its table's width: tiles of 16 up to one, of 32 from there on, or of 128 from kManyRowsTokens on
    for (int64_t width : {(int64_t)0, kManyRowsTokens - 1, (int64_t)kMaxTokens}) {
        size_attn(heads, tab, num_seqs, num_rows, cut_of(heads, group_heads(tab, heads, &p.heads), num_seqs, num_rows, width), &p);
        bytes = std::max(bytes, attn_bytes(p, heads->head_dim));
    }
    return bytes + 256;
}

pevlm_status pevlm_cache_attn_kv4(const void *q, void *out, float *lse, const pevlm_cache *cache, const pevlm_heads *heads, int32_t num_rows,
                                  const int32_t *row_start, const int32_t *row_len, const int32_t *seq_len, const int32_t *sink_len,
                                  const int32_t *window, void *workspace, size_t workspace_bytes, void *stream)
{
    Kv4Attn p;
    memset(&p, 0, sizeof p);
    HeadTable tab;
    pevlm_status st = check_heads(heads, &tab);
    if (st == PEVLM_OK) st = check_pool(cache, &p.pool, heads->n_kv_heads);
    if (st == PEVLM_OK) st = check_table(cache);
    if (st == PEVLM_OK) st = check_pool_memory(cache);
    if (st != PEVLM_OK) return st;
    if (num_rows < 0) return fail(PEVLM_ERR_INVALID_ARG, "num_rows must not be negative");
    if (num_rows == 0) return PEVLM_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out)) return fail(PEVLM_ERR_INVALID_ARG, "q and out must be 16-byte aligned device pointers");
    if (!row_start || !row_len || !seq_len) return fail(PEVLM_ERR_INVALID_ARG, "row_start, row_len and seq_len must not be NULL");
    for (const int32_t *a : {row_start, row_len, seq_len, sink_len, window, (const int32_t *)lse})
        if (!aligned4(a)) return fail(PEVLM_ERR_INVALID_ARG, "arrays must be 4-byte aligned");
    const int64_t width = (int64_t)cache->max_pages * cache->page_size;
    size_attn(heads, tab, cache->num_seqs, num_rows, cut_of(heads, group_heads(tab, heads, &p.heads), cache->num_seqs, num_rows, width), &p);
    // no request is longer than its row of the table
    const int64_t step = kKv4Record << p.step_shift, longest = ((width + step - 1) / step + p.min_steps - 1) / p.min_steps;
    const int64_t grid = (std::min<int64_t>(p.max_items, p.max_units * longest) + 7) / 8 * 8;  // in eighths of the XCDs
    // Few units are cut into many items, whose joining is worth more wavefronts where there are few pairs, 2 / 16 of them: one request of 65.9 K tokens, 1
    // row 25.5 / 19.9 us, 2 rows 27.0 / 21.5, 8 rows 32.7 / 32.8, 40 rows 62.8 / 76.4; 4 requests 39.0 / 39.9, 16 102 / 118
    p.merge_waves = p.max_units <= 16 && p.tile_pairs <= 32 ? 16 : 2;
    const int64_t merge_grid = longest > 1 ? (int64_t)p.max_units * (p.merge_waves == 2 ? ceil_div(p.tile_pairs, 2) : p.tile_pairs) : 0;
    if (((int64_t)p.max_units << p.tile_shift) > kMaxRows || grid * 256 >= kMaxThreads || merge_grid * (p.merge_waves == 16 ? 1024 : 256) >= kMaxThreads)
        return fail(PEVLM_ERR_UNSUPPORTED, "too many rows: %d of %d heads", num_rows, heads->n_q_heads);
    const size_t need = attn_bytes(p, heads->head_dim);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))
        return fail(PEVLM_ERR_WORKSPACE_TOO_SMALL, "cache attention workspace needs %zu bytes, 256-byte aligned (got %zu)",
                    pevlm_cache_attn_workspace_bytes(heads, cache->num_seqs, num_rows), workspace ? workspace_bytes : (size_t)0);
    p.q = q; p.out = out; p.lse = lse;
    p.table = cache->block_table;
    p.row_start = row_start; p.row_len = row_len; p.seq_len = seq_len; p.sink_len = sink_len; p.window = window;
    p.num_seqs = cache->num_seqs;
    p.max_pages = cache->max_pages;
    p.num_rows = num_rows;
    p.n_q_heads = heads->n_q_heads;
    p.part_ml = (float *)workspace;
    p.grid = (int32_t)grid;
    p.merge_grid = (int32_t)merge_grid;
    p.part_acc = (float *)((char *)workspace + ml_bytes(p));
    p.c_log2 = scale_of(heads) * 1.4426950408889634f;
    const hipError_t e = launch_attn_kv4(p, heads->head_dim, heads->dtype == PEVLM_BF16, (hipStream_t)stream);
    return e == hipSuccess ? PEVLM_OK : hip_fail(e, "cache attention launch");
}

}  // extern "C"
