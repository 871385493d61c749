// C ABI of the paged cache (include/spmm_cache.h): argument checks, scratch layout, launches.
#include "cache_internal.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

using namespace spmm_cache;

namespace {

constexpr int64_t TABLE_TOKENS = (int64_t)1 << 30;      // most tokens that a row of a page table may name
constexpr int64_t MOST_ROWS = (int64_t)1 << 20;         // of a page table
constexpr int64_t MOST_ENTRIES = ((int64_t)1 << 31) - 1;
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 22;       // of 128 columns, of all sequences and heads: the same
constexpr int64_t MOST_PAGES = (int64_t)1 << 20;        // of a list of pages
constexpr int64_t MOST_COLUMNS = (int64_t)1 << 27;      // tokens times query heads: a grid's size

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

spmm_status_t check_cache(const spmm_cache_t* c)
{
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return SPMM_E_ARG;
    if (c->type != SPMM_CACHE_BF16 && c->type != SPMM_CACHE_S8) return SPMM_E_ARG;
    if (c->type == SPMM_CACHE_S8 && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale))) return SPMM_E_ARG;
    if (!aligned16(c->bounds) || !aligned16(c->weight)) return SPMM_E_ARG;
    if (c->n_layers < 1 || c->n_heads < 1 || c->head_dim < 1 || c->page_tokens < 1 || c->n_pages < 1) return SPMM_E_ARG;
    if (c->head_dim > HEAD_DIM_MAX || c->head_dim % HEAD_DIM_STEP || c->page_tokens < 16 || c->page_tokens > 256 ||
        (c->page_tokens & (c->page_tokens - 1)) || c->n_pages > INT32_MAX)
        return SPMM_E_UNSUPPORTED;
    return SPMM_OK;
}

spmm_status_t check_table(const spmm_cache_t* c, int64_t ld_table, int64_t rows)
{
    if (ld_table < 1 || rows < 1) return SPMM_E_ARG;
    return ld_table >= TABLE_TOKENS / c->page_tokens || rows > MOST_ROWS || ld_table > MOST_ENTRIES / rows ? SPMM_E_UNSUPPORTED : SPMM_OK;
}

spmm_status_t check_batch(const spmm_cache_t* c, const spmm_batch_t* b)
{
    if (!b || !b->q_start || !b->kv_len || !b->table) return SPMM_E_ARG;
    return check_table(c, b->ld_table, b->n_seqs);
}

spmm_status_t check_heads(const spmm_cache_t* c, int32_t q_heads, int64_t T)
{
    if (q_heads < 1 || q_heads % c->n_heads || T < 1) return SPMM_E_ARG;
    return q_heads > 16384 || T > MOST_COLUMNS / q_heads ? SPMM_E_UNSUPPORTED : SPMM_OK;
}

Pool pool_of(const spmm_cache_t* c, int32_t layer)
{
    const int64_t slots = c->n_pages * c->n_heads * c->page_tokens * layer;
    const int64_t bytes = slots * c->head_dim * (c->type == SPMM_CACHE_S8 ? 1 : 2);
    Pool p = {};
    p.k = (char*)c->k + bytes;
    p.v = (char*)c->v + bytes;
    if (c->type == SPMM_CACHE_S8) {
        p.k_scale = c->k_scale + slots;
        p.v_scale = c->v_scale + slots;
    }
    if (c->bounds) p.bounds = (__bf16*)c->bounds + c->n_pages * c->n_heads * layer * 2 * c->head_dim;
    if (c->weight) p.weight = c->weight + slots;
    p.n_pages = (int32_t)c->n_pages;
    p.n_heads = c->n_heads;
    p.head_dim = c->head_dim;
    while (1 << p.page_shift < c->page_tokens) ++p.page_shift;
    return p;
}

Batch batch_of(const spmm_batch_t* b)
{
    return Batch{b->q_start, b->kv_len, b->table, b->ld_table, (int32_t)b->n_seqs};
}

CopyArgs copy_of(const spmm_cache_t* c)
{
    CopyArgs a = {};
    const int64_t slots = (int64_t)c->n_heads * c->page_tokens, bytes = slots * c->head_dim * (c->type == SPMM_CACHE_S8 ? 1 : 2);
    a.parts[0] = (uint4*)c->k;
    a.parts[1] = (uint4*)c->v;
    a.part_pages[0] = a.part_pages[1] = bytes / 16;
    if (c->type == SPMM_CACHE_S8) {
        a.parts[2] = (uint4*)c->k_scale;
        a.parts[3] = (uint4*)c->v_scale;
        a.part_pages[2] = a.part_pages[3] = slots * 4 / 16;
    }
    if (c->bounds) {
        a.parts[4] = (uint4*)c->bounds;
        a.part_pages[4] = (int64_t)c->n_heads * 2 * c->head_dim * 2 / 16;
    }
    if (c->weight) {
        a.parts[5] = (uint4*)c->weight;
        a.part_pages[5] = slots * 4 / 16;
    }
    a.n_layers = c->n_layers;
    a.n_pages = (int32_t)c->n_pages;
    return a;
}

// scratch of fork and compact: marks and free pages of the pool, two numbers for a row, the copies' lists, their number
struct PageScratch {
    int64_t mark, fresh, src, dst, count, bytes, most;
};
PageScratch page_scratch(const spmm_cache_t* c, int64_t rows)
{
    PageScratch s = {};
    s.most = rows > c->n_pages / 2 + 1 ? rows : c->n_pages / 2 + 1;
    s.fresh = up16(4 * c->n_pages);
    s.src = s.fresh + up16(4 * (c->n_pages + 2 * rows));
    s.dst = s.src + up16(4 * s.most);
    s.count = s.dst + up16(4 * s.most);
    s.bytes = s.count + 16;
    return s;
}

spmm_status_t status_of(int rc) { return rc == 0 ? SPMM_OK : SPMM_E_DEVICE; }

constexpr int64_t MOST_LISTS = (int64_t)1 << 22;        // columns times key/value heads: a grid's size
constexpr int64_t MOST_LISTED = (int64_t)1 << 40;       // pages of all lists together, tokens that stay of all rows
constexpr int64_t MOST_HEADS = (int64_t)1 << 20;        // of all layers

spmm_status_t check_lists(const spmm_cache_t* c, int64_t T, int64_t pages)
{
    return pages > MOST_PAGES || T * c->n_heads > MOST_LISTS || T * c->n_heads > MOST_LISTED / pages ? SPMM_E_UNSUPPORTED : SPMM_OK;
}

spmm_status_t check_selected(const spmm_cache_t* c, int64_t T, const spmm_attend_t* how, int64_t pages, int64_t* bytes)
{
    if (const spmm_status_t s = check_lists(c, T, pages)) return s;
    const int64_t n = selected_work_bytes(c->type, c->page_tokens, T, c->n_heads, how->q_heads / c->n_heads, c->head_dim, pages);
    if (n < 0) return SPMM_E_UNSUPPORTED;
    *bytes = n;
    return SPMM_OK;
}

spmm_status_t check_attend(const spmm_cache_t* c, int64_t T, const spmm_attend_t* how)
{
    if (!how || how->max_new < 1) return SPMM_E_ARG;
    return check_heads(c, how->q_heads, T);
}

// what attention is asked for, but for its sizes
spmm_status_t check_how(const spmm_attend_t* how, const void* out, int64_t ldo)
{
    if (!(how->scale > 0.0f) || !std::isfinite(how->scale) || how->window < 0) return SPMM_E_ARG;
    const int ot = how->out_type;
    if (ot != SPMM_OUT_F32 && ot != SPMM_OUT_BF16 && ot != SPMM_OUT_S8 && ot != SPMM_OUT_U8) return SPMM_E_ARG;
    if ((ot == SPMM_OUT_S8 || ot == SPMM_OUT_U8) &&
        (!(how->out_scale > 0.0f) || how->out_zero_point < (ot == SPMM_OUT_S8 ? -128 : 0) || how->out_zero_point > (ot == SPMM_OUT_S8 ? 127 : 255)))
        return SPMM_E_ARG;
    const int esz = ot == SPMM_OUT_F32 ? 4 : ot == SPMM_OUT_BF16 ? 2 : 1;
    if ((reinterpret_cast<uintptr_t>(out) & (esz - 1)) || ldo > (int64_t)1 << 40) return (ldo > (int64_t)1 << 40) ? SPMM_E_UNSUPPORTED : SPMM_E_ARG;
    return SPMM_OK;
}

float scale_log2_of(float scale) { return (float)std::min((double)scale * 1.4426950408889634, (double)FLT_MAX); }      // (finite: a score of 0 stays 0)

AttendArgs attend_of(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* q, int64_t T, const spmm_attend_t* how, void* out,
                     int64_t ldo, void* work)
{
    const bool coded = how->out_type == SPMM_OUT_S8 || how->out_type == SPMM_OUT_U8;
    AttendArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    a.q = (const __bf16*)q;
    a.out = out;
    a.work = (float*)work;
    a.ldo = ldo;
    a.T = (int32_t)T;
    a.group = how->q_heads / cache->n_heads;
    a.max_new = (int32_t)(how->max_new < T ? how->max_new : T);
    a.causal = how->causal != 0;
    a.window = how->window;
    a.out_type = how->out_type;
    a.out_zero_point = coded ? how->out_zero_point : 0;
    a.scale_log2 = scale_log2_of(how->scale);
    a.out_inv = coded ? 1.0f / how->out_scale : 1.0f;
    return a;
}

spmm_status_t check_select(const spmm_cache_t* c, int64_t T, const spmm_select_t* how)
{
    if (!how || how->pages < 1 || how->first < 0 || how->last < 0 || (int64_t)how->first + how->last > how->pages || how->window < 0) return SPMM_E_ARG;
    if (const spmm_status_t s = check_heads(c, how->q_heads, T)) return s;
    return check_lists(c, T, how->pages);
}

spmm_status_t check_weigh(const spmm_cache_t* c, int64_t T, const spmm_weigh_t* how)
{
    if (!how || how->max_new < 1 || !(how->scale > 0.0f) || !std::isfinite(how->scale) || how->window < 0 || !(how->decay >= 0.0f) || how->decay > 1.0f)
        return SPMM_E_ARG;
    return check_heads(c, how->q_heads, T);
}

// columns of a key/value head of a sequence, at most
int64_t weigh_columns(const spmm_cache_t* c, int64_t T, const spmm_weigh_t* how) { return std::min(how->max_new, T) * (how->q_heads / c->n_heads); }

}  // namespace

extern "C" {

spmm_status_t spmm_cache_append(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* x, int64_t T,
                                int64_t ldx, const spmm_append_t* how, void* q, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!how || !x || !q || !aligned16(q) || layer < 0 || layer >= cache->n_layers || ldx < T) return SPMM_E_ARG;
    if (const spmm_status_t s = check_heads(cache, how->q_heads, T)) return s;
    if (how->x_type != SPMM_OUT_F32 && how->x_type != SPMM_OUT_S8 && how->x_type != SPMM_OUT_U8) return SPMM_E_ARG;
    const bool coded = how->x_type != SPMM_OUT_F32;
    if (coded && (how->x_zero_point < (how->x_type == SPMM_OUT_S8 ? -128 : 0) || how->x_zero_point > (how->x_type == SPMM_OUT_S8 ? 127 : 255) ||
                  !(how->x_scale > 0.0f) || !std::isfinite(how->x_scale)))
        return SPMM_E_ARG;
    if (!(how->eps >= 0.0f) || !std::isfinite(how->eps)) return SPMM_E_ARG;
    if (how->rope && (how->rope_dim < 2 || how->rope_dim % 2 || how->rope_dim > cache->head_dim || how->rope_len < 1)) return SPMM_E_ARG;
    if (ldx > (int64_t)1 << 40) return SPMM_E_UNSUPPORTED;

    AppendArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    a.x = x;
    a.q = (__bf16*)q;
    a.q_weight = how->q_weight;
    a.k_weight = how->k_weight;
    a.rope = how->rope;
    a.positions = how->positions;
    a.ldx = ldx;
    a.rope_len = how->rope_len;
    a.T = (int32_t)T;
    a.q_heads = how->q_heads;
    a.x_zero_point = coded ? how->x_zero_point : 0;
    a.rope_dim = how->rope ? how->rope_dim : 0;
    a.interleaved = how->interleaved != 0;
    a.x_scale = coded ? how->x_scale : 1.0f;
    a.eps = how->eps;
    return status_of(launch_append(a, how->x_type, cache->type, hip_stream));
}

spmm_status_t spmm_attend_work_bytes(const spmm_cache_t* cache, int64_t n_seqs, int64_t T, const spmm_attend_t* how, int64_t* bytes)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!bytes || n_seqs < 1) return SPMM_E_ARG;
    if (const spmm_status_t s = check_attend(cache, T, how)) return s;
    const int64_t max_new = how->max_new < T ? how->max_new : T;
    *bytes = attend_work_bytes(cache->type, n_seqs, cache->n_heads, how->q_heads / cache->n_heads, cache->head_dim, max_new);
    return SPMM_OK;
}

spmm_status_t spmm_cache_attend(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* q, int64_t T,
                                const spmm_attend_t* how, void* out, int64_t ldo, void* work, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!q || !out || !work || !aligned16(q) || !aligned16(work) || layer < 0 || layer >= cache->n_layers || ldo < T) return SPMM_E_ARG;
    if (const spmm_status_t s = check_attend(cache, T, how)) return s;
    if (const spmm_status_t s = check_how(how, out, ldo)) return s;
    const int64_t max_new = how->max_new < T ? how->max_new : T;
    if (batch->n_seqs > 65535 || batch->n_seqs * cache->n_heads > MOST_BLOCKS / ((max_new * (how->q_heads / cache->n_heads) + 127) / 128)) return SPMM_E_UNSUPPORTED;
    return status_of(launch_attend(attend_of(cache, layer, batch, q, T, how, out, ldo, work), cache->type, hip_stream));
}

spmm_status_t spmm_cache_work_bytes(const spmm_cache_t* cache, int64_t n_rows, int64_t* bytes)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!bytes || n_rows < 1) return SPMM_E_ARG;
    if (n_rows > MOST_ROWS) return SPMM_E_UNSUPPORTED;
    *bytes = page_scratch(cache, n_rows).bytes;
    return SPMM_OK;
}

spmm_status_t spmm_cache_fork(const spmm_cache_t* cache, const int32_t* table, int64_t ld_table, const int32_t* kv_len, int64_t n_rows_in,
                              const int32_t* parent, const int32_t* keep, const int32_t* want, int64_t n_rows, int32_t* table_out,
                              int32_t* kv_len_out, int32_t* info, void* work, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!table || !kv_len || !parent || !keep || !want || !table_out || !kv_len_out || !info || !work || !aligned16(work)) return SPMM_E_ARG;
    if (table_out == table || kv_len_out == kv_len) return SPMM_E_ARG;
    if (const spmm_status_t s = check_table(cache, ld_table, n_rows_in)) return s;
    if (const spmm_status_t s = check_table(cache, ld_table, n_rows)) return s;

    const PageScratch p = page_scratch(cache, n_rows);
    char* const w = (char*)work;
    ForkArgs a = {};
    a.table = table;
    a.kv_len = kv_len;
    a.parent = parent;
    a.keep = keep;
    a.want = want;
    a.table_out = table_out;
    a.kv_len_out = kv_len_out;
    a.info = info;
    a.mark = (int32_t*)(w + p.mark);
    a.fresh = (int32_t*)(w + p.fresh);
    a.src = (int32_t*)(w + p.src);
    a.dst = (int32_t*)(w + p.dst);
    a.count = (int32_t*)(w + p.count);
    a.ld_table = ld_table;
    a.rows_in = (int32_t)n_rows_in;
    a.rows = (int32_t)n_rows;
    a.n_pages = (int32_t)cache->n_pages;
    a.page_shift = pool_of(cache, 0).page_shift;
    CopyArgs c = copy_of(cache);
    c.src = a.src;
    c.dst = a.dst;
    c.count = a.count;
    c.most = (int32_t)n_rows;       // (a row copies one page at most)
    return status_of(launch_fork(a, c, hip_stream));
}

spmm_status_t spmm_cache_compact(const spmm_cache_t* cache, const int32_t* table, int64_t ld_table, int64_t n_rows, int32_t* table_out,
                                 int32_t* info, void* work, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!table || !table_out || !info || !work || !aligned16(work)) return SPMM_E_ARG;
    if (const spmm_status_t s = check_table(cache, ld_table, n_rows)) return s;

    const PageScratch p = page_scratch(cache, n_rows);
    char* const w = (char*)work;
    CompactArgs a = {};
    a.table = table;
    a.table_out = table_out;
    a.info = info;
    a.mark = (int32_t*)(w + p.mark);
    a.src = (int32_t*)(w + p.src);
    a.dst = (int32_t*)(w + p.dst);
    a.count = (int32_t*)(w + p.count);
    a.entries = n_rows * ld_table;
    a.n_pages = (int32_t)cache->n_pages;
    CopyArgs c = copy_of(cache);
    c.src = a.src;
    c.dst = a.dst;
    c.count = a.count;
    const int64_t half = cache->n_pages / 2;        // (holes and pages behind them are as many, and no page is both)
    c.most = (int32_t)(half < a.entries ? half > 1 ? half : 1 : a.entries);
    return status_of(launch_compact(a, c, hip_stream));
}

spmm_status_t spmm_cache_copy(const spmm_cache_t* cache, const int32_t* src, const int32_t* dst, int64_t n, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (n < 0 || (n && (!src || !dst))) return SPMM_E_ARG;
    if (n > INT32_MAX) return SPMM_E_UNSUPPORTED;
    if (n == 0) return SPMM_OK;
    CopyArgs c = copy_of(cache);
    c.src = src;
    c.dst = dst;
    c.most = (int32_t)n;
    return status_of(launch_copy(c, hip_stream));
}

spmm_status_t spmm_cache_bounds(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, int64_t T, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!cache->bounds || layer < 0 || layer >= cache->n_layers || T < 1) return SPMM_E_ARG;
    if (batch->n_seqs > 65535) return SPMM_E_UNSUPPORTED;
    BoundsArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    return status_of(launch_bounds(a, cache->type, std::min(T, MOST_COLUMNS), hip_stream));
}

spmm_status_t spmm_cache_score(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* q, int64_t T,
                               const spmm_select_t* how, float* scores, int64_t lds, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!cache->bounds || !q || !aligned16(q) || !scores || (reinterpret_cast<uintptr_t>(scores) & 3) || layer < 0 || layer >= cache->n_layers || lds < batch->ld_table)
        return SPMM_E_ARG;
    if (const spmm_status_t s = check_select(cache, T, how)) return s;
    if (lds > (int64_t)1 << 30) return SPMM_E_UNSUPPORTED;
    ScoreArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    a.q = (const __bf16*)q;
    a.scores = scores;
    a.lds = lds;
    a.T = (int32_t)T;
    a.group = how->q_heads / cache->n_heads;
    a.causal = how->causal != 0;
    a.window = how->window;
    return status_of(launch_score(a, hip_stream));
}

spmm_status_t spmm_cache_select(const spmm_cache_t* cache, const spmm_batch_t* batch, const float* scores, int64_t T, int64_t lds,
                                const spmm_select_t* how, int32_t* lists, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!scores || !lists || (reinterpret_cast<uintptr_t>(scores) & 3) || (reinterpret_cast<uintptr_t>(lists) & 3) || lds < batch->ld_table) return SPMM_E_ARG;
    if (const spmm_status_t s = check_select(cache, T, how)) return s;
    if (lds > (int64_t)1 << 30) return SPMM_E_UNSUPPORTED;
    SelectArgs a = {};
    a.batch = batch_of(batch);
    a.scores = scores;
    a.lists = lists;
    a.lds = lds;
    a.T = (int32_t)T;
    a.n_heads = cache->n_heads;
    a.page_shift = pool_of(cache, 0).page_shift;
    a.pages = how->pages;
    a.first = how->first;
    a.last = how->last;
    a.causal = how->causal != 0;
    a.window = how->window;
    return status_of(launch_select(a, hip_stream));
}

spmm_status_t spmm_selected_work_bytes(const spmm_cache_t* cache, int64_t T, const spmm_attend_t* how, int64_t pages, int64_t* bytes)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!bytes || pages < 1) return SPMM_E_ARG;
    if (const spmm_status_t s = check_attend(cache, T, how)) return s;
    return check_selected(cache, T, how, pages, bytes);
}

spmm_status_t spmm_cache_attend_selected(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* q, int64_t T,
                                         const spmm_attend_t* how, const int32_t* lists, int64_t pages, void* out, int64_t ldo, void* work,
                                         void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!q || !out || !work || !lists || !aligned16(q) || !aligned16(work) || (reinterpret_cast<uintptr_t>(lists) & 3) || layer < 0 || layer >= cache->n_layers ||
        ldo < T || pages < 1)
        return SPMM_E_ARG;
    if (const spmm_status_t s = check_attend(cache, T, how)) return s;
    if (const spmm_status_t s = check_how(how, out, ldo)) return s;
    int64_t bytes;
    if (const spmm_status_t s = check_selected(cache, T, how, pages, &bytes)) return s;
    SelectedArgs a = {};
    a.attend = attend_of(cache, layer, batch, q, T, how, out, ldo, work);
    a.lists = lists;
    a.pages = (int32_t)pages;
    return status_of(launch_attend_selected(a, cache->type, hip_stream));
}

spmm_status_t spmm_weigh_work_bytes(const spmm_cache_t* cache, const spmm_batch_t* batch, int64_t T, const spmm_weigh_t* how, int64_t* bytes)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!bytes || !batch) return SPMM_E_ARG;
    if (const spmm_status_t s = check_table(cache, batch->ld_table, batch->n_seqs)) return s;
    if (const spmm_status_t s = check_weigh(cache, T, how)) return s;
    if (batch->n_seqs > 65535) return SPMM_E_UNSUPPORTED;
    *bytes = weigh_work_bytes(cache->page_tokens, cache->n_pages, batch->n_seqs, batch->ld_table, cache->n_heads, weigh_columns(cache, T, how), T * how->q_heads);
    return SPMM_OK;
}

spmm_status_t spmm_cache_weigh(const spmm_cache_t* cache, int32_t layer, const spmm_batch_t* batch, const void* q, int64_t T,
                               const spmm_weigh_t* how, void* work, void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (const spmm_status_t s = check_batch(cache, batch)) return s;
    if (!cache->weight || !q || !work || !aligned16(q) || !aligned16(work) || layer < 0 || layer >= cache->n_layers) return SPMM_E_ARG;
    if (const spmm_status_t s = check_weigh(cache, T, how)) return s;
    if (batch->n_seqs > 65535) return SPMM_E_UNSUPPORTED;
    WeighArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    a.q = (const __bf16*)q;
    a.work = (float*)work;
    a.T = (int32_t)T;
    a.group = how->q_heads / cache->n_heads;
    a.max_new = (int32_t)std::min(how->max_new, T);
    a.causal = how->causal != 0;
    a.window = how->window;
    a.scale_log2 = scale_log2_of(how->scale);
    a.decay = how->decay;
    return status_of(launch_weigh(a, cache->type, hip_stream));
}

spmm_status_t spmm_cache_evict(const spmm_cache_t* cache, const int32_t* table, int64_t ld_table, const int32_t* kv_len, int64_t n_rows,
                               const int32_t* keep, const spmm_evict_t* how, const int32_t* table_to, int32_t* kv_len_out, int32_t* kept,
                               void* hip_stream)
{
    if (const spmm_status_t s = check_cache(cache)) return s;
    if (!cache->weight || !table || !kv_len || !keep || !how || !table_to || !kv_len_out || !kept || kv_len_out == kv_len) return SPMM_E_ARG;
    if (how->first < 0 || how->recent < 0 || how->most < 1) return SPMM_E_ARG;
    if (const spmm_status_t s = check_table(cache, ld_table, n_rows)) return s;
    const int64_t heads = (int64_t)cache->n_layers * cache->n_heads;
    if (n_rows > 65535 || heads > MOST_HEADS || how->most > TABLE_TOKENS || how->most > (MOST_LISTED / n_rows) / heads) return SPMM_E_UNSUPPORTED;
    EvictArgs a = {};
    a.pool = pool_of(cache, 0);
    a.table = table;
    a.kv_len = kv_len;
    a.keep = keep;
    a.table_to = table_to;
    a.kv_len_out = kv_len_out;
    a.kept = kept;
    a.ld_table = ld_table;
    a.most = how->most;
    a.layer_slots = cache->n_pages * cache->n_heads * cache->page_tokens;
    a.n_rows = (int32_t)n_rows;
    a.n_layers = cache->n_layers;
    a.first = how->first;
    a.recent = how->recent;
    return status_of(launch_evict(a, cache->type, hip_stream));
}

}  // extern "C"
