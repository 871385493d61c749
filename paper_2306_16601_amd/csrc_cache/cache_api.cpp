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
constexpr int64_t MOST_COLUMNS = (int64_t)1 << 27;      // tokens times query heads: a grid's size

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

spmm_status_t check_cache(const spmm_cache_t* c)
{
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return SPMM_E_ARG;
    if (c->type != SPMM_CACHE_BF16 && c->type != SPMM_CACHE_S8) return SPMM_E_ARG;
    if (c->type == SPMM_CACHE_S8 && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale))) return SPMM_E_ARG;
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

spmm_status_t check_attend(const spmm_cache_t* c, int64_t T, const spmm_attend_t* how)
{
    if (!how || how->max_new < 1) return SPMM_E_ARG;
    return check_heads(c, how->q_heads, T);
}

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
    if (!(how->scale > 0.0f) || !std::isfinite(how->scale) || how->window < 0) return SPMM_E_ARG;
    const int ot = how->out_type;
    if (ot != SPMM_OUT_F32 && ot != SPMM_OUT_BF16 && ot != SPMM_OUT_S8 && ot != SPMM_OUT_U8) return SPMM_E_ARG;
    const bool coded = ot == SPMM_OUT_S8 || ot == SPMM_OUT_U8;
    if (coded && (!(how->out_scale > 0.0f) || how->out_zero_point < (ot == SPMM_OUT_S8 ? -128 : 0) || how->out_zero_point > (ot == SPMM_OUT_S8 ? 127 : 255)))
        return SPMM_E_ARG;
    const int esz = ot == SPMM_OUT_F32 ? 4 : ot == SPMM_OUT_BF16 ? 2 : 1;
    if ((reinterpret_cast<uintptr_t>(out) & (esz - 1)) || ldo > (int64_t)1 << 40) return (ldo > (int64_t)1 << 40) ? SPMM_E_UNSUPPORTED : SPMM_E_ARG;
    const int64_t max_new = how->max_new < T ? how->max_new : T;
    if (batch->n_seqs > 65535 || batch->n_seqs * cache->n_heads > MOST_BLOCKS / ((max_new * (how->q_heads / cache->n_heads) + 127) / 128)) return SPMM_E_UNSUPPORTED;

    AttendArgs a = {};
    a.pool = pool_of(cache, layer);
    a.batch = batch_of(batch);
    a.q = (const __bf16*)q;
    a.out = out;
    a.work = (float*)work;
    a.ldo = ldo;
    a.T = (int32_t)T;
    a.group = how->q_heads / cache->n_heads;
    a.max_new = (int32_t)max_new;
    a.causal = how->causal != 0;
    a.window = how->window;
    a.out_type = ot;
    a.out_zero_point = coded ? how->out_zero_point : 0;
    a.scale_log2 = (float)std::min((double)how->scale * 1.4426950408889634, (double)FLT_MAX);      // (finite: a score of 0 stays 0)
    a.out_inv = coded ? 1.0f / how->out_scale : 1.0f;
    return status_of(launch_attend(a, cache->type, hip_stream));
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

}  // extern "C"
