// Declarations shared by the paged cache's host glue (cache_api.cpp) and its kernels; the public interface is
// include/spmm_cache.h.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "spmm_cache.h"

namespace spmm_cache {

constexpr int HEAD_DIM_MAX = 128;
constexpr int HEAD_DIM_STEP = 16;

// one layer of a cache, as kernels take it
struct Pool {
    void *k, *v;
    float *k_scale, *v_scale;
    __bf16* bounds;
    float* weight;
    int32_t n_pages, n_heads, head_dim, page_shift;
};

struct Batch {
    const int32_t *q_start, *kv_len, *table;
    int64_t ld_table;
    int32_t n_seqs;
};

struct AppendArgs {
    Pool pool;
    Batch batch;
    const void* x;
    __bf16* q;
    const float *q_weight, *k_weight, *rope;
    const int32_t* positions;
    int64_t ldx, rope_len;
    int32_t T, q_heads, x_zero_point, rope_dim, interleaved;
    float x_scale, eps;
};

struct AttendArgs {
    Pool pool;
    Batch batch;
    const __bf16* q;
    void* out;
    float* work;
    int64_t ldo;
    int32_t T, group, max_new, causal, window, out_type, out_zero_point;
    float scale_log2, out_inv;      // scale * log2(e); 1 / out_scale
};

constexpr int PARTS = 6;

// pages of all layers that are copied: src[i] -> dst[i], i < *count
struct CopyArgs {
    uint4* parts[PARTS];            // keys, values and their scales, bounds, weights; nullptr where there are none
    int64_t part_pages[PARTS];      // 16-byte units of a page in that part
    const int32_t *src, *dst, *count;
    int64_t n_layers;
    int32_t n_pages, most;          // most: bound of *count (and the number where count is nullptr)
};

struct ForkArgs {
    const int32_t *table, *kv_len, *parent, *keep, *want;
    int32_t *table_out, *kv_len_out, *info;
    int32_t *mark, *fresh, *src, *dst, *count;      // scratch: per page; per row; copies
    int64_t ld_table;
    int32_t rows_in, rows, n_pages, page_shift;
};

struct CompactArgs {
    const int32_t* table;
    int32_t *table_out, *info;
    int32_t *mark, *src, *dst, *count;
    int64_t entries;                // of the table
    int32_t n_pages;
};

struct BoundsArgs {
    Pool pool;
    Batch batch;
};

struct ScoreArgs {
    Pool pool;
    Batch batch;
    const __bf16* q;
    float* scores;
    int64_t lds;
    int32_t T, group, causal, window;
};

struct SelectArgs {
    Batch batch;
    const float* scores;
    int32_t* lists;
    int64_t lds;
    int32_t T, n_heads, page_shift, pages, first, last, causal, window;
};

struct SelectedArgs {
    AttendArgs attend;
    const int32_t* lists;
    int32_t pages, parts;           // of a list; workgroups that share one
};

struct WeighArgs {
    Pool pool;
    Batch batch;
    const __bf16* q;
    float* work;
    int32_t* owner;                 // scratch, of each page (nullptr: one sequence): a row that names it, ~ of it where another one does too
    int32_t T, group, max_new, causal, window, parts, keep;
    float scale_log2, decay;
};

struct EvictArgs {
    Pool pool;                      // of the first layer
    const int32_t *table, *kv_len, *keep, *table_to;
    int32_t *kv_len_out, *kept;
    int64_t ld_table, most, layer_slots;        // layer_slots: tokens of a layer's pages, times heads
    int32_t n_rows, n_layers, first, recent;
};

// launches; a HIP status
int launch_append(const AppendArgs& a, spmm_out_t x_type, spmm_cache_type_t type, void* stream);
int launch_attend(const AttendArgs& a, spmm_cache_type_t type, void* stream);
int launch_attend_few(const AttendArgs& a, spmm_cache_type_t type, void* stream);
int64_t few_work_bytes(int64_t n_seqs, int dim, int64_t cols);
int launch_attend_many(const AttendArgs& a, spmm_cache_type_t type, void* stream);
int64_t many_work_bytes(spmm_cache_type_t type, int64_t n_seqs, int n_heads, int dim, int64_t cols);
int64_t attend_work_bytes(spmm_cache_type_t type, int64_t n_seqs, int32_t n_heads, int32_t group, int32_t head_dim, int64_t max_new);
int launch_copy(const CopyArgs& a, void* stream);
int launch_bounds(const BoundsArgs& a, spmm_cache_type_t type, int64_t T, void* stream);
int launch_score(const ScoreArgs& a, void* stream);
int launch_select(const SelectArgs& a, void* stream);
// -1: more parts of lists than a grid holds
int64_t selected_work_bytes(spmm_cache_type_t type, int page_tokens, int64_t T, int n_heads, int group, int dim, int64_t pages);
int launch_attend_selected(const SelectedArgs& a, spmm_cache_type_t type, void* stream);
int64_t weigh_work_bytes(int page_tokens, int64_t n_pages, int64_t n_seqs, int64_t ld_table, int n_heads, int64_t cols, int64_t columns);
int launch_weigh(const WeighArgs& a, spmm_cache_type_t type, void* stream);
int launch_evict(const EvictArgs& a, spmm_cache_type_t type, void* stream);
int launch_fork(const ForkArgs& a, const CopyArgs& c, void* stream);
int launch_compact(const CompactArgs& a, const CopyArgs& c, void* stream);

template <typename A>
inline int launch(void (*kernel)(A), dim3 grid, dim3 block, const A& a, void* stream)
{
    void* args[] = {const_cast<A*>(&a)};
    return (int)hipLaunchKernel((const void*)kernel, grid, block, args, 0, (hipStream_t)stream);
}

#if defined(__HIPCC__)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The sequence that column t belongs to: the last b with q_start[b] <= t (there may be empty ones before it).
// -1 where t lies before the first or behind the last.
__device__ __forceinline__ int sequence_of(const Batch& s, const int t)
{
    int lo = 0, hi = s.n_seqs;      // the first b with q_start[b] > t lies in [lo, hi], or there is none below n_seqs + 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s.q_start[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo < s.n_seqs && t >= s.q_start[lo] ? lo : -1;
}

// The same, which looks first where t is if every sequence has one new token.
__device__ __forceinline__ int sequence_near(const Batch& s, const int t)
{
    const int b = t < s.n_seqs ? t : s.n_seqs - 1;
    return s.q_start[b] <= t && t < s.q_start[b + 1] ? b : sequence_of(s, t);
}

// Tokens of a sequence that its table can name (a table's row names less than 2^30: cache_api.cpp).
__host__ __device__ __forceinline__ int tokens_of(const Batch& s, const int b, const int page_shift)
{
    const int64_t most = s.ld_table << page_shift;
    const int n = s.kv_len[b];
    return n < 0 ? 0 : (int64_t)n < most ? n : (int)most;
}

// The tokens that a column sees: from .. to of its sequence's row (none: from > to).
struct Span {
    int from, to;
};
__host__ __device__ __forceinline__ Span span_of(const Batch& s, const int b, const int t, const int page_shift, const int causal, const int window)
{
    const int len = tokens_of(s, b, page_shift);
    const int64_t at = (int64_t)s.kv_len[b] - ((int64_t)s.q_start[b + 1] - t);
    if (at < 0 || len == 0) return Span{0, -1};
    Span r;
    r.to = causal && at < len ? (int)at : len - 1;
    const int64_t from = window ? at + 1 - window : 0;
    r.from = from <= 0 ? 0 : from < len ? (int)from : len;
    return r;
}

// A page number that lies in the pool, whatever the table holds.
__device__ __forceinline__ int page_in_pool(const int page, const int n_pages)
{
    return (uint32_t)page < (uint32_t)n_pages ? page : 0;
}

#endif

}  // namespace spmm_cache
