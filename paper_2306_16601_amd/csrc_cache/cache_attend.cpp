// Which attention kernel a call takes.
#include "cache_internal.h"

namespace spmm_cache {

// Columns of a key/value head (query heads that share it times new tokens) up to which the cache is read straight to registers.
// At 32 columns, 8 heads of 128 dims, that way against tiles in LDS: one sequence of 2000 keys 16.5 / 31.2 us, 8 of 30000 179 /
// 194, in 8 bits 121 / 220, 32 of 500 18.1 / 27.2; its registers hold no more columns.
constexpr int64_t FEW = 32;

int64_t attend_work_bytes(spmm_cache_type_t type, int64_t n_seqs, int32_t n_heads, int32_t group, int32_t head_dim, int64_t max_new)
{
    return max_new * group <= FEW ? few_work_bytes(n_seqs, head_dim, max_new * group) : many_work_bytes(type, n_seqs, n_heads, head_dim, max_new * group);
}

int launch_attend(const AttendArgs& a, spmm_cache_type_t type, void* stream)
{
    return (int64_t)a.max_new * a.group <= FEW ? launch_attend_few(a, type, stream) : launch_attend_many(a, type, stream);
}

}  // namespace spmm_cache
