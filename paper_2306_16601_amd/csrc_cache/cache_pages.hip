// Which pages belong to which sequence: forking, trimming, freeing and growing in one call, compacting, and the copies.
//
// What a page table says is worked out by one workgroup (a table of 64 sequences of 16 thousand tokens is 64 KB), in
// passes over the table and over a mark for each page; the pages that have to move are then copied by the whole device,
// which reads and writes them once: memory bounds it.  The lists of copies and their number stay on the device.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int THREADS = 1024;
constexpr int COPY_THREADS = 256;
constexpr int PIECE = 1024;         // 16-byte units that a workgroup copies at a time

// marks of a page: 0 free, USED in the old table, TAIL + (most - row) kept tokens of that row (the lowest) end inside,
// WHOLE kept as a whole
constexpr int32_t USED = 1, WHOLE = 0x7fffffff, TAIL_TOP = 0x7ffffffe;

__device__ __forceinline__ int32_t read_mark(const int32_t* p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void raise_mark(int32_t* p, const int32_t v)
{
    __hip_atomic_fetch_max(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sum of v over the threads before this one; *all: over all of them.  Every thread of the workgroup calls it.
__device__ int before(const int v, int* const all)
{
    __shared__ int waves[THREADS / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int s = v;
    for (int i = 1; i < 64; i <<= 1) {
        const int o = __shfl_up(s, i);
        if (lane >= i) s += o;
    }
    __syncthreads();        // (the last call's sums have been read)
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int base = 0, sum = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) base += waves[w];
        sum += waves[w];
    }
    *all = sum;
    return base + s - v;
}

struct Kept {
    int row, tokens, pages;     // of the old table: its row (-1: none), tokens kept, pages wanted in all
    bool too_many;              // more than the table is wide
};

__device__ __forceinline__ Kept kept_of(const ForkArgs& a, const int j)
{
    Kept k = {-1, 0, 0, false};
    const int p = a.parent[j];
    const int64_t most = a.ld_table << a.page_shift;
    if (p >= 0 && p < a.rows_in) {
        k.row = p;
        k.tokens = (int)min((int64_t)max(min(a.keep[j], a.kv_len[p]), 0), most);
    }
    const int room = max(k.tokens, a.want[j]);
    k.pages = (int)(((int64_t)room + (1 << a.page_shift) - 1) >> a.page_shift);
    k.too_many = k.pages > a.ld_table;
    if (k.too_many) k.pages = (int)a.ld_table;
    return k;
}

__global__ __launch_bounds__(THREADS) void cache_fork(const ForkArgs a)
{
    const int tid = threadIdx.x, shift = a.page_shift, inside = (1 << shift) - 1;
    __shared__ int too_wide;
    if (tid == 0) too_wide = 0;
    for (int p = tid; p < a.n_pages; p += THREADS) __hip_atomic_store(a.mark + p, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int64_t e = tid; e < a.rows_in * a.ld_table; e += THREADS) {
        const int p = a.table[e];
        if ((uint32_t)p < (uint32_t)a.n_pages) raise_mark(a.mark + p, USED);
    }
    for (int64_t e = tid; e < a.rows * a.ld_table; e += THREADS) {
        const int j = (int)(e / a.ld_table), i = (int)(e % a.ld_table);
        const Kept k = kept_of(a, j);
        if (k.too_many) too_wide = 1;
        if (k.row < 0 || i > (k.tokens - 1) >> shift) continue;
        const int p = a.table[k.row * a.ld_table + i];
        if ((uint32_t)p >= (uint32_t)a.n_pages) continue;
        raise_mark(a.mark + p, i < k.tokens >> shift ? WHOLE : TAIL_TOP - j);
    }
    __syncthreads();

    // new pages and copies of each row
    int need = 0, copies = 0;
    for (int j0 = 0; j0 < a.rows; j0 += THREADS) {
        const int j = j0 + tid;
        int fresh = 0, copy = 0;
        if (j < a.rows) {
            const Kept k = kept_of(a, j);
            if (k.tokens & inside) {
                const int p = a.table[k.row * a.ld_table + (k.tokens >> shift)];
                copy = (uint32_t)p < (uint32_t)a.n_pages && read_mark(a.mark + p) != TAIL_TOP - j;
            }
            fresh = copy + k.pages - ((k.tokens + inside) >> shift);
        }
        int all, all_copies;
        const int at = before(fresh, &all), at_copy = before(copy, &all_copies);
        if (j < a.rows) {
            a.fresh[2 * j] = need + at;
            a.fresh[2 * j + 1] = copy ? copies + at_copy : -1;
        }
        need += all;
        copies += all_copies;
    }
    // the lowest free pages
    int32_t* const free_pages = a.fresh + 2 * a.rows;
    int found = 0, stay = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
        const int p = p0 + tid, mark = p < a.n_pages ? read_mark(a.mark + p) : USED;
        int all, all_stay;
        const int at = found + before(mark == 0, &all);
        before(mark > USED, &all_stay);
        if (mark == 0 && at < need) free_pages[at] = p;
        found += all;
        stay += all_stay;
    }
    __syncthreads();
    const int missing = need > found ? need - found : 0;
    const bool go = !missing && !too_wide;
    if (tid == 0) {
        a.info[0] = missing ? missing : too_wide ? 1 : 0;
        a.info[1] = go ? copies : 0;
        a.info[2] = go ? stay + need : 0;
        a.info[3] = 0;
        *a.count = go ? copies : 0;
    }
    if (!go) return;
    for (int64_t e = tid; e < a.rows * a.ld_table; e += THREADS) {
        const int j = (int)(e / a.ld_table), i = (int)(e % a.ld_table);
        const Kept k = kept_of(a, j);
        const int whole = k.tokens >> shift, held = (k.tokens + inside) >> shift, at = a.fresh[2 * j], copy = a.fresh[2 * j + 1];
        int p = -1;
        if (i < held) p = a.table[k.row * a.ld_table + i];
        if (i == whole && i < held && copy >= 0) {
            a.src[copy] = p;
            a.dst[copy] = p = free_pages[at];
        }
        if (i >= held && i < k.pages) p = free_pages[at + (copy >= 0) + i - held];
        a.table_out[e] = p;
        if (i == 0) a.kv_len_out[j] = k.tokens;
    }
}

__global__ __launch_bounds__(THREADS) void cache_compact(const CompactArgs a)
{
    const int tid = threadIdx.x;
    for (int p = tid; p < a.n_pages; p += THREADS) __hip_atomic_store(a.mark + p, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int64_t e = tid; e < a.entries; e += THREADS) {
        const int p = a.table[e];
        if ((uint32_t)p < (uint32_t)a.n_pages) raise_mark(a.mark + p, USED);
    }
    __syncthreads();
    int used = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
        int all;
        before(p0 + tid < a.n_pages && read_mark(a.mark + p0 + tid), &all);
        used += all;
    }
    // the i-th page in use behind the front goes to the i-th hole in it
    int holes = 0, late = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
        const int p = p0 + tid;
        const bool is = p < a.n_pages && read_mark(a.mark + p);
        const bool hole = p < used && !is, moves = p >= used && is;
        int all_holes, all_late;
        const int at_hole = holes + before(hole, &all_holes), at_late = late + before(moves, &all_late);
        if (hole) a.dst[at_hole] = p;
        if (moves) {
            a.src[at_late] = p;
            __hip_atomic_store(a.mark + p, USED + 1 + at_late, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        holes += all_holes;
        late += all_late;
    }
    __syncthreads();
    if (tid == 0) {
        a.info[0] = 0;
        a.info[1] = late;
        a.info[2] = used;
        a.info[3] = 0;
        *a.count = late;
    }
    for (int64_t e = tid; e < a.entries; e += THREADS) {
        int p = a.table[e];
        if ((uint32_t)p < (uint32_t)a.n_pages) {
            const int mark = read_mark(a.mark + p);
            if (mark > USED) p = a.dst[mark - USED - 1];
        }
        a.table_out[e] = p;
    }
}

__global__ __launch_bounds__(COPY_THREADS) void cache_copy_pages(const CopyArgs a)
{
    const int64_t count = a.count ? min(*a.count, a.most) : a.most;
    int64_t pieces[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += pieces[i] = a.parts[i] ? (a.part_pages[i] + PIECE - 1) / PIECE : 0;
    const int64_t all = count * a.n_layers * sum;
    for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
        const int64_t page = w / sum, layer = page % a.n_layers;
        int64_t piece = w % sum, units = a.part_pages[0];
        uint4* part = a.parts[0];
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (part == a.parts[i] && piece >= pieces[i]) {
                piece -= pieces[i];
                part = a.parts[i + 1];
                units = a.part_pages[i + 1];
            }
        const int src = a.src[page / a.n_layers], dst = a.dst[page / a.n_layers];
        if ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages) continue;
        const uint4* const from = part + (layer * a.n_pages + src) * units;
        uint4* const to = part + (layer * a.n_pages + dst) * units;
        uint4 v[PIECE / COPY_THREADS];
#pragma unroll
        for (int i = 0; i < PIECE / COPY_THREADS; ++i) {
            const int64_t u = piece * PIECE + i * COPY_THREADS + threadIdx.x;
            if (u < units) v[i] = from[u];
        }
#pragma unroll
        for (int i = 0; i < PIECE / COPY_THREADS; ++i) {
            const int64_t u = piece * PIECE + i * COPY_THREADS + threadIdx.x;
            if (u < units) to[u] = v[i];
        }
    }
}

int launch_copy(const CopyArgs& a, void* stream)
{
    return launch(cache_copy_pages, dim3(2048), dim3(COPY_THREADS), a, stream);
}

int launch_fork(const ForkArgs& a, const CopyArgs& c, void* stream)
{
    const int rc = launch(cache_fork, dim3(1), dim3(THREADS), a, stream);
    return rc ? rc : launch_copy(c, stream);
}

int launch_compact(const CompactArgs& a, const CopyArgs& c, void* stream)
{
    const int rc = launch(cache_compact, dim3(1), dim3(THREADS), a, stream);
    return rc ? rc : launch_copy(c, stream);
}

}  // namespace spmm_cache
