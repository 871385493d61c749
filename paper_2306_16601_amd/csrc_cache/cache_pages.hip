// Which pages belong to which sequence: forking, trimming, freeing and growing in one call, compacting, and the copies.
//
// What a page table says is worked out by one workgroup (a table of 64 sequences of 16 thousand tokens is 64 KB), in
// passes over the table and over a mark for each page; the pages that have to move are then copied by the whole device,
// which reads and writes them once: memory bounds it (500 pages of 12 layers, 1.2 GB: 239 us, 4.9 TB/s, what a large copy
// reaches; the tables 8 us before that).  The lists of copies and their number stay on the device.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int THREADS = 1024;
constexpr int COPY_THREADS = 256;
constexpr int PIECE = 1024;         // 16-byte units that a workgroup copies at a time
constexpr int COPY_GRID = 2048;     // workgroups: 8 on each of 256 CUs

// marks of a page: 0 free, USED in the old table, TAIL_TOP - row kept tokens of that row (the lowest) end inside, WHOLE kept
// as a whole
constexpr int32_t USED = 1, WHOLE = 0x7fffffff, TAIL_TOP = 0x7ffffffe;

// Marks lie in LDS where they fit: a pass over global ones takes a microsecond or two to be seen by the next.
constexpr int LDS_PAGES = 16384, LDS_ROWS = 1024;
extern __shared__ int32_t lds[];

template <bool LDS>
struct Marks {
    int32_t* at;
    __device__ __forceinline__ int32_t read(const int p) const { return LDS ? at[p] : __hip_atomic_load(at + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
    __device__ __forceinline__ void write(const int p, const int32_t v) const
    {
        if (LDS) at[p] = v;
        else __hip_atomic_store(at + p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __device__ __forceinline__ void raise(const int p, const int32_t v) const
    {
        if (LDS) __hip_atomic_fetch_max(at + p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        else __hip_atomic_fetch_max(at + p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
};

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

// LDS: marks of the pages, and of up to LDS_ROWS rows what they keep
template <bool LDS>
__global__ __launch_bounds__(THREADS) void cache_fork(const ForkArgs a)
{
    const int tid = threadIdx.x, shift = a.page_shift, inside = (1 << shift) - 1;
    const uint32_t width = (uint32_t)a.ld_table, entries_in = (uint32_t)a.rows_in * width, entries = (uint32_t)a.rows * width;
    __shared__ int too_wide;
    __shared__ Kept rows[LDS_ROWS];
    const Marks<LDS> mark = {LDS ? lds : a.mark};
    const bool few_rows = a.rows <= LDS_ROWS;
    const auto kept = [&](const int j) { return few_rows ? rows[j] : kept_of(a, j); };
    if (tid == 0) too_wide = 0;
    for (int p = tid; p < a.n_pages; p += THREADS) mark.write(p, 0);
    if (few_rows && tid < a.rows) rows[tid] = kept_of(a, tid);
    __syncthreads();
    for (uint32_t e = tid; e < entries_in; e += THREADS) {
        const int p = a.table[e];
        if ((uint32_t)p < (uint32_t)a.n_pages) mark.raise(p, USED);
    }
    for (uint32_t e = tid; e < entries; e += THREADS) {
        const int j = (int)(e / width), i = (int)(e % width);
        const Kept k = kept(j);
        if (k.too_many) too_wide = 1;
        if (k.row < 0 || i > (k.tokens - 1) >> shift) continue;
        const int p = a.table[k.row * a.ld_table + i];
        if ((uint32_t)p >= (uint32_t)a.n_pages) continue;
        mark.raise(p, i < k.tokens >> shift ? WHOLE : TAIL_TOP - j);
    }
    __syncthreads();

    // new pages and copies of each row
    int need = 0, copies = 0;
    for (int j0 = 0; j0 < a.rows; j0 += THREADS) {
        const int j = j0 + tid;
        int fresh = 0, copy = 0;
        if (j < a.rows) {
            const Kept k = kept(j);
            if (k.tokens & inside) {
                const int p = a.table[k.row * a.ld_table + (k.tokens >> shift)];
                copy = (uint32_t)p < (uint32_t)a.n_pages && mark.read(p) != TAIL_TOP - j;
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
        const int p = p0 + tid, m = p < a.n_pages ? mark.read(p) : USED;
        int all, all_stay;
        const int at = found + before(m == 0, &all);
        before(m > USED, &all_stay);
        if (m == 0 && at < need) free_pages[at] = p;
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
    for (uint32_t e = tid; e < entries; e += THREADS) {
        const int j = (int)(e / width), i = (int)(e % width);
        const Kept k = kept(j);
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

template <bool LDS>
__global__ __launch_bounds__(THREADS) void cache_compact(const CompactArgs a)
{
    const int tid = threadIdx.x;
    const Marks<LDS> mark = {LDS ? lds : a.mark};
    for (int p = tid; p < a.n_pages; p += THREADS) mark.write(p, 0);
    __syncthreads();
    for (int64_t e = tid; e < a.entries; e += THREADS) {
        const int p = a.table[e];
        if ((uint32_t)p < (uint32_t)a.n_pages) mark.raise(p, USED);
    }
    __syncthreads();
    int used = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
        int all;
        before(p0 + tid < a.n_pages && mark.read(p0 + tid), &all);
        used += all;
    }
    // the i-th page in use behind the front goes to the i-th hole in it
    int holes = 0, late = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
        const int p = p0 + tid;
        const bool is = p < a.n_pages && mark.read(p);
        const bool hole = p < used && !is, moves = p >= used && is;
        int all_holes, all_late;
        const int at_hole = holes + before(hole, &all_holes), at_late = late + before(moves, &all_late);
        if (hole) a.dst[at_hole] = p;
        if (moves) {
            a.src[at_late] = p;
            mark.write(p, USED + 1 + at_late);
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
            const int m = mark.read(p);
            if (m > USED) p = a.dst[m - USED - 1];
        }
        a.table_out[e] = p;
    }
}

__global__ __launch_bounds__(COPY_THREADS) void cache_copy_pages(const CopyArgs a)
{
    const int64_t count = a.count ? min(*a.count, a.most) : a.most;
    uint32_t pieces[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += pieces[i] = a.parts[i] ? (uint32_t)((a.part_pages[i] + PIECE - 1) / PIECE) : 0;
    const int64_t all = count * a.n_layers * sum;
    for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
        // (page, layer, piece): in 32 bits where they suffice
        uint32_t piece, layer;
        int64_t pair;
        if (all >> 32) {
            pair = w / sum / a.n_layers;
            layer = (uint32_t)(w / sum % a.n_layers);
            piece = (uint32_t)(w % sum);
        } else {
            const uint32_t page = (uint32_t)w / sum;
            piece = (uint32_t)w % sum;
            pair = page / (uint32_t)a.n_layers;
            layer = page % (uint32_t)a.n_layers;
        }
        const int src = a.src[pair], dst = a.dst[pair];
        int64_t units = a.part_pages[0];
        u32x4* part = (u32x4*)a.parts[0];
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (part == (u32x4*)a.parts[i] && piece >= pieces[i]) {
                piece -= pieces[i];
                part = (u32x4*)a.parts[i + 1];
                units = a.part_pages[i + 1];
            }
        if ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages) continue;
        const u32x4* const from = part + ((int64_t)layer * a.n_pages + src) * units + piece * (int64_t)PIECE + threadIdx.x;
        u32x4* const to = part + ((int64_t)layer * a.n_pages + dst) * units + piece * (int64_t)PIECE + threadIdx.x;
        const int64_t left = units - piece * (int64_t)PIECE - threadIdx.x;
        if (units - piece * (int64_t)PIECE >= PIECE) {
            u32x4 v[PIECE / COPY_THREADS];
#pragma unroll
            for (int i = 0; i < PIECE / COPY_THREADS; ++i) v[i] = from[i * COPY_THREADS];
#pragma unroll
            for (int i = 0; i < PIECE / COPY_THREADS; ++i) to[i * COPY_THREADS] = v[i];
        } else {
            for (int i = 0; i < left; i += COPY_THREADS) to[i] = from[i];
        }
    }
}

int launch_copy(const CopyArgs& a, void* stream)
{
    int64_t pieces = 0;
    for (int i = 0; i < 4; ++i) pieces += a.parts[i] ? (a.part_pages[i] + PIECE - 1) / PIECE : 0;
    const int64_t all = a.most * a.n_layers * pieces;
    return launch(cache_copy_pages, dim3((unsigned)(all < COPY_GRID ? all : COPY_GRID)), dim3(COPY_THREADS), a, stream);
}

template <typename A>
static int launch_tables(void (*in_lds)(A), void (*in_memory)(A), const A& a, const CopyArgs& c, void* stream)
{
    const bool fits = a.n_pages <= LDS_PAGES;
    void* args[] = {const_cast<A*>(&a)};
    const int rc = (int)hipLaunchKernel(fits ? (const void*)in_lds : (const void*)in_memory, dim3(1), dim3(THREADS), args, fits ? 4 * (size_t)a.n_pages : 0, (hipStream_t)stream);
    return rc ? rc : launch_copy(c, stream);
}

int launch_fork(const ForkArgs& a, const CopyArgs& c, void* stream) { return launch_tables(cache_fork<true>, cache_fork<false>, a, c, stream); }
int launch_compact(const CompactArgs& a, const CopyArgs& c, void* stream) { return launch_tables(cache_compact<true>, cache_compact<false>, a, c, stream); }

}  // namespace spmm_cache
