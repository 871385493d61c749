// Which pages a new token reads: the first, the last, and those of the highest scores, in ascending order (cache_choose.h).
//
// A wave has a row of up to 1024 pages in its registers; longer ones take a workgroup, and those of more than 32 thousand pages are read
// again at each pass.  Reading the scores once would take 13 us for 16000 rows of 970 of them; it takes 21.1:
// 600 vector instructions a row are 15 us of it.
#include "cache_choose.h"

namespace spmm_cache {

constexpr int SMALL_WAVES = 4;      // of a workgroup of rows that take a wave each

// What a row chooses from.
struct Row {
    int first, pages;       // visible pages
    int from, n, need;      // of those that are not taken anyway: the first one, how many, how many of them are taken
    int head;               // taken before them
    const float* scores;
    int32_t* list;
};

// false: a column of no sequence
__device__ __forceinline__ bool row_of(const SelectArgs& a, const int i, Row* const r)      // (there are at most 2^22)
{
    const int t = i / a.n_heads, b = sequence_near(a.batch, t);
    if (b < 0) return false;
    const Span s = span_of(a.batch, b, t, a.page_shift, a.causal, a.window);
    r->first = s.from <= s.to ? s.from >> a.page_shift : 0;
    r->pages = s.from <= s.to ? (s.to >> a.page_shift) - r->first + 1 : 0;
    r->head = a.first;
    r->from = r->first + a.first;
    r->n = r->pages - a.first - a.last;
    r->need = a.pages - a.first - a.last;
    r->scores = a.scores + (int64_t)i * a.lds;
    r->list = a.lists + (int64_t)i * a.pages;
    return true;
}

// All of a short row's pages are taken.
__device__ __forceinline__ bool all_of(const SelectArgs& a, const Row& r, const int at, const int step)
{
    if (r.pages > a.pages) return false;
    for (int i = at; i < a.pages; i += step) r.list[i] = i < r.pages ? r.first + i : -1;
    return true;
}

// Those that are taken whatever their scores are.
__device__ __forceinline__ void ends_of(const SelectArgs& a, const Row& r, const int at, const int step)
{
    for (int i = at; i < a.first; i += step) r.list[i] = r.first + i;
    for (int i = at; i < a.last; i += step) r.list[a.pages - a.last + i] = r.first + r.pages - a.last + i;
}

// Ranks of a row's scores, those of a thread.  (Behind the last score it is loaded again: loads that may be left out come one after the other.)
template <int WAVES, int REGS>
__device__ __forceinline__ void ranks_of(const Row& r, const int thread, uint32_t (&v)[REGS])
{
    float x[REGS];
#pragma unroll
    for (int k = 0; k < REGS; ++k) x[k] = r.scores[r.from + min(k * 64 * WAVES + thread, r.n - 1)];
#pragma unroll
    for (int k = 0; k < REGS; ++k) v[k] = k * 64 * WAVES + thread < r.n ? rank_of(x[k]) : 0;
}

template <int REGS>
__global__ __launch_bounds__(64 * SMALL_WAVES) void cache_select(const SelectArgs a)
{
    __shared__ Bins<1> bins[SMALL_WAVES];
    const int lane = threadIdx.x % 64, i = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * SMALL_WAVES + threadIdx.x / 64));
    Row r;
    if (i >= a.T * a.n_heads || !row_of(a, i, &r) || all_of(a, r, lane, 64)) return;
    ends_of(a, r, lane, 64);
    if (r.need == 0) return;
    uint32_t v[REGS];
    ranks_of<1>(r, lane, v);
    choose<1>(v, r.need, bins[threadIdx.x / 64], (int (*)[2])nullptr, [&](const int j, const int place) { r.list[r.head + place] = r.from + j; });
}

template <int WAVES, int REGS>
__global__ __launch_bounds__(64 * WAVES) void cache_select_long(const SelectArgs a)
{
    __shared__ Bins<WAVES> bins;
    __shared__ int totals[(REGS ? REGS : 1) * WAVES][2];
    for (int i = blockIdx.x; i < a.T * a.n_heads; i += gridDim.x) {
        Row r;
        if (!row_of(a, i, &r) || all_of(a, r, threadIdx.x, 64 * WAVES)) continue;
        ends_of(a, r, threadIdx.x, 64 * WAVES);
        if (r.need == 0) continue;
        const auto put = [&](const int j, const int place) { r.list[r.head + place] = r.from + j; };
        __syncthreads();        // (the last row's counts have been read)
        if constexpr (REGS > 0) {
            uint32_t v[REGS];
            ranks_of<WAVES>(r, threadIdx.x, v);
            choose<WAVES>(v, r.need, bins, totals, put);
        } else {
            choose_long<WAVES>(r.n, r.need, bins, totals, [&](const int j) { return rank_of(r.scores[r.from + j]); }, put);
        }
    }
}

int launch_select(const SelectArgs& a, void* stream)
{
    const int64_t rows = (int64_t)a.T * a.n_heads, most = a.batch.ld_table;
    const unsigned grid = (unsigned)(rows < 1 << 20 ? rows : 1 << 20);
    const dim3 small((unsigned)((rows + SMALL_WAVES - 1) / SMALL_WAVES)), threads(64 * SMALL_WAVES);
    // As few waves as hold a row, 64 / 4096 rows, us: 1000 pages by a wave 6.5 / 9.2, by four 8.2 / 33; 4000 pages by four 8.9 / 36, by sixteen 15 / 215; 8000 by four
    // with 32 registers 11.6 / 66, by sixteen 15.2 / 219; 16000 by sixteen with 16 registers 11.3 / 163, with 32 15.5 / 221; 30000 with the row in registers 15.8,
    // without 47.
    if (most <= 128) return launch(cache_select<2>, small, threads, a, stream);
    if (most <= 256) return launch(cache_select<4>, small, threads, a, stream);
    if (most <= 512) return launch(cache_select<8>, small, threads, a, stream);
    if (most <= 1024) return launch(cache_select<16>, small, threads, a, stream);
    if (most <= 4096) return launch(cache_select_long<4, 16>, dim3(grid), dim3(256), a, stream);
    if (most <= 8192) return launch(cache_select_long<4, 32>, dim3(grid), dim3(256), a, stream);
    if (most <= 16384) return launch(cache_select_long<16, 16>, dim3(grid), dim3(1024), a, stream);
    if (most <= 32768) return launch(cache_select_long<16, 32>, dim3(grid), dim3(1024), a, stream);
    return launch(cache_select_long<16, 0>, dim3(grid), dim3(1024), a, stream);
}

}  // namespace spmm_cache
