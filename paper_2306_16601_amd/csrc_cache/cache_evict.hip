// Tokens that stay: which ones, and the moves that bring them together.
//
// cache_evict_choose: a workgroup has the weights of a row's head of a layer in its registers (up to 32 thousand tokens) and finds the
// largest (cache_choose.h).  cache_evict_move: a workgroup moves a slice of a row's head, all of its tokens in their order.  A token never
// goes to a later place than its own, so that what a step of tokens is written over has been read, where the pages are the same ones,
// once the step itself has been read; slices (dims of keys, or of values) have nothing to do with each other.  Keys are moved 16 bytes a
// lane.  Values, whose tokens are contiguous, go page by page through LDS, 16 dims of all tokens from the next one that stays on, where those that stay are picked
// out and leave 16 bytes a lane: nearly all lines of the values are read wherever one token in sixteen stays.
//
// 8 rows of up to 12 thousand tokens in 8 bits, 8 layers of 8 heads of 128 dims, to 2048 each: 24.6 us to choose, 221 to move (772 MB read and 291 written by the counters,
// 4.8 TB/s, as a copy; without the picks it takes as long); 4 rows of 1000, 12 layers of 12 heads of 64 dims in bfloat16, to 250: 6.7 and 25.7 (98 MB read, 38 written, 5.3 TB/s
// with what the last-level cache has of it).
#include "cache_choose.h"

#include <type_traits>

namespace spmm_cache {

constexpr int MOVE_THREADS = 256;
constexpr int PIECE = 1024;         // tokens that are moved with one list of places
constexpr int EACH = PIECE / MOVE_THREADS;      // of these of a thread
constexpr int KEYS_AHEAD = 8;       // steps whose loads are under way together
constexpr int VALUE_DIMS = 16;      // of a workgroup
template <int BYTES>
constexpr int SPAN = 1024 / BYTES;  // tokens whose values are in LDS at a time

// How many tokens of a row there are, and how many stay: all of them, the first, the last.
struct Stay {
    int len, n, first, last;
};
__device__ __forceinline__ Stay stay_of(const EvictArgs& a, const int b)
{
    const Batch rows = {nullptr, a.kv_len, a.table, a.ld_table, a.n_rows};
    Stay s;
    s.len = tokens_of(rows, b, a.pool.page_shift);
    s.n = max((int)min((int64_t)min(a.keep[b], s.len), a.most), 0);
    s.first = min(a.first, s.n);
    s.last = min(a.recent, s.n - s.first);
    return s;
}

// W: waves of a row's head, REGS: values of a lane (0: any number, read again at each pass)
template <int W, int REGS>
__global__ __launch_bounds__(64 * W, (REGS > 16 ? 4 : 8)) void cache_evict_choose(const EvictArgs a)
{
    __shared__ Bins<W> bins;
    __shared__ int totals[(REGS ? REGS : 1) * W][2];
    const int H = a.pool.n_heads, h = blockIdx.x % H, layer = blockIdx.x / H, b = blockIdx.y;
    const int shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const Stay s = stay_of(a, b);
    int32_t* const kept = a.kept + (((int64_t)layer * a.n_rows + b) * H + h) * a.most;
    if (blockIdx.x == 0 && threadIdx.x == 0) a.kv_len_out[b] = s.n;
    for (int64_t i = s.n + threadIdx.x; i < a.most; i += 64 * W) kept[i] = -1;
    for (int i = threadIdx.x; i < s.first; i += 64 * W) kept[i] = i;
    for (int i = threadIdx.x; i < s.last; i += 64 * W) kept[s.n - s.last + i] = s.len - s.last + i;
    const int n = s.len - s.first - s.last, need = s.n - s.first - s.last;
    if (need == 0) return;
    const int32_t* const table = a.table + b * a.ld_table;
    const float* const weight = a.pool.weight + layer * a.layer_slots;
    const auto rank = [&](const int i) {
        const int at = s.first + i;
        return rank_of(weight[(((int64_t)page_in_pool(table[at >> shift], a.pool.n_pages) * H + h) << shift) + (at & inside)]);
    };
    const auto put = [&](const int i, const int place) { kept[s.first + place] = s.first + i; };
    if (need == n) {
        for (int i = threadIdx.x; i < n; i += 64 * W) put(i, i);
        return;
    }
    if constexpr (REGS > 0) {
        // (behind the last token its weight is loaded again: loads that may be left out come one after the other)
        uint32_t v[REGS];
#pragma unroll
        for (int k = 0; k < REGS; ++k) v[k] = rank(min(k * 64 * W + (int)threadIdx.x, n - 1));
#pragma unroll
        for (int k = 0; k < REGS; ++k) v[k] = k * 64 * W + (int)threadIdx.x < n ? v[k] : 0;
        choose<W>(v, need, bins, totals, put);
    } else {
        choose_long<W>(n, need, bins, totals, rank, put);
    }
}

// The place of a token of a row among all of a layer's, times heads; -1: nowhere.
__device__ __forceinline__ int64_t slot_of(const EvictArgs& a, const int32_t* const pages, const int h, const int at)
{
    const int shift = a.pool.page_shift, page = pages[at >> shift];
    return (uint32_t)page < (uint32_t)a.pool.n_pages ? (((int64_t)page * a.pool.n_heads + h) << shift) + (at & ((1 << shift) - 1)) : -1;
}

// What a workgroup moves: a slice of a row's head of a layer.
struct Moved {
    int slice, h, layer, b;
    Stay stay;
    const int32_t *table, *table_to, *kept;
};
__device__ __forceinline__ Moved moved(const EvictArgs& a, const int slices)
{
    Moved m;
    // (a head's slices one after the other on one XCD, which workgroups are dealt to in turn: 8 rows in 8 bits 226 us against 235 with slices side by side)
    const int heads = gridDim.x / slices, lh = blockIdx.x % heads, H = a.pool.n_heads;
    m.slice = blockIdx.x / heads;
    m.h = lh % H;
    m.layer = lh / H;
    m.b = blockIdx.y;
    m.stay = stay_of(a, m.b);
    m.table = a.table + m.b * a.ld_table;
    m.table_to = a.table_to + m.b * a.ld_table;
    m.kept = a.kept + (((int64_t)m.layer * a.n_rows + m.b) * H + m.h) * a.most;
    return m;
}

// LDS of a workgroup: a piece of the tokens, and where every 16 of them go, which lie in one page
struct ForKeys {
    int64_t from[PIECE], to[PIECE / 16];
};
template <int BYTES>
struct ForValues {
    alignas(16) char tokens[VALUE_DIMS * SPAN<BYTES> * BYTES * 5 / 4];
    alignas(16) uint16_t at[PIECE]; // where a token is in `tokens`, once its pages are there (of the first dim)
    int ids[PIECE], found;
    int64_t to[PIECE / 16];
};

// Keys: slices of the dims, 16 bytes of a token a lane; and, as the last slice, what is a number a token: weights and scales.
template <int BYTES>
__device__ __forceinline__ void move_keys(const EvictArgs& a, const Moved& m, const int slices, ForKeys& lds)
{
    int64_t *const from = lds.from, *const to = lds.to;
    const int tid = threadIdx.x, row = a.pool.head_dim * BYTES;
    const int64_t layer_slots = m.layer * a.layer_slots;
    for (int i0 = 0; i0 < m.stay.n; i0 += PIECE) {
        const int n = min(m.stay.n - i0, PIECE);
        __syncthreads();        // (the last piece has been read)
        int at[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) at[k] = m.kept[i0 + min(k * MOVE_THREADS + tid, n - 1)];
#pragma unroll
        for (int k = 0; k < EACH; ++k) from[k * MOVE_THREADS + tid] = max(slot_of(a, m.table, m.h, at[k]), (int64_t)0);
        if (tid * 16 < n) to[tid] = slot_of(a, m.table_to, m.h, i0 + tid * 16);
        __syncthreads();
        if (m.slice < slices) {
            const int per = row / 16 / slices, c = tid % per, rows = MOVE_THREADS / per, r = tid / per;
            char* const pool = (char*)a.pool.k + layer_slots * row + (m.slice * per + c) * 16;
            for (int i1 = 0; i1 < n; i1 += rows * KEYS_AHEAD) {
                u32x4 v[KEYS_AHEAD];
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) v[k] = *(const u32x4*)(pool + from[min(i1 + k * rows + r, n - 1)] * row);
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) asm volatile("" : "+v"(v[k]));       // (loads are back, not only under way, before anyone stores)
                __syncthreads();
                if (r >= rows) continue;
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) {
                    const int i = i1 + k * rows + r;
                    if (i >= n) break;
                    const int64_t slot = to[i / 16];
                    if (slot >= 0) *(u32x4*)(pool + (slot + i % 16) * row) = v[k];
                }
            }
        } else {
            float* const parts[3] = {a.pool.weight, a.pool.k_scale, a.pool.v_scale};
            for (int i1 = 0; i1 < n; i1 += MOVE_THREADS) {
                const int i = i1 + tid;
                float v[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (i < n && parts[p]) v[p] = parts[p][layer_slots + from[i]];
#pragma unroll
                for (int p = 0; p < 3; ++p) asm volatile("" : "+v"(v[p]));
                __syncthreads();
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (i < n && parts[p] && to[i / 16] >= 0) parts[p][layer_slots + to[i / 16] + i % 16] = v[p];
            }
        }
    }
}

// Values: VALUE_DIMS dims, whose tokens of a page are one run of memory.  Pages go through LDS, SPAN tokens at a time from the first that has one that
// stays; the tokens that stay are picked out there, 16 bytes of them a lane, and lanes side by side write a page's dims one after the other.
template <int BYTES>
__device__ __forceinline__ void move_values(const EvictArgs& a, const Moved& m, ForValues<BYTES>& lds)
{
    constexpr int LOADS = VALUE_DIMS * SPAN<BYTES> * BYTES / 16 / MOVE_THREADS, GROUP = 16 / BYTES, LOG = BYTES == 1 ? 4 : 3;
    using E = typename std::conditional<BYTES == 1, uint8_t, uint16_t>::type;
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    E* const tokens = (E*)lds.tokens;
    int *const ids = lds.ids, &found = lds.found;
    uint16_t* const place = lds.at;
    int64_t* const to = lds.to;
    const int tid = threadIdx.x, shift = a.pool.page_shift, inside = (1 << shift) - 1, D = a.pool.head_dim, H = a.pool.n_heads, d0 = m.slice * VALUE_DIMS;
    const int last_page = max(m.stay.len - 1, 0) >> shift;
    const int pitch = (1 << shift) + (BYTES << shift >= 64 ? GROUP : 0);       // of a dim's row in LDS, so that dims begin at different banks
    E* const pool = (E*)a.pool.v + m.layer * a.layer_slots * D;
    for (int i = tid; i < PIECE; i += MOVE_THREADS) place[i] = 0;      // (a place that is there, for tokens whose own is not known yet)
    for (int i0 = 0; i0 < m.stay.n; i0 += PIECE) {
        const int n = min(m.stay.n - i0, PIECE);
        __syncthreads();        // (the last piece has been read)
        int at[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) at[k] = m.kept[i0 + min(k * MOVE_THREADS + tid, n - 1)];
#pragma unroll
        for (int k = 0; k < EACH; ++k) ids[k * MOVE_THREADS + tid] = at[k];
        if (tid * 16 < n) {
            // (of the slice's first dim: pages hold a head's dims one after the other)
            const int64_t slot = slot_of(a, m.table_to, m.h, i0 + tid * 16);
            to[tid] = slot < 0 ? -1 : (slot >> shift << shift) * D + ((int64_t)d0 << shift) + (slot & inside);
        }
        __syncthreads();
        u32x4 v[LOADS];
        const auto load = [&](const int start) {
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int off = (k * MOVE_THREADS + tid) * GROUP, page = (start >> shift) + (off >> shift) / VALUE_DIMS;
                const int number = page_in_pool(m.table[min(page, last_page)], a.pool.n_pages);
                v[k] = *(const u32x4*)(pool + ((((int64_t)number * H + m.h) * D + d0) << shift) + (off & ((VALUE_DIMS << shift) - 1)));
            }
        };
        int start = ids[0] & ~inside;
        load(start);
        for (int begin = 0; begin < n;) {
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int off = (k * MOVE_THREADS + tid) * GROUP;
                *(u32x4*)&tokens[(off >> shift) * pitch + (off & inside)] = v[k];
            }
            for (int i = begin + tid; i < min(n, begin + SPAN<BYTES>); i += MOVE_THREADS) {
                const int at = ids[i] - start;
                if (at >= SPAN<BYTES>) break;
                place[i] = (uint16_t)((at >> shift) * VALUE_DIMS * pitch + (at & inside));
                if (i + 1 == n || ids[i + 1] - start >= SPAN<BYTES>) found = i + 1;
            }
            __syncthreads();
            // whole groups go, and the tokens behind them with the next pages, unless there is no group
            const int here = found, end = here == n || (here & ~15) <= begin ? here : here & ~15, next = end < n ? ids[end] & ~inside : start;
            if (end < n) load(next);
            // (what is stored lies before what is loaded and needed: a token goes to no later place than its own)
            const int first_page = begin >> shift, items = (((end - 1) >> shift) + 1 - first_page) << (shift - LOG + 4);
            for (int x = tid; x < items; x += MOVE_THREADS) {
                const int i = ((first_page + (x >> (shift - LOG + 4))) << shift) + (x & (inside >> LOG)) * GROUP, d = x >> (shift - LOG) & (VALUE_DIMS - 1);
                if (i >= end || i + GROUP <= begin) continue;
                const int64_t first = to[i / 16];
                if (first < 0) continue;
                // (of a group's tokens those that do not go now have another place, or none yet)
                E v[GROUP];
#pragma unroll
                for (int e = 0; e < GROUP; e += 8) {
                    const u16x8 from = *(const u16x8*)&place[i + e];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[e + j] = tokens[from[j] + d * pitch];
                }
                E* const out = pool + first + ((int64_t)d << shift) + i % 16;
                if (i >= begin && i + GROUP <= end) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = BYTES == 1 ? v[GROUP / 4 * j] | v[GROUP / 4 * j + 1] << 8 | v[GROUP / 4 * j + GROUP / 4 - 2] << 16 | (uint32_t)v[GROUP / 4 * j + GROUP / 4 - 1] << 24
                                          : v[2 * j] | (uint32_t)v[2 * j + 1] << 16;
                    *(u32x4*)out = w;
                } else {
#pragma unroll
                    for (int e = 0; e < GROUP; ++e)
                        if (i + e >= begin && i + e < end) out[e] = v[e];
                }
            }
            __syncthreads();
            begin = end;
            start = next;
        }
    }
}

// Slices of a head, each of which a workgroup moves: VALUE_DIMS dims of the values, `keys` parts of the keys' dims, weights and scales.
template <int BYTES>
__global__ __launch_bounds__(MOVE_THREADS, 5) void cache_evict_move(const EvictArgs a, const int keys)
{
    __shared__ union {
        ForKeys keys;
        ForValues<BYTES> values;
    } lds;
    const int values = a.pool.head_dim / VALUE_DIMS;
    Moved m = moved(a, values + keys + 1);
    if (m.slice < values) {
        move_values<BYTES>(a, m, lds.values);
    } else {
        m.slice -= values;
        move_keys<BYTES>(a, m, keys, lds.keys);
    }
}

int launch_evict(const EvictArgs& a, const spmm_cache_type_t type, void* stream)
{
    const int64_t most = a.ld_table << a.pool.page_shift, heads = (int64_t)a.n_layers * a.pool.n_heads;
    const dim3 rows((unsigned)heads, (unsigned)a.n_rows);
    int rc;
    // As few waves and registers as hold a row, us, 4 (32) rows of 4 layers of 8 heads: 1000 tokens with 4 registers of 4 waves 5.9 (8.4), with 16 of
    // them 7.8 (11.9); 4000 with 16 registers of 4 waves 10.1 (17), of 16 waves 12.6 (32); 8000 with 32 registers of 4 waves 16.4 (25.8), with 16 of 16 16.5 (42.6); 16000 with
    // 16 registers of 16 waves 19.8, with weights read again at each pass 58; 32000 26.7 and 146.
    if (most <= 64 * 4 * 4) rc = launch(cache_evict_choose<4, 4>, rows, dim3(64 * 4), a, stream);
    else if (most <= 64 * 4 * 16) rc = launch(cache_evict_choose<4, 16>, rows, dim3(64 * 4), a, stream);
    else if (most <= 64 * 4 * 32) rc = launch(cache_evict_choose<4, 32>, rows, dim3(64 * 4), a, stream);
    else if (most <= 64 * 16 * 16) rc = launch(cache_evict_choose<16, 16>, rows, dim3(64 * 16), a, stream);
    else if (most <= 64 * 16 * 32) rc = launch(cache_evict_choose<16, 32>, rows, dim3(64 * 16), a, stream);
    else rc = launch(cache_evict_choose<16, 0>, rows, dim3(64 * 16), a, stream);
    if (rc) return rc;
    // (keys in slices of 128 bytes where they have that many: 32 rows of 4000 tokens 393 us against 413, but 4 rows 47 against 44)
    int keys = type == SPMM_CACHE_BF16 && a.pool.head_dim == 128 ? 2 : 1;
    void* args[] = {const_cast<EvictArgs*>(&a), &keys};
    return (int)hipLaunchKernel(type == SPMM_CACHE_S8 ? (const void*)cache_evict_move<1> : (const void*)cache_evict_move<2>,
                                dim3((unsigned)(heads * (a.pool.head_dim / VALUE_DIMS + keys + 1)), (unsigned)a.n_rows), dim3(MOVE_THREADS), args, 0, (hipStream_t)stream);
}

}  // namespace spmm_cache
