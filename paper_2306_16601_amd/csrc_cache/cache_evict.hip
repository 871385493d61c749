// Tokens that stay: which ones, and the moves that bring them together.
//
// cache_evict_choose: a workgroup has the weights of a row's head of a layer in its registers (up to 32 thousand tokens) and finds the
// largest (cache_choose.h).  cache_evict_move: a workgroup moves a slice of a row's head, all of its tokens in their order.  A token never
// goes to a later place than its own, so that what a piece of tokens is written over has been read, where the pages are the same ones,
// once the piece itself has been read by all; slices (dims of keys, or of values) have nothing to do with each other.  Keys are moved 16 bytes a
// lane; values, whose tokens are contiguous, are gathered token by token, as their tokens are chosen one by one, and written 16 bytes
// a lane.
#include "cache_choose.h"

#include <type_traits>

namespace spmm_cache {

constexpr int CHOOSE_WAVES = 16, CHOOSE_REGS = 32;
constexpr int MOVE_THREADS = 256;

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

template <int REGS>
__global__ __launch_bounds__(64 * CHOOSE_WAVES) void cache_evict_choose(const EvictArgs a)
{
    constexpr int W = CHOOSE_WAVES;
    __shared__ int counts[2 * W], totals[(REGS ? REGS : 1) * W][2];
    const int H = a.pool.n_heads, h = blockIdx.x % H, layer = blockIdx.x / H, b = blockIdx.y;
    const int shift = a.pool.page_shift, inside = (1 << shift) - 1, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
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
        uint32_t v[REGS];
#pragma unroll
        for (int k = 0; k < REGS; ++k) {
            const int i = (k * W + wave) * 64 + lane;
            v[k] = i < n ? rank(i) : 0;
        }
        const Border border = border_of<W>(v, need, counts);
        put_chosen<W>(v, border, totals, put);
    } else {
        choose_long<W>(n, need, counts, totals, rank, put);
    }
}

// Slices of a head: KEYS of its keys' dims, VALUES of its values', one of what is a number a token (scales, weights).
template <spmm_cache_type_t TYPE>
__global__ __launch_bounds__(MOVE_THREADS) void cache_evict_move(const EvictArgs a, const int slices)
{
    constexpr int BYTES = TYPE == SPMM_CACHE_S8 ? 1 : 2, EACH = 16 / BYTES;      // elements of 16 bytes
    const int H = a.pool.n_heads, D = a.pool.head_dim, shift = a.pool.page_shift, inside = (1 << shift) - 1, tid = threadIdx.x;
    const int slice = blockIdx.x % slices, lh = blockIdx.x / slices, h = lh % H, layer = lh / H, b = blockIdx.y;
    const Stay s = stay_of(a, b);
    if (s.n == 0) return;
    const int32_t *const table = a.table + b * a.ld_table, *const table_to = a.table_to + b * a.ld_table;
    const int32_t* const kept = a.kept + (((int64_t)layer * a.n_rows + b) * H + h) * a.most;
    const int64_t layer_slots = layer * a.layer_slots;
    // the place of a token among all of the layer's; -1: nowhere
    const auto place = [&](const int32_t* const pages, const int at) {
        const int page = pages[at >> shift];
        return (uint32_t)page < (uint32_t)a.pool.n_pages ? (((int64_t)page * H + h) << shift) + (at & inside) : (int64_t)-1;
    };
    // in place, the first tokens that stay are where they are already
    const int sides = (slices - 1) / 2;
    if (slice < sides) {
        // keys: a lane moves 16 bytes of a token
        const int per = D / EACH / sides, c = tid % per, rows = MOVE_THREADS / per, r = tid / per;
        u32x4* const pool = (u32x4*)((char*)a.pool.k + layer_slots * D * BYTES) + slice * per + c;
        const int unit = D / EACH;
        constexpr int AHEAD = 4;
        for (int i0 = 0; i0 < s.n; i0 += rows * AHEAD) {
            u32x4 v[AHEAD] = {};
            int64_t to[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = i0 + k * rows + r;
                to[k] = -1;
                if (r < rows && i < s.n) {
                    const int64_t from = place(table, kept[i]);
                    to[k] = place(table_to, i);
                    if (from == to[k]) to[k] = -1;
                    if (to[k] >= 0) v[k] = pool[(from < 0 ? 0 : from) * unit];
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) asm volatile("" : "+v"(v[k]));       // (loads are back, not only under way, before anyone stores)
            __syncthreads();
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (to[k] >= 0) pool[to[k] * unit] = v[k];
        }
    } else if (slice < 2 * sides) {
        // values: a lane moves EACH tokens of a dim
        const int dims = D / sides, d0 = (slice - sides) * dims;
        char* const pool = (char*)a.pool.v + layer_slots * D * BYTES;
        using E = typename std::conditional<TYPE == SPMM_CACHE_S8, uint8_t, uint16_t>::type;
        // (the place of dim d of a token whose slot, among those of its head, is known: pages hold dims in rows)
        const auto value_at = [&](const int64_t slot, const int d) { return ((E*)pool) + (slot >> shift << shift) * D + ((int64_t)d << shift) + (slot & inside); };
        const int groups = (s.n + EACH - 1) / EACH;
        const int lanes = min(MOVE_THREADS, 64);
        for (int g0 = 0; g0 < groups; g0 += lanes) {
            const int g = g0 + tid % lanes, i0 = g * EACH;
            int64_t from[EACH];
            const bool mine = g < groups;
            int64_t to = -1;
            if (mine) {
                to = place(table_to, i0);       // (EACH tokens are in one page)
#pragma unroll
                for (int e = 0; e < EACH; ++e) from[e] = i0 + e < s.n ? place(table, kept[i0 + e]) : -1;
            }
            for (int d = d0 + tid / lanes; d < d0 + dims; d += MOVE_THREADS / lanes) {
                E v[EACH];
                if (mine && to >= 0) {
#pragma unroll
                    for (int e = 0; e < EACH; ++e) v[e] = from[e] >= 0 ? *value_at(from[e], d) : (E)0;
                }
                // (a wave has a dim's tokens, and later pieces of it: its loads are back before it stores)
                if (mine && to >= 0) {
                    E* const out = value_at(to, d);
                    if (i0 + EACH <= s.n) {
                        u32x4 w;
                        __builtin_memcpy(&w, v, 16);
                        *(u32x4*)out = w;
                    } else {
#pragma unroll
                        for (int e = 0; e < EACH; ++e)
                            if (i0 + e < s.n) out[e] = v[e];
                    }
                }
            }
        }
    } else {
        float* const parts[3] = {a.pool.weight, a.pool.k_scale, a.pool.v_scale};
        for (int i0 = 0; i0 < s.n; i0 += MOVE_THREADS) {
            const int i = i0 + tid;
            float v[3] = {0.0f, 0.0f, 0.0f};
            int64_t to = -1;
            if (i < s.n) {
                const int64_t from = place(table, kept[i]);
                to = place(table_to, i);
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (parts[p]) v[p] = parts[p][layer_slots + (from < 0 ? 0 : from)];
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) asm volatile("" : "+v"(v[p]));
            __syncthreads();
            if (to >= 0)
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (parts[p]) parts[p][layer_slots + to] = v[p];
        }
    }
}

int launch_evict(const EvictArgs& a, const spmm_cache_type_t type, void* stream)
{
    const int64_t most = a.ld_table << a.pool.page_shift, heads = (int64_t)a.n_layers * a.pool.n_heads;
    const dim3 rows((unsigned)heads, (unsigned)a.n_rows), threads(64 * CHOOSE_WAVES);
    int rc;
    if (most <= 64 * CHOOSE_WAVES * 8) rc = launch(cache_evict_choose<8>, rows, threads, a, stream);
    else if (most <= 64 * CHOOSE_WAVES * CHOOSE_REGS) rc = launch(cache_evict_choose<CHOOSE_REGS>, rows, threads, a, stream);
    else rc = launch(cache_evict_choose<0>, rows, threads, a, stream);
    if (rc) return rc;
    int sides = 1;
    int slices = 2 * sides + 1;
    void* args[] = {const_cast<EvictArgs*>(&a), &slices};
    return (int)hipLaunchKernel(type == SPMM_CACHE_S8 ? (const void*)cache_evict_move<SPMM_CACHE_S8> : (const void*)cache_evict_move<SPMM_CACHE_BF16>,
                                dim3((unsigned)(heads * slices), (unsigned)a.n_rows), dim3(MOVE_THREADS), args, 0, (hipStream_t)stream);
}

}  // namespace spmm_cache
