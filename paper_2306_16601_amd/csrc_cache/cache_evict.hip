// Tokens that stay: which ones, and the moves that bring them together.
//
// cache_evict_choose: a workgroup has the weights of a row's head of a layer in its registers (up to 32 thousand tokens) and finds the
// largest (cache_choose.h).  cache_evict_move: a workgroup moves a slice of a row's head, all of its tokens in their order.  A token never
// goes to a later place than its own, so that what a step of tokens is written over has been read, where the pages are the same ones,
// once the step itself has been read; slices (dims of keys, or of values) have nothing to do with each other.  Keys are moved 16 bytes a
// lane.  Values, whose tokens are contiguous, are gathered one by one, tokens side by side in a wave, so that it finds them in a few lines
// of memory: nearly all lines of the values are read wherever one token in sixteen stays.
#include "cache_choose.h"

#include <type_traits>

namespace spmm_cache {

constexpr int CHOOSE_WAVES = 16, CHOOSE_REGS = 32;
constexpr int MOVE_THREADS = 256;
constexpr int PIECE = 1024;         // tokens that are moved with one list of places
constexpr int KEYS_AHEAD = 8, VALUES_AHEAD = 4;
constexpr int VALUE_DIMS = 4;       // of a wave

struct MoveShape {
    int keys, values;       // slices of a head's keys, and of its values
};

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

// (two workgroups on a CU where the registers allow it)
template <int REGS>
__global__ __launch_bounds__(64 * CHOOSE_WAVES, (REGS > 16 ? 4 : 8)) void cache_evict_choose(const EvictArgs a)
{
    constexpr int W = CHOOSE_WAVES;
    __shared__ Bins<W> bins;
    __shared__ int totals[(REGS ? REGS : 1) * W][2];
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
        choose<W>(v, need, bins, totals, put);
    } else {
        choose_long<W>(n, need, bins, totals, rank, put);
    }
}

// Where a piece of the tokens that stay are and go to: bytes from the first of a layer's keys, values or numbers, -1: nowhere.
struct Piece {
    int64_t from[PIECE], to[PIECE / 16];        // `to` of every 16 tokens, which lie in one page
};

// A workgroup moves a slice of a row's head: dims of its keys, dims of its values, or its scales and weights.
template <spmm_cache_type_t TYPE>
__global__ __launch_bounds__(MOVE_THREADS, 5) void cache_evict_move(const EvictArgs a, const MoveShape f)
{
    constexpr int BYTES = TYPE == SPMM_CACHE_S8 ? 1 : 2;
    __shared__ Piece piece;
    const int H = a.pool.n_heads, D = a.pool.head_dim, shift = a.pool.page_shift, inside = (1 << shift) - 1, tid = threadIdx.x;
    const int slices = f.keys + f.values + 1, slice = blockIdx.x % slices, lh = blockIdx.x / slices, h = lh % H, layer = lh / H, b = blockIdx.y;
    const Stay s = stay_of(a, b);
    if (s.n == 0) return;
    const bool keys = slice < f.keys, values = !keys && slice < f.keys + f.values;
    const int32_t *const table = a.table + b * a.ld_table, *const table_to = a.table_to + b * a.ld_table;
    const int32_t* const kept = a.kept + (((int64_t)layer * a.n_rows + b) * H + h) * a.most;
    const int64_t layer_slots = layer * a.layer_slots;
    const auto place = [&](const int32_t* const pages, const int at) {
        const int page = pages[at >> shift];
        if ((uint32_t)page >= (uint32_t)a.pool.n_pages) return (int64_t)-1;
        const int64_t head = ((int64_t)page * H + h) << shift;
        const int off = at & inside;
        return keys ? (head + off) * D * BYTES : values ? (head * D + off) * BYTES : (head + off) * 4;
    };
    for (int i0 = 0; i0 < s.n; i0 += PIECE) {
        const int n = min(s.n - i0, PIECE);
        __syncthreads();        // (the last piece has been read)
        for (int i = tid; i < n; i += MOVE_THREADS) {
            piece.from[i] = max(place(table, kept[i0 + i]), (int64_t)0);
            if (i % 16 == 0) piece.to[i / 16] = place(table_to, i0 + i);
        }
        __syncthreads();
        if (keys) {
            // a lane has 16 bytes of a token
            const int row = D * BYTES, per = row / 16 / f.keys, c = tid % per, rows = MOVE_THREADS / per, r = tid / per;
            char* const pool = (char*)a.pool.k + layer_slots * row + (slice * per + c) * 16;
            for (int i1 = 0; i1 < n; i1 += rows * KEYS_AHEAD) {
                u32x4 v[KEYS_AHEAD] = {};
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) {
                    const int i = i1 + k * rows + r;
                    if (r < rows && i < n) v[k] = *(const u32x4*)(pool + piece.from[i]);
                }
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) asm volatile("" : "+v"(v[k]));       // (loads are back, not only under way, before anyone stores)
                __syncthreads();
#pragma unroll
                for (int k = 0; k < KEYS_AHEAD; ++k) {
                    const int i = i1 + k * rows + r;
                    if (r < rows && i < n && piece.to[i / 16] >= 0) *(u32x4*)(pool + piece.to[i / 16] + i % 16 * row) = v[k];
                }
            }
        } else if (values) {
            // a wave has VALUE_DIMS dims and no other wave has them, a lane four tokens of one
            using E = typename std::conditional<TYPE == SPMM_CACHE_S8, uint8_t, uint16_t>::type;
            constexpr int LANES = 64 / VALUE_DIMS, TOKENS = LANES * 4;       // of a dim; tokens of a wave's step
            const int dims = D / f.values, lane = tid % 64, j = lane % LANES * 4;
            for (int d = (slice - f.keys) * dims + tid / 64 * VALUE_DIMS + lane / LANES; d < (slice - f.keys + 1) * dims; d += MOVE_THREADS / 64 * VALUE_DIMS) {
                char* const pool = (char*)a.pool.v + (layer_slots * D + ((int64_t)d << shift)) * BYTES;
                for (int i1 = j; i1 - j < n; i1 += TOKENS * VALUES_AHEAD) {
                    uint32_t v[VALUES_AHEAD][BYTES] = {};
#pragma unroll
                    for (int k = 0; k < VALUES_AHEAD; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[k][e * BYTES / 4] |= (uint32_t) * (const E*)(pool + piece.from[min(i1 + k * TOKENS + e, n - 1)]) << (e * 8 * BYTES % 32);
                    // (a wave's loads are back before its first store, which waits for the last of them)
#pragma unroll
                    for (int k = 0; k < VALUES_AHEAD; ++k)
#pragma unroll
                        for (int w = 0; w < BYTES; ++w) asm volatile("" : "+v"(v[k][w]));
#pragma unroll
                    for (int k = 0; k < VALUES_AHEAD; ++k) {
                        const int i = i1 + k * TOKENS;
                        if (i >= n || piece.to[i / 16] < 0) continue;
                        char* const out = pool + piece.to[i / 16] + i % 16 * BYTES;
                        if (i + 4 <= n) {
                            if constexpr (BYTES == 1) *(uint32_t*)out = v[k][0];
                            else *(u32x2*)out = u32x2{v[k][0], v[k][BYTES - 1]};
                        } else {
#pragma unroll
                            for (int e = 0; e < 3; ++e)
                                if (i + e < n) ((E*)out)[e] = (E)(v[k][e * BYTES / 4] >> (e * 8 * BYTES % 32));
                        }
                    }
                }
            }
        } else {
            char* const parts[3] = {(char*)a.pool.weight, (char*)a.pool.k_scale, (char*)a.pool.v_scale};
            for (int i1 = 0; i1 < n; i1 += MOVE_THREADS) {
                const int i = i1 + tid;
                float v[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (i < n && parts[p]) v[p] = *(const float*)(parts[p] + layer_slots * 4 + piece.from[i]);
#pragma unroll
                for (int p = 0; p < 3; ++p) asm volatile("" : "+v"(v[p]));
                __syncthreads();
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (i < n && parts[p] && piece.to[i / 16] >= 0) *(float*)(parts[p] + layer_slots * 4 + piece.to[i / 16] + i % 16 * 4) = v[p];
            }
        }
    }
}

int launch_evict(const EvictArgs& a, const spmm_cache_type_t type, void* stream)
{
    const int64_t most = a.ld_table << a.pool.page_shift, heads = (int64_t)a.n_layers * a.pool.n_heads;
    const dim3 rows((unsigned)heads, (unsigned)a.n_rows), threads(64 * CHOOSE_WAVES);
    int rc;
    if (most <= 64 * CHOOSE_WAVES * 8) rc = launch(cache_evict_choose<8>, rows, threads, a, stream);
    else if (most <= 64 * CHOOSE_WAVES * 16) rc = launch(cache_evict_choose<16>, rows, threads, a, stream);
    else if (most <= 64 * CHOOSE_WAVES * CHOOSE_REGS) rc = launch(cache_evict_choose<CHOOSE_REGS>, rows, threads, a, stream);
    else rc = launch(cache_evict_choose<0>, rows, threads, a, stream);
    if (rc) return rc;
    // a slice has 128 bytes of a key at least, and 16 dims of values, one step of four waves
    MoveShape f = {1, a.pool.head_dim / 16};
    if (type == SPMM_CACHE_BF16 && a.pool.head_dim == 128) f.keys = 2;
    void* args[] = {const_cast<EvictArgs*>(&a), &f};
    return (int)hipLaunchKernel(type == SPMM_CACHE_S8 ? (const void*)cache_evict_move<SPMM_CACHE_S8> : (const void*)cache_evict_move<SPMM_CACHE_BF16>,
                                dim3((unsigned)(heads * (f.keys + f.values + 1)), (unsigned)a.n_rows), dim3(MOVE_THREADS), args, 0, (hipStream_t)stream);
}

}  // namespace spmm_cache
