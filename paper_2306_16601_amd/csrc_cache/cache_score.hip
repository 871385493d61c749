// Upper bounds of the products of a page's keys and the new tokens' queries, from the page's bounds.
//
// sum_d q_d > 0 ? q_d hi_d : q_d lo_d  is one product of length 2 D: [max(q, 0), min(q, 0)] . [hi, lo], and a page's bounds lie in that
// order.  So it goes through the matrix instruction, with the query heads of a key/value head as rows and pages as columns: a
// lane then holds four rows of one page, and the highest of the heads that share a key/value head, whose rows are padded to a power of
// two, is taken among a lane's registers and between the four lanes of a page.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
constexpr int PAGES = 16;           // of a step of a wave
constexpr int ROWS = 16;            // of a tile of queries

typedef short s16x8 __attribute__((ext_vector_type(8)));

// NaN where one of them is
__device__ __forceinline__ float higher(const float a, const float b) { return __builtin_elementwise_maximum(a, b); }

struct ScoreShape {
    int padded, log;    // heads of a token in a tile: 1, 2, 4, 8 or 16; its logarithm
    int tokens;         // of a workgroup
    int turns;          // tiles of a token, where it has more than 16 heads
    int steps;          // of pages that a wave takes
};

// KS: steps of 32 of the length 2 D (heads have 16 KS dims); TILES: tiles of queries that a wave has
template <int KS, int TILES>
__global__ __launch_bounds__(THREADS, (TILES > 1 ? 2 : 3)) void cache_score(const ScoreArgs a, const ScoreShape f)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    constexpr int D = 16 * KS;
    const int H = a.pool.n_heads, G = a.group, h = blockIdx.x % H, per = ROWS / f.padded;
    const int width = (int)a.batch.ld_table;
    const int t0 = (int)(blockIdx.x / H) * f.tokens, t1 = min(t0 + f.tokens, a.T);
    const int p0 = (int)(blockIdx.y * WAVES + wave) * f.steps * PAGES, p1 = min(p0 + f.steps * PAGES, width);

    for (int t = t0; t < t1;) {
        // the columns from t on that are one sequence's
        const int b = sequence_of(a.batch, t);
        if (b < 0) {
            ++t;
            continue;
        }
        const int end = min(t1, a.batch.q_start[b + 1]), n = end - t;
        const int32_t* const table = a.batch.table + b * a.batch.ld_table;
        const int shift = a.pool.page_shift, len = tokens_of(a.batch, b, shift);
        // position of column t: of the others it is so many more (they lie between -2^30 and 2^30)
        const int at0 = (int)max((int64_t)a.batch.kv_len[b] - ((int64_t)a.batch.q_start[b + 1] - t), (int64_t)-(1 << 30));
        const int seen = span_of(a.batch, b, end - 1, shift, a.causal, a.window).to >> shift;      // (no column before sees a later page)
#pragma unroll 1
        for (int turn = 0; turn < f.turns; ++turn) {
            // queries: row r of tile x is token (x * 16 + r) / padded, head r % padded (of this turn), or another of it where there is none
            bf16x8 q[TILES][KS];
            int row = col;
            asm volatile("" : "+v"(row));       // (or the tiles' rows are kept over the loop, and spilled)
#pragma unroll
            for (int x = 0; x < TILES; ++x) {
                const int r = x * ROWS + row, token = min(r >> f.log, n - 1), head = min(turn * ROWS + (r & (f.padded - 1)), G - 1);
                const __bf16* const src = a.q + (((int64_t)(t + token) * H + h) * G + head) * D;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int d = 32 * s + 8 * g;
                    const bool low = KS % 2 && s == KS / 2 ? d >= D : s >= (KS + 1) / 2;
                    const s16x8 v = *(const s16x8*)(src + (low ? d - D : d)), negative = v >> 15;
                    q[x][s] = __builtin_bit_cast(bf16x8, low ? v & negative : v & ~negative);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            const auto load = [&](const int p, bf16x8 (&v)[KS]) {
                const int page = page_in_pool(table[max(min(p + col, seen), 0)], a.pool.n_pages);
                const bf16x8* const src = (const bf16x8*)(a.pool.bounds + ((int64_t)page * H + h) * 2 * D) + g;
#pragma unroll
                for (int s = 0; s < KS; ++s) v[s] = src[4 * s];
            };
            const auto store = [&](const int p, const f32x4 (&sc)[TILES]) {
                int g_out = g;
                asm volatile("" : "+v"(g_out));     // (or what the stores need of each tile is worked out before the loop, and spilled)
                if (p + col >= width) return;
#pragma unroll
                for (int x = 0; x < TILES; ++x) {
                    // rows 4 g .. 4 g + 3 of the lane's page: the highest of each token's
                    float s[4] = {sc[x][0], sc[x][1], sc[x][2], sc[x][3]};
                    if (f.padded >= 2) s[0] = higher(s[0], s[1]), s[2] = higher(s[2], s[3]);
                    if (f.padded >= 4) s[0] = higher(s[0], s[2]);
                    if (f.padded >= 8) s[0] = higher(s[0], __shfl_xor(s[0], 16));
                    if (f.padded >= 16) s[0] = higher(s[0], __shfl_xor(s[0], 32));
                    // row 4 g + i is a token's first head, or none
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i & (f.padded - 1) || (f.padded > 4 && 4 * g_out & (f.padded - 1))) continue;
                        const int token = x * per + ((4 * g_out + i) >> f.log);
                        if (token >= n) continue;
                        const int at = at0 + token, to = a.causal ? min(at, len - 1) : len - 1, from = a.window ? max(at, a.window - 1) - (a.window - 1) : 0;
                        const bool visible = at >= 0 && from <= to && p + col >= from >> shift && p + col <= to >> shift;
                        float* const out = a.scores + ((int64_t)(t + token) * H + h) * a.lds + p + col;
                        float y = visible ? s[i] : -__builtin_inff();
                        if (turn && visible) y = higher(y, *out);
                        *out = y;
                    }
                }
            };
            f32x4 sc[TILES];
            bf16x8 v[KS];
            load(p0, v);
            int p = p0;
#pragma unroll 1
            for (; p < p1 && p <= seen; p += PAGES) {
#pragma unroll
                for (int x = 0; x < TILES; ++x) sc[x] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int x = 0; x < TILES; ++x) sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[x][s], v[s], sc[x], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                load(p + PAGES, v);         // (of the last step: pages that are there, and are not used)
                __builtin_amdgcn_sched_barrier(0);
                store(p, sc);
            }
            // what lies behind the visible pages
#pragma unroll
            for (int x = 0; x < TILES; ++x) sc[x] = f32x4{0, 0, 0, 0};
#pragma unroll 1
            for (; p < p1; p += PAGES) store(p, sc);
        }
        t = end;
    }
}

template <int KS>
static int launch_steps(const ScoreArgs& a, const ScoreShape& f, const int tiles, const dim3 grid, void* stream)
{
    void* args[] = {const_cast<ScoreArgs*>(&a), const_cast<ScoreShape*>(&f)};
    return (int)hipLaunchKernel(tiles > 1 ? (const void*)cache_score<KS, 4> : (const void*)cache_score<KS, 1>, grid, dim3(THREADS), args, 0, (hipStream_t)stream);
}

int launch_score(const ScoreArgs& a, void* stream)
{
    ScoreShape f = {};
    f.padded = 1;
    while (f.padded < a.group && f.padded < ROWS) f.padded *= 2, ++f.log;
    f.turns = (a.group + ROWS - 1) / ROWS;
    const int per = ROWS / f.padded, tiles = a.T > 4 * per * (int64_t)a.batch.n_seqs ? 4 : 1;
    // (a block's columns are one sequence's where there are as many sequences as columns, or nearly)
    f.tokens = a.T > 2 * (int64_t)a.batch.n_seqs ? per * tiles : 1;
    const int64_t blocks = ((int64_t)a.T + f.tokens - 1) / f.tokens * a.pool.n_heads, most = (a.batch.ld_table + PAGES * WAVES - 1) / (PAGES * WAVES);
    const int64_t steps = blocks * most / 512 < 8 ? blocks * most / 512 : 8, least = most / 65535 + 1;       // (a grid is at most 65535 high)
    f.steps = (int)(steps < least ? least : steps);
    const dim3 grid((unsigned)blocks, (unsigned)((most + f.steps - 1) / f.steps));
    switch (a.pool.head_dim / 16) {
    case 1: return launch_steps<1>(a, f, tiles, grid, stream);
    case 2: return launch_steps<2>(a, f, tiles, grid, stream);
    case 3: return launch_steps<3>(a, f, tiles, grid, stream);
    case 4: return launch_steps<4>(a, f, tiles, grid, stream);
    case 5: return launch_steps<5>(a, f, tiles, grid, stream);
    case 6: return launch_steps<6>(a, f, tiles, grid, stream);
    case 7: return launch_steps<7>(a, f, tiles, grid, stream);
    default: return launch_steps<8>(a, f, tiles, grid, stream);
    }
}

}  // namespace spmm_cache
