// Upper bounds of the products of a page's keys and the new tokens' queries, from the page's bounds.
//
// sum_d q_d > 0 ? q_d hi_d : q_d lo_d  is one product of length 2 D: [max(q, 0), min(q, 0)] . [hi, lo], and a page's bounds lie in that
// order.  So it goes through the matrix instruction, with the query heads of a key/value head as rows and pages as columns: a
// lane then holds four rows of one page, and the highest of the heads that share a key/value head, whose rows are padded to a power of
// two, is taken among a lane's registers and between the four lanes of a page.
//
// It needs each page's bounds once for all its columns, and writes a score each.  A chunk's waves multiply four tiles of queries with
// each page, and a workgroup's four waves share the pages through LDS: lanes that lie side by side in the instruction's operand are
// other pages, so that loads straight into it take a cache line a lane, and those, not bytes, bounded the kernel.  Scores of 500 columns of 32
// heads for 970 pages of 8: 17.8 us (11 with neither loads nor stores), 25.1 with
// loads into operands two steps ahead, 28 one step ahead.  A batch's next tokens, or a few columns each, have one tile, and there
// each wave takes pages of its own: one token of 16 heads and 486 pages takes 4.0 us, of which a launch is 2.4.
#include "cache_internal.h"

#include <algorithm>

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
    int tokens;         // of a wave
    int turns;          // tiles of a token, where it has more than 16 heads
    int steps;          // of pages, one after the other
};

// Columns t .. t + n - 1, which are one sequence's, and a key/value head.
struct Columns {
    int t, n, h;
    int at0;        // position of column t: of the others it is so many more (they lie between -2^30 and 2^30)
    int len, seen;  // its tokens; the last page that one of the columns up to `end` sees
};
__device__ __forceinline__ Columns columns_of(const ScoreArgs& a, const int b, const int t, const int end, const int h)
{
    const int shift = a.pool.page_shift;
    Columns c;
    c.t = t;
    c.n = end - t;
    c.h = h;
    c.at0 = (int)max((int64_t)a.batch.kv_len[b] - ((int64_t)a.batch.q_start[b + 1] - t), (int64_t)-(1 << 30));
    c.len = tokens_of(a.batch, b, shift);
    c.seen = span_of(a.batch, b, end - 1, shift, a.causal, a.window).to >> shift;       // (no column before sees a later page)
    return c;
}

// Queries as the product's rows: row r of tile x is token (x * 16 + r) / padded, head r % padded of this turn, or another of it where there is none.
template <int KS, int TILES>
__device__ __forceinline__ void load_queries(const ScoreArgs& a, const Columns& c, const int log, const int turn, bf16x8 (&q)[TILES][KS])
{
    constexpr int D = 16 * KS;
    const int H = a.pool.n_heads, G = a.group, g = threadIdx.x % 64 / 16;
    int row = threadIdx.x % 16;
    asm volatile("" : "+v"(row));       // (or the tiles' rows are kept over the loop, and spilled)
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
        const int r = x * ROWS + row, token = max(min(r >> log, c.n - 1), 0), head = min(turn * ROWS + (r & ((1 << log) - 1)), G - 1);
        const __bf16* const src = a.q + (((int64_t)(c.t + token) * H + c.h) * G + head) * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 32 * s + 8 * g;
            const bool low = KS % 2 && s == KS / 2 ? d >= D : s >= (KS + 1) / 2;
            const s16x8 v = *(const s16x8*)(src + (low ? d - D : d)), negative = v >> 15;
            q[x][s] = __builtin_bit_cast(bf16x8, low ? v & negative : v & ~negative);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The scores of pages p .. p + 15 from the products.  Lanes behind the last token or page store what that one's do once more: were they
// left out, a wait for loads would have to wait for the stores behind them too, as those may not have been made.
template <int TILES>
__device__ __forceinline__ void store_scores(const ScoreArgs& a, const Columns& c, const int log, const int turn, const int p, const f32x4 (&sc)[TILES])
{
    const int padded = 1 << log, per = ROWS >> log, shift = a.pool.page_shift, at_page = min(p + (int)(threadIdx.x % 16), (int)a.batch.ld_table - 1);
    int g = threadIdx.x % 64 / 16;
    asm volatile("" : "+v"(g));     // (or what the stores need of each tile is worked out before the loop, and spilled)
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
        // rows 4 g .. 4 g + 3 of the lane's page: the highest of each token's, in each of its rows where it has more than 4
        float s[4] = {sc[x][0], sc[x][1], sc[x][2], sc[x][3]};
        if (padded >= 2) s[0] = higher(s[0], s[1]), s[2] = higher(s[2], s[3]);
        if (padded >= 4) s[0] = higher(s[0], s[2]);
        if (padded >= 8) s[0] = higher(s[0], __shfl_xor(s[0], 16));
        if (padded >= 16) s[0] = higher(s[0], __shfl_xor(s[0], 32));
        const auto put = [&](const int i) {
            const int token = min(x * per + ((4 * g + i) >> log), c.n - 1);
            const int at = c.at0 + token, to = a.causal ? min(at, c.len - 1) : c.len - 1, from = a.window ? max(at, a.window - 1) - (a.window - 1) : 0;
            const bool visible = at >= 0 && from <= to && at_page >= from >> shift && at_page <= to >> shift;
            float* const out = a.scores + ((int64_t)(c.t + token) * a.pool.n_heads + c.h) * a.lds + at_page;
            float y = visible ? s[i] : -__builtin_inff();
            if (turn && visible) y = higher(y, *out);
            *out = y;
        };
        put(0);
        if (padded <= 2) put(2);
        if (padded == 1) put(1), put(3);
    }
}

// Few columns of a sequence: a wave has a tile of them, and pages of its own.
// KS: steps of 32 of the length 2 D (heads have 16 KS dims)
template <int KS>
__global__ __launch_bounds__(THREADS, 3) void cache_score(const ScoreArgs a, const ScoreShape f)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    constexpr int D = 16 * KS;
    const int H = a.pool.n_heads, h = blockIdx.x % H, width = (int)a.batch.ld_table;
    const int t0 = (int)(blockIdx.x / H) * f.tokens, t1 = min(t0 + f.tokens, a.T);
    const int p0 = (int)(blockIdx.y * WAVES + wave) * f.steps * PAGES, p1 = min(p0 + f.steps * PAGES, width);
    for (int t = t0; t < t1;) {
        const int b = sequence_near(a.batch, t);
        if (b < 0) {
            ++t;
            continue;
        }
        const int end = min(t1, a.batch.q_start[b + 1]);
        const Columns c = columns_of(a, b, t, end, h);
        const int32_t* const table = a.batch.table + b * a.batch.ld_table;
#pragma unroll 1
        for (int turn = 0; turn < f.turns; ++turn) {
            bf16x8 q[1][KS];
            load_queries<KS, 1>(a, c, f.log, turn, q);
            const auto entry = [&](const int p) { return table[max(min(min(p + col, width - 1), c.seen), 0)]; };
            const auto load = [&](const int page, bf16x8 (&v)[KS]) {
                const bf16x8* const src = (const bf16x8*)(a.pool.bounds + ((int64_t)page_in_pool(page, a.pool.n_pages) * H + h) * 2 * D) + g;
#pragma unroll
                for (int s = 0; s < KS; ++s) v[s] = src[4 * s];
            };
            f32x4 sc[1];
            bf16x8 v[KS];
            load(entry(p0), v);
            int p = p0, page = entry(p0 + PAGES);
#pragma unroll 1
            for (; p < p1 && p <= c.seen; p += PAGES) {
                sc[0] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s) sc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[0][s], v[s], sc[0], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                load(page, v);      // (behind the last step: pages that are there, and are not used)
                page = entry(p + 2 * PAGES);
                __builtin_amdgcn_sched_barrier(0);
                store_scores<1>(a, c, f.log, turn, p, sc);
            }
            // what lies behind the visible pages
            sc[0] = f32x4{0, 0, 0, 0};
#pragma unroll 1
            for (; p < p1; p += PAGES) store_scores<1>(a, c, f.log, turn, p, sc);
        }
        t = end;
    }
}

// Many columns of a sequence: each wave of a workgroup has four tiles of them, and all have the same pages, whose bounds go through LDS.
template <int KS, int LOG>
__global__ __launch_bounds__(THREADS, 2) void cache_score_many(const ScoreArgs a, const ScoreShape f)
{
    constexpr int D = 16 * KS, ROW = 4 * KS + 1;        // a page's bounds in LDS, in 16 bytes (one more: 16 pages' lie in other banks)
    constexpr int PARTS = PAGES * 4 * KS, EACH = (PARTS + THREADS - 1) / THREADS;
    __shared__ u32x4 bounds[2][PAGES * ROW];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, h = blockIdx.x % H, width = (int)a.batch.ld_table, turns = LOG == 4 ? f.turns : 1;
    const int t0 = (int)(blockIdx.x / H) * f.tokens * WAVES, t1 = min(t0 + f.tokens * WAVES, a.T);
    const int p0 = (int)blockIdx.y * f.steps * PAGES, p1 = min(p0 + f.steps * PAGES, width);
    for (int t = t0; t < t1;) {
        const int b = sequence_near(a.batch, t);
        if (b < 0) {
            ++t;
            continue;
        }
        const int end = min(t1, a.batch.q_start[b + 1]), mine = min(t + wave * f.tokens, end);
        Columns c = columns_of(a, b, t, end, h);
        c.at0 += mine - t;
        c.t = min(mine, end - 1);       // (a wave with none loads what another does, and stores nothing)
        c.n = min(end - mine, f.tokens);
        const int32_t* const table = a.batch.table + b * a.batch.ld_table;
#pragma unroll 1
        for (int turn = 0; turn < turns; ++turn) {
            bf16x8 q[4][KS];
            load_queries<KS, 4>(a, c, LOG, turn, q);
            // this thread's parts of a step: looked up two steps ahead, loaded one step ahead (behind the last step: of pages that are there)
            int page[EACH];
            u32x4 part[EACH];
            const auto look = [&](const int p) {
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    page[i] = table[max(min(min(p + (int)(min(i * THREADS + threadIdx.x, PARTS - 1u) / (4 * KS)), width - 1), c.seen), 0)];
            };
            const auto load = [&] {
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    part[i] = *((const u32x4*)(a.pool.bounds + ((int64_t)page_in_pool(page[i], a.pool.n_pages) * H + h) * 2 * D) +
                                min(i * THREADS + threadIdx.x, PARTS - 1u) % (4 * KS));
            };
            const auto stage = [&](const int to) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const unsigned at = i * THREADS + threadIdx.x;
                    if (PARTS % THREADS == 0 || at < PARTS) bounds[to][at / (4 * KS) * ROW + at % (4 * KS)] = part[i];
                }
            };
            look(p0);
            load();
            look(p0 + PAGES);
            f32x4 sc[4];
            int p = p0;
#pragma unroll 1
            for (int to = 0; p < p1 && p <= c.seen; p += PAGES, to ^= 1) {
                stage(to);
                __syncthreads();        // (and the buffer of the step before is read by none once all are here again)
                load();
                look(p + 2 * PAGES);
#pragma unroll
                for (int x = 0; x < 4; ++x) sc[x] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, bounds[to][col * ROW + 4 * s + g]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[x][s], v, sc[x], 0, 0, 0);
                }
                if (c.n > 0) store_scores<4>(a, c, LOG, turn, p, sc);
            }
            // what lies behind the visible pages
#pragma unroll
            for (int x = 0; x < 4; ++x) sc[x] = f32x4{0, 0, 0, 0};
#pragma unroll 1
            for (; c.n > 0 && p < p1; p += PAGES) store_scores<4>(a, c, LOG, turn, p, sc);
            __syncthreads();
        }
        t = end;
    }
}

template <int KS>
static int launch_steps(const ScoreArgs& a, const ScoreShape& f, const bool many, const dim3 grid, void* stream)
{
    const void* const forms[] = {(const void*)cache_score_many<KS, 0>, (const void*)cache_score_many<KS, 1>, (const void*)cache_score_many<KS, 2>,
                                 (const void*)cache_score_many<KS, 3>, (const void*)cache_score_many<KS, 4>};
    void* args[] = {const_cast<ScoreArgs*>(&a), const_cast<ScoreShape*>(&f)};
    return (int)hipLaunchKernel(many ? forms[f.log] : (const void*)cache_score<KS>, grid, dim3(THREADS), args, 0, (hipStream_t)stream);
}

int launch_score(const ScoreArgs& a, void* stream)
{
    ScoreShape f = {};
    f.padded = 1;
    while (f.padded < a.group && f.padded < ROWS) f.padded *= 2, ++f.log;
    f.turns = (a.group + ROWS - 1) / ROWS;
    const int per = ROWS / f.padded;
    // (32 heads on 8, 16 thousand tokens, us, many against few: 17 columns 6.9 / 9.7, 64 7.5 / 12.9, 500 17.2 / 70, 8 times 32 20 / 38; 4 columns 5.1 either way)
    const bool many = a.T > 4 * per * (int64_t)a.batch.n_seqs;
    // (a block's columns are one sequence's where there are as many sequences as columns, or nearly)
    f.tokens = many ? 4 * per : a.T > 2 * (int64_t)a.batch.n_seqs ? per : 1;
    const int tokens = many ? f.tokens * WAVES : f.tokens, pages = many ? PAGES : PAGES * WAVES;      // of a workgroup, and of a step of it
    const int64_t blocks = ((int64_t)a.T + tokens - 1) / tokens * a.pool.n_heads, most = (a.batch.ld_table + pages - 1) / pages;
    // 512 workgroups, or up to 8 steps: 500 columns and 970 pages 17.1 us, 17.1 with 256, 20.6 with 1024, 20.6 with up to 4 steps, 17.0 with 16; 64 single tokens of up to 8
    // thousand 20.7, 21.1, 22.8, 22.8, 20.7; 4 times 2 columns of 100 thousand 31.7, 31.6, 34.8, 35.3, 31.7; 1024 columns of 30 thousand 56.8, 56.7, 56.8, 54.3, 53.3.
    const int64_t wanted = (blocks * most + 511) / 512, least = most / 65535 + 1;       // (a grid is at most 65535 high)
    f.steps = (int)std::max(std::min(wanted, (int64_t)8), least);
    const dim3 grid((unsigned)blocks, (unsigned)((most + f.steps - 1) / f.steps));
    switch (a.pool.head_dim / 16) {
    case 1: return launch_steps<1>(a, f, many, grid, stream);
    case 2: return launch_steps<2>(a, f, many, grid, stream);
    case 3: return launch_steps<3>(a, f, many, grid, stream);
    case 4: return launch_steps<4>(a, f, many, grid, stream);
    case 5: return launch_steps<5>(a, f, many, grid, stream);
    case 6: return launch_steps<6>(a, f, many, grid, stream);
    case 7: return launch_steps<7>(a, f, many, grid, stream);
    default: return launch_steps<8>(a, f, many, grid, stream);
    }
}

}  // namespace spmm_cache
