// Attention where a key/value head has many columns (chunks of prompts): bound by the matrix instructions and by the
// exponentials between them.
//
// A workgroup takes a block of 128 columns of a sequence's head, or of 256, 32 for each of its waves, and walks over tiles of
// 64 keys that all waves share through LDS (two buffers; the next tile is on its way while this one is multiplied).
// bfloat16 operands go from the pages to LDS without passing through registers, 16 bytes a lane; rows of LDS are 8 or 16 such
// chunks, whose order is turned by the row's number so that 16 rows read together lie in different banks, and the order is
// made by where a lane reads, not by where it writes.  Codes of 8 bits are widened to binary16 and multiplied by their scales
// (over a power of two for the tile) on the way.  Scores, weights and sums stay in registers: see cache_attend.h; with the
// 32x32 instruction the lane's 16 scores of a tile of 32 keys are tokens 8 h .. 8 h + 7 of each half (h = lane / 32).
// The running maximum moves only when a score exceeds it by 2^8: the weights have the room, and the sums need no scaling then
// (two prompts of 4097 tokens 313 us, with every larger score 330; whole calls, means of two runs of 400, as below).
//
// A wave goes through two phases for a tile: products (values of tile i with its weights, then scores of tile i + 1), and
// the softmax of tile i + 1.  Two waves share a SIMD, and the matrix unit stands still while both are in the second.  With
// bfloat16 that is left to chance, between two workgroups of 128 columns: two prompts of 4097 tokens, 32 heads on 8 of 128,
// 313 us (0.88 PFLOP/s, the matrix unit busy for 43 % of the cycles, at 2.0 GHz: the card's power bounds it as well).  With 256
// columns, waves 4 to 7 held half a tile behind waves 0 to 3 by a barrier after each phase, the compiler spills 77 registers and it takes
// 485 us (346 against 332 before results were stored by type); so that form is
// taken for 8 bits only, whose widening twice the columns share (500 tokens behind 15000: 197 us, 128 columns 213).
//
// Blocks are dealt out head by head, the longest first, to one XCD after the other, so that blocks that read the same keys
// share an L2 (in the order of their numbers 360 instead of 313 us, and 16 sequences of up to
// 384 tokens 24.3 instead of 19.4).  Where the device could run twice as many workgroups as there are blocks, or more, the tiles
// of each block are dealt to `parts` workgroups, and cache_join_many joins what they write to scratch (500 tokens behind 15000,
// 8 bits: 197 instead of 695 us).
#include "cache_attend.h"

#include <cfloat>
#include <type_traits>

#define INLINE __attribute__((always_inline))

namespace spmm_cache {

constexpr int TILE = 64;            // keys
constexpr int CUS = 256, XCDS = 8;
constexpr float ROOM = 8.0f;

// GROUPS: of four waves
template <int GROUPS>
constexpr int BLOCK = 128 * GROUPS;         // columns
template <int GROUPS>
constexpr int ROUND = CUS * 2 / GROUPS;     // workgroups that the device runs at a time

__host__ __device__ constexpr int64_t part_floats(const int dim, const int cols) { return (int64_t)cols * (dim + 2); }

__device__ __forceinline__ int uniform(const int v) { return __builtin_amdgcn_readfirstlane(v); }

// A block of columns: c0 .. c1 - 1 of a sequence's head, and its tiles.
struct Block {
    int c0, c1, tile0, tiles;
};

__device__ __forceinline__ Block block_of(const AttendArgs& a, const Sequence& s, const int j, const int cols)
{
    Block k = {j * cols, min((j + 1) * cols, s.tokens * a.group), 0, 0};
    if (k.c0 >= k.c1) return k;
    k.tile0 = s.first_seen(a, k.c0 / a.group) / TILE;
    k.tiles = max(s.last_seen(a, (k.c1 - 1) / a.group) / TILE + 1 - k.tile0, 1);
    return k;
}

// the other half of the wave's value.  (The operands are told apart: of the swap of a value with itself, the compiler may take
// one result for both.)
__device__ __forceinline__ float other_half(const float v)
{
    uint32_t same = __builtin_bit_cast(uint32_t, v);
    asm volatile("" : "+v"(same));
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), same, false, false);
    return __builtin_bit_cast(float, threadIdx.x & 32 ? r[0] : r[1]);
}

// largest of a wave: within rows of 16 lanes, then of the rows
template <int CONTROL>
__device__ __forceinline__ float max_dpp(const float v)
{
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = max_dpp<0x121>(v);      // row_ror:1
    v = max_dpp<0x122>(v);
    v = max_dpp<0x124>(v);
    v = max_dpp<0x128>(v);
    float most = v;
#pragma unroll
    for (int row = 0; row < 64; row += 16) most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), row)));
    return most;
}

// chunk of LDS, of 16 bytes, that chunk c of a row lies in: rows of 8 chunks (two rows cover the banks), or of 16
template <int CHUNKS>
__device__ __forceinline__ int turned(const int row, const int c)
{
    return CHUNKS == 16 ? c ^ (row & 15) : c ^ (row >> 1 & 7);
}

// In place: as an expression, under a condition, it costs copies of all sums where the condition does not hold.
__device__ __forceinline__ void scale_in_place(float& o, const float by)
{
    float y = o;
    asm volatile("v_mul_f32 %0, %1, %0" : "+v"(y) : "v"(by));
    o = y;
}

// Eight codes times scales, in binary16, rounded once: (n + 128) s - 128 s is n s but for the last place of binary32, and for scales that
// are not finite.
template <typename F>
__device__ __forceinline__ f16x8 scaled(uint32_t a, uint32_t b, const F& by)
{
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    f16x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (_Float16)__fmaf_rn((float)((j < 4 ? a : b) >> 8 * (j % 4) & 0xff), by(j), -128.0f * by(j));
    return r;
}

// the same for any scales
template <typename F>
__device__ __forceinline__ f16x8 product(const uint32_t a, const uint32_t b, const F& by)
{
    f16x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (_Float16)((float)(int8_t)((j < 4 ? a : b) >> 8 * (j % 4)) * by(j));
    return r;
}

// A barrier for what is in LDS: stores to memory are not waited for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <int DIM>
struct Half {       // keys [64][DIM], or values [DIM][64], of a tile, in 16 bits
    uint4 at[TILE * DIM / 8];
};

template <int DIM, spmm_cache_type_t TYPE, bool EXACT, int GROUPS, bool SPLIT>
__global__ __launch_bounds__(256 * GROUPS, 2) void cache_attend_many(const AttendArgs a, const int blocks, const int parts)
{
    constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    constexpr int WAVES = 4 * GROUPS, THREADS = 64 * WAVES;
    constexpr int KC = DIM / 8, DT = DIM / 32, KS = DIM / 16;       // chunks of a key's row, dim tiles, steps of scores
    constexpr int CPI = DIM / 8 / WAVES;                            // instructions of a wave for a tile's keys, and for its values
    constexpr int UNITS = 2 * TILE * DIM / 16 / THREADS;            // 16 codes that a thread widens
    __shared__ Half<DIM> keys0, keys1, values0, values1;       // (apart, so that loads to one are not waited for by reads of another)
    __shared__ float scales[S8 ? WAVES : 1][2][TILE];
    __shared__ int odd_found;

    const int tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64), col = lane % 32, half = lane / 32;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;

    if constexpr (!EXACT) {     // what lies beyond the head's dims is never loaded
        for (int i = tid; i < TILE * DIM / 8; i += THREADS) keys0.at[i] = keys1.at[i] = values0.at[i] = values1.at[i] = uint4{0, 0, 0, 0};
        __syncthreads();
    }

    // where a lane reads the first operands of a tile; step k of keys lies at off_k ^ 32 k, step e of values at off_v ^ 32 e.
    // Row r of a tile of scores is token r with bits 2 and 3 exchanged.
    const int k_row = (col & 0x13) | (col & 4) << 1 | (col & 8) >> 1;
    int off_k = (k_row * KC + turned<KC>(k_row, half)) * 16, off_v = (col * 8 + turned<8>(col, half)) * 16;

    // XCD x takes the x-th part of all (head, sequence) pairs with their blocks
    const uint32_t all = gridDim.x / XCDS, id = blockIdx.x % XCDS * all + blockIdx.x / XCDS;
    const uint32_t place = SPLIT ? id / (uint32_t)parts : id, part = SPLIT ? id % (uint32_t)parts : 0;
    const uint32_t pair = place / (uint32_t)blocks, j = blocks - 1 - place % (uint32_t)blocks;
    const int h = (int)(pair / (uint32_t)a.batch.n_seqs), b = (int)(pair % (uint32_t)a.batch.n_seqs);
    if (h >= H) return;
    const Sequence s = sequence(a, b);
    const Block blk = block_of(a, s, (int)j, BLOCK<GROUPS>);
    if (blk.tiles == 0) return;
    const int u0 = SPLIT ? (int)((int64_t)blk.tiles * part / parts) : 0;
    const int u1 = SPLIT ? (int)((int64_t)blk.tiles * (part + 1) / parts) : blk.tiles;
    if (SPLIT && u0 == u1) return;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    const int last_page = max(s.len - 1, 0) >> shift;

    const int seen_from = s.first_seen(a, blk.c0 / G), seen_to = s.last_seen(a, (blk.c1 - 1) / G);          // by some column
    const int all_from = s.first_seen(a, (blk.c1 - 1) / G), all_to = s.last_seen(a, blk.c0 / G);            // by all

    // ---- a tile on its way to LDS: the keys of tile i + 1 with the values of tile i ----
    // bfloat16: instruction j of the wave fills 1 KB, 16 bytes a lane.  Page numbers are asked for a tile ahead.  A wave's
    // keys lie in one page; values of a tile do where pages have 64 tokens and more.
    const uint32_t page_bytes = (uint32_t)(H * D) << shift << (S8 ? 0 : 1);
    const char* const k_head = (const char*)a.pool.k + ((int64_t)h * D << shift) * 2;
    const char* const v_head = (const char*)a.pool.v + (((int64_t)h * D + wave * CPI * 8) << shift) * 2;
    constexpr int NP = CPI > 1 ? 2 : 1;        // of a wave's rows of values, that are turned differently
    int page_k = 0, page_v[2] = {0, 0};
    uint32_t off_fk[S8 ? 1 : CPI], off_fv[NP];
    if constexpr (!S8) {
#pragma unroll
        for (int j = 0; j < CPI; ++j) {
            const int row = (wave * CPI + j) * (64 / KC) + lane / KC;
            off_fk[j] = ((row - wave * CPI * (64 / KC)) * D + 8 * turned<KC>(row, lane % KC)) * 2;
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) off_fv[j] = ((lane / 8 << shift) + (8 * turned<8>((wave * CPI + j) * 8 + lane / 8, lane % 8) & inside)) * 2;
    }
    constexpr int ROWS = 64 / WAVES;        // keys that a wave fetches
    const auto page_at = [&](const int key) INLINE { return table[min(max(key, 0) >> shift, last_page)]; };       // (never beyond the sequence's)
    const auto name = [&](const int k0) INLINE {       // of the keys of the tile at k0 + TILE, and the values of that at k0
        if constexpr (!S8) {
            page_k = page_at(k0 + TILE + ROWS * wave);
#pragma unroll
            for (int j = 0; j < NP; ++j) page_v[j] = page_at(k0 + (shift < 6 ? 8 * turned<8>((wave * CPI + j) * 8 + lane / 8, lane % 8) : 0));
        }
    };
    // (in parts, so that a step can issue them between its products: all at once they fill the address unit's queue)
    const char *k_from = nullptr, *v_from[NP] = {};
    const auto aim = [&](const int k0) INLINE {      // at the keys of the tile at k0 + TILE, and the values of that at k0
        k_from = k_head + (int64_t)page_in_pool(uniform(page_k), a.pool.n_pages) * page_bytes + ((k0 + TILE + ROWS * wave) & inside) * D * 2;
        if (shift >= 6) {
            const char* const v = v_head + (int64_t)page_in_pool(uniform(page_v[0]), a.pool.n_pages) * page_bytes + (k0 & inside) * 2;
#pragma unroll
            for (int j = 0; j < NP; ++j) v_from[j] = v + off_fv[j];
        } else {
#pragma unroll
            for (int j = 0; j < NP; ++j) v_from[j] = v_head + off_fv[j] + (uint64_t)(uint32_t)page_in_pool(page_v[j], a.pool.n_pages) * page_bytes;
        }
    };
    const auto fetch_k = [&](Half<DIM>& t, const int j) INLINE {
        if (EXACT || 8 * turned<KC>((wave * CPI + j) * (64 / KC) + lane / KC, lane % KC) < D)
            __builtin_amdgcn_global_load_lds((global_void*)(k_from + off_fk[j]), (lds_void*)(t.at + (wave * CPI + j) * 64), 16, 0, 0);
    };
    const auto fetch_v = [&](Half<DIM>& t, const int j) INLINE {
        if (EXACT || (wave * CPI + j) * 8 < D)
            __builtin_amdgcn_global_load_lds((global_void*)(v_from[j % NP] + (((int64_t)8 * j) << shift) * 2), (lds_void*)(t.at + (wave * CPI + j) * 64), 16, 0, 0);
    };
    // 8 bits: a thread has units of 16 codes in registers until the phases before have ended, keys in the first half of
    // all units and values in the second; a lane has the scales of a key, and of a value's token
    u32x4 raw[S8 ? UNITS : 1];
    int unit_page[S8 ? UNITS : 1], lane_page_k = 0, lane_page_v = 0;
    float lane_k = 0.0f, lane_v = 0.0f;
    constexpr int UPR = DIM / 16, HALF_UNITS = TILE * DIM / 16;     // units of a key's row, and of a tile's keys
    const auto is_key = [&](const int i) INLINE { return UNITS > 1 ? i < UNITS / 2 : tid < HALF_UNITS; };
    const auto unit_of = [&](const int i) INLINE { return UNITS > 1 ? tid + THREADS * (i % (UNITS / 2 > 0 ? UNITS / 2 : 1)) : tid % HALF_UNITS; };
    const auto name_codes = [&](const int k0) INLINE {
        if constexpr (S8) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) unit_page[i] = page_at(is_key(i) ? k0 + TILE + unit_of(i) / UPR : k0 + unit_of(i) % 4 * 16);
            lane_page_k = page_at(k0 + TILE + lane);
            lane_page_v = page_at(k0 + lane);
        }
    };
    const auto fetch_codes = [&](const int k0) INLINE {        // keys of the tile at k0 + TILE, values of that at k0
        if constexpr (S8) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int64_t page = (int64_t)page_in_pool(unit_page[i], a.pool.n_pages) * H + h;
                const int u = unit_of(i), d = is_key(i) ? u % UPR * 16 : u / 4;
                const int64_t at = is_key(i) ? ((page << shift) + ((k0 + TILE + u / UPR) & inside)) * D + d : ((page * D + d) << shift) + ((k0 + u % 4 * 16) & inside);
                raw[i] = EXACT || d < D ? *(const u32x4*)((const int8_t*)(is_key(i) ? a.pool.k : a.pool.v) + at) : u32x4{0, 0, 0, 0};
            }
            lane_k = a.pool.k_scale[(((int64_t)page_in_pool(lane_page_k, a.pool.n_pages) * H + h) << shift) + ((k0 + TILE + lane) & inside)];
            lane_v = a.pool.v_scale[(((int64_t)page_in_pool(lane_page_v, a.pool.n_pages) * H + h) << shift) + ((k0 + lane) & inside)];
        }
    };
    // powers of two that are left out: of the keys widened last, and before them; of the values; what the sums have to be
    // multiplied by before the values widened last are added, and before those widened before them are
    float k_up = 1.0f, k_up_last = 1.0f, v_up = __builtin_bit_cast(float, 2u << 23), v_less_next = 1.0f, v_less = 1.0f;
    const auto widen_codes = [&](Half<DIM>& tk, Half<DIM>& tv, const int k0) INLINE {
        if constexpr (S8) {
            const bool k_here = k0 + TILE + lane >= seen_from && k0 + TILE + lane <= seen_to, v_here = k0 + lane >= seen_from && k0 + lane <= seen_to;
            if (!k_here) lane_k = 0.0f;     // (they may be anything)
            if (!v_here) lane_v = 0.0f;
            const float mk = wave_max(fabsf(lane_k) <= 3.4e38f ? fabsf(lane_k) : 0.0f), mv = wave_max(fabsf(lane_v) <= 3.4e38f ? fabsf(lane_v) : 0.0f);
            k_up_last = k_up;
            float up;
            const float k_down = to_unit(mk, &k_up);
            to_unit(mv, &up);
            up = fmaxf(up, v_up);
            v_less_next = v_up / up;
            v_up = up;
            const float v_down = __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, up));
            __builtin_amdgcn_wave_barrier();
            scales[wave][0][lane] = lane_k * k_down;
            scales[wave][1][lane] = lane_v * v_down;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int u = unit_of(i), row = is_key(i) ? u / UPR : u / 4;
                if (is_key(i)) {
                    const float by = scales[wave][0][row];
                    const int c = u % UPR * 2;
                    *(f16x8*)(tk.at + row * KC + turned<KC>(row, c)) = scaled(raw[i][0], raw[i][1], [&](int) { return by; });
                    *(f16x8*)(tk.at + row * KC + turned<KC>(row, c + 1)) = scaled(raw[i][2], raw[i][3], [&](int) { return by; });
                } else {
                    const float* const by = scales[wave][1] + u % 4 * 16;
                    const int c = u % 4 * 2;
                    *(f16x8*)(tv.at + row * 8 + turned<8>(row, c)) = scaled(raw[i][0], raw[i][1], [&](const int j) { return by[j]; });
                    *(f16x8*)(tv.at + row * 8 + turned<8>(row, c + 1)) = scaled(raw[i][2], raw[i][3], [&](const int j) { return by[8 + j]; });
                }
            }
            if (__any(!(fabsf(lane_v) <= 3.4e38f))) {       // (infinite values; such keys have scores of NaN)
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int u = unit_of(i), row = u / 4, c = u % 4 * 2;
                    const float* const by = scales[wave][1] + u % 4 * 16;
                    if (is_key(i)) continue;
                    *(f16x8*)(tv.at + row * 8 + turned<8>(row, c)) = product(raw[i][0], raw[i][1], [&](const int j) { return by[j]; });
                    *(f16x8*)(tv.at + row * 8 + turned<8>(row, c + 1)) = product(raw[i][2], raw[i][3], [&](const int j) { return by[8 + j]; });
                }
            }
        }
    };
    // What no column sees may hold anything (pages are not cleared): it counts as 0, and so does what is not finite where
    // some columns see it and others do not (odd_sum).
    const auto clean = [&](Half<DIM>& t, const int k0) INLINE {
        bool odd = false;
        for (int i = tid; i < DIM * 8; i += THREADS) {
            const int row = i / 8, c = turned<8>(row, i % 8);
            u32x4 v = __builtin_bit_cast(u32x4, t.at[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = k0 + 8 * c + 2 * j;
                if (key < seen_from || key > seen_to) v[j] &= 0xffff0000u;
                if (key + 1 < seen_from || key + 1 > seen_to) v[j] &= 0xffffu;
            }
            const u32x4 w = S8 ? finite_half_or_zero(v) : finite_or_zero(v);
            odd |= (v[0] != w[0]) | (v[1] != w[1]) | (v[2] != w[2]) | (v[3] != w[3]);
            t.at[i] = __builtin_bit_cast(uint4, w);
        }
        if (odd) odd_found = 1;
    };

    if (tid == 0) odd_found = 0;
    const int first = (blk.tile0 + u0) * TILE;
    const int end = min((blk.tile0 + u1) * TILE, seen_to + 1);      // (where nobody sees anything there is a tile all the same)
    const int n = first < end ? (end - first + TILE - 1) / TILE : 0;
    if (n) {        // the first keys, before the queries are asked for
        if constexpr (S8) {
            name_codes(first - TILE);       // (the values of a tile before the first one: in the pool, and written over)
            fetch_codes(first - TILE);
            name_codes(first);
        } else {
            name(first - TILE);
            aim(first - TILE);
#pragma unroll
            for (int j = 0; j < CPI; ++j) fetch_k(keys0, j);
            name(first);
        }
    }

    // columns
    const int mine = blk.c0 + wave * 32 + col;
    int lo, hi;
    u32x4 q[KS];
    float unit = a.scale_log2;      // of scores: log2(e) * scale, and the power of two that the queries were divided by
    {
        const bool there = mine < blk.c1;
        const int token = there ? mine / G : 0, head = h * G + (there ? mine % G : 0);
        lo = s.first_seen(a, token);
        hi = there ? s.last_seen(a, token) : -1;
        const __bf16* const src = a.q + ((int64_t)(s.first + token) * (H * G) + head) * D;
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int d = 16 * k + 8 * half;
            q[k] = there && (EXACT || d < D) ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
            if constexpr (S8) {
                const bf16x8 v = __builtin_bit_cast(bf16x8, q[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf((float)v[j]));
            }
        }
        if constexpr (S8) {
            most = fmaxf(most, other_half(most));
            float up;
            const float down = to_unit(most, &up);
            unit *= up;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8 v = __builtin_bit_cast(bf16x8, q[k]);
                f16x8 w;
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (_Float16)((float)v[j] * down);
                q[k] = __builtin_bit_cast(u32x4, w);
            }
        }
    }
    f32x16 o[DT], sc[2];
    u32x4 p[4];
    float m = NONE, l = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    // ---- products: values of a tile with its weights, then scores of the next one (if there is one) ----
    const auto multiply = [&](const Half<DIM>& tv, const Half<DIM>& tk, const bool scores, auto&& between) INLINE {
        asm volatile("" : "+v"(off_k), "+v"(off_v));        // (worked out for each tile: registers are scarce)
        constexpr int PV = 4 * DT, QK = 2 * KS, AHEAD = 6;      // operands are read so many instructions ahead
        u32x4 x[PV + QK];
        const auto read = [&](const int i) INLINE {
            if (i < PV) x[i] = *(const u32x4*)((const char*)tv.at + (off_v ^ 32 * (i / DT)) + 32 * (i % DT) * 8 * 16);
            else x[i] = *(const u32x4*)((const char*)tk.at + (off_k ^ 32 * ((i - PV) / 2)) + 32 * ((i - PV) % 2) * KC * 16);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            read(i + AHEAD);
            const int d = i % DT, e = i / DT;
            if constexpr (S8) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x[i]), __builtin_bit_cast(f16x8, p[e]), o[d], 0, 0, 0);
            else o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[i]), __builtin_bit_cast(bf16x8, p[e]), o[d], 0, 0, 0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!scores) return;
#pragma unroll
        for (int i = 0; i < QK; ++i) {
            if (i + AHEAD < QK) read(PV + i + AHEAD);
            const int g = i % 2, k = i / 2;
            const f32x16 zero = {};
            if constexpr (S8) sc[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x[PV + i]), __builtin_bit_cast(f16x8, q[k]), k ? sc[g] : zero, 0, 0, 0);
            else sc[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[PV + i]), __builtin_bit_cast(bf16x8, q[k]), k ? sc[g] : zero, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // ---- softmax of a tile's scores ----
    const auto weigh = [&](const int k0, const float keys_up, auto&& between) INLINE {
        // (never 0, which what is hidden, -inf, must not be multiplied by: scores are below 2^19, and with less than that 0)
        const float by = S8 ? fmaxf(unit * keys_up, FLT_MIN) : unit;
        if (k0 < all_from || k0 + TILE - 1 > all_to) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int key = k0 + 16 * (i / 8) + 8 * half + i % 8;
                sc[i / 16][i % 16] = key >= lo && key <= hi ? sc[i / 16][i % 16] : NONE;
            }
        }
        float top = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i / 16][i % 16]);
        top = fmaxf(top, other_half(top)) * by;
        if (__any(top > m + ROOM)) {
            const float mn = fmaxf(m, top);
            float fade = __builtin_amdgcn_exp2f(m - (mn == NONE ? 0.0f : mn));
            m = mn;
            l *= fade;
            asm volatile("s_nop 1" : "+v"(fade));       // (the exponential needs that before its result is read)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) { float y = o[d][i]; scale_in_place(y, fade); o[d][i] = y; }
        }
        const float ms = m == NONE ? 0.0f : m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[e / 2][e % 2 * 8 + j], by, -ms));
            if constexpr (S8) {
                f16x8 w;
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (_Float16)x[j];
                l = sum_of(w, l);
                p[e] = __builtin_bit_cast(u32x4, w);
            } else {
                bf16x8 w;
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (__bf16)x[j];
                l = sum_of(w, l);
                p[e] = __builtin_bit_cast(u32x4, w);
            }
            between(e);
        }
    };

    if (n) {
        if constexpr (S8) {
            widen_codes(keys0, values1, first - TILE);
            v_up = __builtin_bit_cast(float, 2u << 23);
            v_less_next = v_less = 1.0f;
            fetch_codes(first);
            name_codes(first + TILE);
        }
        __syncthreads();
    }
    // Step t: waves ahead multiply values t - 1 and keys t, then weigh tile t; waves behind weigh tile t - 1, then multiply.
    const auto step = [&](auto is_ahead, Half<DIM>& k_now, Half<DIM>& k_next, Half<DIM>& v_now, Half<DIM>& v_last, const int t) INLINE {
        constexpr bool ahead = decltype(is_ahead)::value;
        const int k0 = first + t * TILE;
        const bool more = t < n, more_k = t + 1 < n;
        if constexpr (!S8) aim(k0);
        // 8 bits: the codes of this step are in registers; those of the next are asked for as soon as they are not
        const auto widen_now = [&]() INLINE {
            if (S8 && more) {
                widen_codes(k_next, v_now, k0);
                if (more_k) {
                    fetch_codes(k0 + TILE);
                    name_codes(k0 + 2 * TILE);
                }
            }
        };
        // a quarter of the wave's loads to LDS
        const auto fetch = [&](const int part) INLINE {
            if constexpr (!S8) {
                constexpr int EACH = (2 * CPI + 3) / 4;
#pragma unroll
                for (int i = part * EACH; i < (part + 1) * EACH && i < 2 * CPI; ++i) {
                    if (i < CPI) {
                        if (more_k) fetch_k(k_next, i);
                    } else {
                        if (more) fetch_v(v_now, i - CPI);
                    }
                }
                if (part == 3 && more) name(k0 + TILE);
            }
        };
        const auto nothing = [](const int) INLINE {};
        __builtin_amdgcn_sched_barrier(0);
        const auto products = [&](auto&& between) INLINE {
            if constexpr (S8) {
                if (v_less != 1.0f) {
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) { float y = o[d][i]; scale_in_place(y, v_less); o[d][i] = y; }
                }
            }
            multiply(v_last, k_now, more, between);
            if (t == 0) {       // (there were no weights yet)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
            }
        };
        if constexpr (ahead) {
            products([&](const int i) INLINE {
                if (i % DT == DT - 1) fetch(i / DT);
            });
        } else {
            if (t > 0) {
                weigh(k0 - TILE, k_up_last, fetch);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) fetch(i);
            }
            widen_now();        // (beside the other waves' products)
        }
        if (GROUPS > 1) asm volatile("s_barrier" ::: "memory");
        if constexpr (!ahead) {
            products(nothing);
        } else {
            if (more) weigh(k0, k_up, nothing);
            widen_now();
        }
        v_less = v_less_next;
        if constexpr (S8) lds_barrier();
        else __syncthreads();       // (loads to LDS are waited for as memory is)
        if (more && (k0 < all_from || k0 + TILE - 1 > all_to)) {
            clean(v_now, k0);
            __syncthreads();
        }
    };
    const auto walk = [&](auto is_ahead) INLINE {
        for (int t = 0; t <= n; t += 2) {
            step(is_ahead, keys0, keys1, values0, values1, t);
            if (t + 1 <= n) step(is_ahead, keys1, keys0, values1, values0, t + 1);
        }
    };
    if (n) {
        if (GROUPS == 1 || wave < 4) walk(std::true_type{});
        else walk(std::false_type{});
    }

    float* const slot = SPLIT ? a.work + (((int64_t)b * blocks + j) * H + h) * parts * part_floats(DIM, BLOCK<GROUPS>) + part * part_floats(DIM, BLOCK<GROUPS>) : nullptr;
    l += other_half(l);
    int i = mine;
    asm volatile("" : "+v"(i));     // (or addresses of results are worked out before the loop, and spilled)
    if constexpr (SPLIT) {
        if (half == 0) {
            slot[wave * 32 + col] = m;
            slot[BLOCK<GROUPS> + wave * 32 + col] = l;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) slot[2 * BLOCK<GROUPS> + wave * 32 * DIM + (d * 16 + r) * 64 + lane] = o[d][r] * (S8 ? v_up : 1.0f);
    } else if (i < blk.c1) {
        const float inv = l == 0.0f ? 0.0f : (S8 ? v_up : 1.0f) / l, nothing = of_nothing(lo, hi);
        const int64_t to = ((int64_t)(h * G + i % G) * D + 4 * half) * a.ldo + s.first + i / G;
        store_type(a, [&](auto* out, auto encode) INLINE {
            auto* const column = out + to;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = 32 * d + 8 * (r / 4) + r % 4;
                    if (EXACT || row + 4 * half < D) column[row * a.ldo] = encode(l == 0.0f ? nothing : o[d][r] * inv);
                }
        });
    }
    lds_barrier();
    if (!odd_found) return;
    uint64_t* const marks = (uint64_t*)keys0.at;        // of a thread's results: those that are +inf or NaN, and those that are -inf or NaN
    if constexpr (!SPLIT) {
        static_assert(sizeof(keys0) >= 2 * THREADS * sizeof(uint64_t) && DT * 16 <= 64, "a bit for each sum of each thread");
        uint64_t plus = 0, minus = 0;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float y = o[d][r] + (l - l);
                plus |= (uint64_t)!(y < -NONE) << (d * 16 + r);
                minus |= (uint64_t)!(y > NONE) << (d * 16 + r);
            }
        marks[tid] = plus;
        marks[THREADS + tid] = minus;
    }
    __syncthreads();        // (the results are written)
    for (int i = tid; i < BLOCK<GROUPS> * DIM; i += THREADS) {
        const int row = i % DIM, c = blk.c0 + i / DIM, token = c / G;
        if (c >= blk.c1 || row >= D) continue;
        float sum = odd_sum<TYPE, TILE>(a, table, last_page, h, row, max(first, s.first_seen(a, token)), min(end - 1, s.last_seen(a, token)), all_from, all_to);
        if (fabsf(sum) <= 3.4e38f) continue;
        const int w = i / DIM / 32, at = row / 32 * 16 + row % 32 / 8 * 4 + row % 4, from = row % 8 / 4 * 32 + i / DIM % 32;      // register and lane
        if constexpr (SPLIT) {
            slot[2 * BLOCK<GROUPS> + w * 32 * DIM + at * 64 + from] += sum;
        } else {
            if (marks[w * 64 + from] >> at & 1) sum -= NONE;
            if (marks[THREADS + w * 64 + from] >> at & 1) sum += NONE;
            store_out(a, ((int64_t)(h * G + c % G) * D + row) * a.ldo + s.first + token, sum);
        }
    }
}

// Joins the parts of a block, in the order of the keys: a wave for 32 columns and 32 dims.
template <int DIM, int GROUPS>
__global__ __launch_bounds__(64) void cache_join_many(const AttendArgs a, const int blocks, const int parts)
{
    const int lane = threadIdx.x, col = lane % 32, half = lane / 32, h = blockIdx.y, w = blockIdx.x / (DIM / 32), d = blockIdx.x % (DIM / 32);
    const int b = (int)(blockIdx.z / (uint32_t)blocks), j = (int)(blockIdx.z % (uint32_t)blocks);
    const Sequence s = sequence(a, b);
    const Block blk = block_of(a, s, j, BLOCK<GROUPS>);
    const int i = blk.c0 + w * 32 + col;
    if (blk.tiles == 0 || blk.c0 + w * 32 >= blk.c1) return;
    const float* const first = a.work + (((int64_t)b * blocks + j) * a.pool.n_heads + h) * parts * part_floats(DIM, BLOCK<GROUPS>);
    float top = NONE, all = 0.0f, y[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = 0.0f;
#pragma unroll 2
    for (int x = 0; x < parts; ++x) {
        if ((int64_t)blk.tiles * x / parts == (int64_t)blk.tiles * (x + 1) / parts) continue;       // (a part of no tiles)
        const float* const p = first + x * part_floats(DIM, BLOCK<GROUPS>);
        const float m = p[w * 32 + col], l = p[BLOCK<GROUPS> + w * 32 + col], mn = fmaxf(top, m), ms = mn == NONE ? 0.0f : mn;
        const float fade = __builtin_amdgcn_exp2f(top - ms), share = __builtin_amdgcn_exp2f(m - ms);
        top = mn;
        all = all * fade + l * share;
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = y[r] * fade + p[2 * BLOCK<GROUPS> + w * 32 * DIM + (d * 16 + r) * 64 + lane] * share;
    }
    if (i >= blk.c1) return;
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    const int token = i / a.group, head = h * a.group + i % a.group;
    const float nothing = of_nothing(s.first_seen(a, token), s.last_seen(a, token));
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
        if (row < a.pool.head_dim) store_out(a, ((int64_t)head * a.pool.head_dim + row) * a.ldo + s.first + token, all == 0.0f ? nothing : y[r] * inv);
    }
}

// Blocks of 256 columns for 8 bits, where they fill the matrix instructions nearly as well as blocks of 128 do.
static bool wide_blocks(const spmm_cache_type_t type, const int64_t cols)
{
    if (type != SPMM_CACHE_S8) return false;
    return (cols + 255) / 256 * 16 <= (cols + 127) / 128 * 9;        // (at most 9 / 8 of the padded columns)
}

// How many blocks a sequence has, and workgroups a block: more than one where the device could run two for each block.
template <int GROUPS>
static int parts_of(const int64_t n_seqs, const int n_heads, const int64_t cols, const int64_t tiles, int* const blocks)
{
    *blocks = (int)((cols + BLOCK<GROUPS> - 1) / BLOCK<GROUPS>);
    const int64_t parts = ROUND<GROUPS> / (n_seqs * n_heads * *blocks);
    return (int)(parts < 2 ? 1 : parts < tiles ? parts : tiles);
}

static int64_t tiles_of(const int64_t tokens) { return (tokens + TILE - 1) / TILE; }

template <int GROUPS>
static int64_t work_bytes(const int64_t n_seqs, const int n_heads, const int dim, const int64_t cols)
{
    int blocks;
    const int64_t parts = parts_of<GROUPS>(n_seqs, n_heads, cols, ROUND<GROUPS>, &blocks);
    return parts < 2 ? 16 : 4 * n_seqs * n_heads * blocks * parts * part_floats(dim > 64 ? 128 : 64, BLOCK<GROUPS>);
}

int64_t many_work_bytes(const spmm_cache_type_t type, const int64_t n_seqs, const int n_heads, const int dim, const int64_t cols)
{
    return wide_blocks(type, cols) ? work_bytes<2>(n_seqs, n_heads, dim, cols) : work_bytes<1>(n_seqs, n_heads, dim, cols);
}

static int launch_two(const void* kernel, const dim3 grid, const dim3 block, const AttendArgs& a, int x, int y, void* stream)
{
    void* args[] = {const_cast<AttendArgs*>(&a), &x, &y};
    return (int)hipLaunchKernel(kernel, grid, block, args, 0, (hipStream_t)stream);
}

template <int DIM, spmm_cache_type_t TYPE, int GROUPS>
static int launch_typed(const AttendArgs& a, void* stream)
{
    int blocks;
    const int parts = parts_of<GROUPS>(a.batch.n_seqs, a.pool.n_heads, (int64_t)a.max_new * a.group, tiles_of(a.batch.ld_table << a.pool.page_shift), &blocks);
    const int64_t all = (int64_t)a.batch.n_seqs * a.pool.n_heads * blocks * parts;
    const bool exact = a.pool.head_dim == DIM;
    const void* const kernel =
        parts > 1 ? exact ? (const void*)cache_attend_many<DIM, TYPE, true, GROUPS, true> : (const void*)cache_attend_many<DIM, TYPE, false, GROUPS, true>
                  : exact ? (const void*)cache_attend_many<DIM, TYPE, true, GROUPS, false> : (const void*)cache_attend_many<DIM, TYPE, false, GROUPS, false>;
    const int rc = launch_two(kernel, dim3((unsigned)((all + XCDS - 1) / XCDS * XCDS)), dim3(256 * GROUPS), a, blocks, parts, stream);
    if (rc || parts < 2) return rc;
    return launch_two((const void*)cache_join_many<DIM, GROUPS>, dim3(4 * GROUPS * (DIM / 32), a.pool.n_heads, a.batch.n_seqs * blocks), dim3(64), a, blocks, parts, stream);
}

template <int DIM>
static int launch_dim(const AttendArgs& a, const spmm_cache_type_t type, void* stream)
{
    if (type == SPMM_CACHE_BF16) return launch_typed<DIM, SPMM_CACHE_BF16, 1>(a, stream);
    return wide_blocks(type, (int64_t)a.max_new * a.group) ? launch_typed<DIM, SPMM_CACHE_S8, 2>(a, stream) : launch_typed<DIM, SPMM_CACHE_S8, 1>(a, stream);
}

int launch_attend_many(const AttendArgs& a, const spmm_cache_type_t type, void* stream)
{
    return a.pool.head_dim > 64 ? launch_dim<128>(a, type, stream) : launch_dim<64>(a, type, stream);
}

}  // namespace spmm_cache
