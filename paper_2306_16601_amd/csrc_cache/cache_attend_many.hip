// Attention where a key/value head has many columns (chunks of prompts): bound by the matrix instructions and by the
// exponentials between them.
//
// A workgroup takes a block of 128 * NC columns of a sequence's head, 32 * NC for each of its four waves, and walks over
// tiles of 64 keys that all waves share through LDS (two buffers; the next tile is on its way while this one is multiplied).
// bfloat16 operands go from the pages to LDS without passing through registers, 16 bytes a lane; rows of LDS are 8 or 16 such
// chunks, whose order is turned by the row's number so that 16 rows read together lie in different banks, and the order is
// made by where a lane reads, not by where it writes.  Codes of 8 bits are widened to binary16 and multiplied by their scales
// (over a power of two for the tile) on the way.  Scores, weights and sums stay in registers: see cache_attend.h; with the
// 32x32 instruction the lane's 16 scores of a tile of 32 keys are tokens 8 h .. 8 h + 7 of each half (h = lane / 32).
// The running maximum moves only when a score exceeds it by 2^8: the weights have the room, and the sums need no scaling then.
//
// Blocks are dealt out head by head, the longest first, to one XCD after the other, so that blocks that read the same keys
// share an L2.  Where there are fewer blocks than the device can run, the tiles of all blocks are numbered and cut into equal
// runs, as in cache_attend_few, and cache_join_many joins the parts.
#include "cache_attend.h"

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;
constexpr int TILE = 64;            // keys
constexpr int CUS = 256, XCDS = 8;
constexpr float ROOM = 8.0f;

template <int NC>
constexpr int BLOCK = WAVES * 32 * NC;      // columns

template <int NC>
constexpr int PER_CU = NC > 1 ? 1 : 2;      // workgroups on a CU

__host__ __device__ inline int64_t parts_at(const int64_t items) { return ((items + 1) * 8 + 15) / 16 * 4; }      // in floats
__host__ __device__ constexpr int64_t part_floats(const int dim, const int cols) { return (int64_t)cols * (dim + 2); }

__device__ __forceinline__ int uniform(const int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(const int64_t v)
{
    return (int64_t)(uint32_t)uniform((int)v) | (int64_t)uniform((int)(v >> 32)) << 32;
}

// Sum over the threads before this one; *all: over all.  Every thread of the workgroup calls it.
__device__ __forceinline__ int64_t before(const int64_t v, int64_t* const all)
{
    __shared__ int64_t waves[WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t s = v;
    for (int i = 1; i < 64; i <<= 1) {
        const int64_t o = __shfl_up(s, i);
        if (lane >= i) s += o;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int64_t base = 0;
    *all = 0;
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) base += waves[w];
        *all += waves[w];
    }
    return base + s - v;
}

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

// the other half of the wave's value
__device__ __forceinline__ float other_half(const float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, threadIdx.x & 32 ? r[0] : r[1]);
}

// chunk of LDS, of 16 bytes, that chunk c of a row lies in: rows of 8 chunks (two rows cover the banks), or of 16
template <int CHUNKS>
__device__ __forceinline__ int turned(const int row, const int c)
{
    return CHUNKS == 16 ? c ^ (row & 15) : c ^ (row >> 1 & 7);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// The tiles of keys [64][DIM] and values [DIM][64] in 16 bits.
template <int DIM>
struct Tile {
    uint4 k[TILE * DIM / 8];
    uint4 v[DIM * TILE / 8];
};

template <int DIM, spmm_cache_type_t TYPE, bool EXACT, int NC, bool SPLIT>
__global__ __launch_bounds__(THREADS, PER_CU<NC>) void cache_attend_many(const AttendArgs a, const int blocks)
{
    constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    constexpr int KC = DIM / 8, DT = DIM / 32, KS = DIM / 16;       // chunks of a key's row, dim tiles, steps of scores
    constexpr int UNITS = DIM / 64;                                 // 16 codes that a thread widens, of keys and of values
    constexpr int CPI = DIM / 32;                                   // instructions of a wave for a tile's keys, and for its values
    __shared__ Tile<DIM> tile0, tile1;
    __shared__ int odd_found;
    __shared__ int64_t found[2];

    const int tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64), col = lane % 32, half = lane / 32;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;

    if constexpr (!EXACT) {     // what lies beyond the head's dims is never loaded
        for (int i = tid; i < TILE * DIM / 8; i += THREADS) tile0.k[i] = tile0.v[i] = tile1.k[i] = tile1.v[i] = uint4{0, 0, 0, 0};
        __syncthreads();
    }

    // what this workgroup does: block `item` of head h, tiles u0 .. u1 - 1 of it; in runs, more of them
    int64_t item, at = 0, done = 0, to = 1;
    int h = 0;
    if constexpr (SPLIT) {
        const int64_t items = (int64_t)a.batch.n_seqs * blocks;
        int64_t* const prefix = (int64_t*)a.work;
        int64_t total = 0, mine = 0, ahead = 0;
        for (int pass = 0; pass < 2; ++pass) {
            int64_t sum = 0;
            for (int64_t i0 = 0; i0 < items; i0 += THREADS) {
                const int64_t i = i0 + tid;
                if (pass == 0 || items > THREADS) {
                    mine = i < items ? (int64_t)block_of(a, sequence(a, (int)(i / blocks)), (int)(i % blocks), BLOCK<NC>).tiles * H : 0;
                    int64_t all;
                    ahead = sum + before(mine, &all);
                    sum += all;
                } else {
                    sum = total;
                }
                if (pass == 0) {
                    if (blockIdx.x == 0 && i < items) prefix[i] = ahead;
                    continue;
                }
                if (done >= ahead && done < ahead + mine) {
                    found[0] = i;
                    found[1] = done - ahead;
                }
                if (done < sum) break;
            }
            if (pass == 0) {
                total = sum;
                if (blockIdx.x == 0 && tid == 0) prefix[items] = total;
                const int64_t runs = min((int64_t)gridDim.x, total);
                if (blockIdx.x >= runs) return;
                done = blockIdx.x * total / runs;
                to = (blockIdx.x + 1) * total / runs;
            }
        }
        __syncthreads();
        item = uniform(found[0]);
        at = uniform(found[1]);
    } else {
        // XCD x takes the x-th part of all (head, sequence) pairs with their blocks
        const uint32_t all = gridDim.x / XCDS, id = blockIdx.x % XCDS * all + blockIdx.x / XCDS;
        const uint32_t pair = id / (uint32_t)blocks, j = blocks - 1 - id % (uint32_t)blocks;
        h = (int)(pair / (uint32_t)a.batch.n_seqs);
        if (h >= H) return;
        item = (int64_t)(pair % (uint32_t)a.batch.n_seqs) * blocks + j;
    }

    while (done < to) {
        const int b = (int)(item / blocks);
        const Sequence s = sequence(a, b);
        const Block blk = block_of(a, s, (int)(item % blocks), BLOCK<NC>);
        if constexpr (SPLIT) {
            if (at >= (int64_t)blk.tiles * H) {
                ++item;
                at = 0;
                continue;
            }
            h = (int)(at / blk.tiles);
        } else {
            if (blk.tiles == 0) return;
        }
        const int u0 = SPLIT ? (int)(at % blk.tiles) : 0;
        const int u1 = SPLIT ? (int)min((int64_t)blk.tiles, u0 + (to - done)) : blk.tiles;
        const int32_t* const table = a.batch.table + b * a.batch.ld_table;
        const int last_page = max(s.len - 1, 0) >> shift;

        // columns
        int lo[NC], hi[NC];
        u32x4 q[NC][KS];
        float unit[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int i = blk.c0 + (wave * NC + c) * 32 + col;
            const bool there = i < blk.c1;
            const int token = there ? i / G : 0, head = h * G + (there ? i % G : 0);
            lo[c] = s.first_seen(a, token);
            hi[c] = there ? s.last_seen(a, token) : -1;
            unit[c] = a.scale_log2;
            const __bf16* const src = a.q + ((int64_t)(s.first + token) * (H * G) + head) * D;
            float most = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int d = 16 * k + 8 * half;
                q[c][k] = there && (EXACT || d < D) ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
                if constexpr (S8) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, q[c][k]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf((float)v[j]));
                }
            }
            if constexpr (S8) {
                most = fmaxf(most, other_half(most));
                float up;
                const float down = to_unit(most, &up);
                unit[c] *= up;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, q[c][k]);
                    f16x8 w;
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = (_Float16)((float)v[j] * down);
                    q[c][k] = __builtin_bit_cast(u32x4, w);
                }
            }
        }
        const int seen_from = s.first_seen(a, blk.c0 / G), seen_to = s.last_seen(a, (blk.c1 - 1) / G);          // by some column
        const int all_from = s.first_seen(a, (blk.c1 - 1) / G), all_to = s.last_seen(a, blk.c0 / G);            // by all

        f32x16 o[NC][DT];
        float m[NC], l[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m[c] = NONE;
            l[c] = 0.0f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[c][d][i] = 0.0f;
        }

        // ---- a tile on its way to LDS ----
        const auto page_of = [&](const int key) { return (int64_t)page_in_pool(table[min(key >> shift, last_page)], a.pool.n_pages) * H + h; };

        // bfloat16: instruction j of the wave fills 1 KB, 16 bytes a lane.  The page numbers of a tile are asked for with the
        // tile before it.
        int page_k = 0, page_v[2] = {0, 0};
        const auto name = [&](const int k0) {
            if constexpr (!S8) {
                page_k = table[min((k0 + 16 * wave) >> shift, last_page)];
                page_v[0] = table[min((k0 + 8 * turned<8>(lane / 8, lane % 8)) >> shift, last_page)];
                page_v[1] = table[min((k0 + 8 * turned<8>(8 + lane / 8, lane % 8)) >> shift, last_page)];
            }
        };
        const auto fetch = [&](Tile<DIM>& t, const int k0) {
            if constexpr (!S8) {
                const int64_t slot = (((int64_t)page_in_pool(uniform(page_k), a.pool.n_pages) * H + h) << shift) + ((k0 + 16 * wave) & inside);
                const char* const k = (const char*)a.pool.k + slot * D * 2;
#pragma unroll
                for (int j = 0; j < CPI; ++j) {
                    const int row = j * (64 / KC) + lane / KC, c = turned<KC>(row, lane % KC);
                    if (EXACT || 8 * c < D)
                        __builtin_amdgcn_global_load_lds((global_void*)(k + (row * D + 8 * c) * 2), (lds_void*)(t.k + (wave * CPI + j) * 64), 16, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < CPI; ++j) {
                    const int row = (wave * CPI + j) * 8 + lane / 8, c = turned<8>((j & 1) * 8 + lane / 8, lane % 8);
                    const int64_t page = (int64_t)page_in_pool(page_v[j & 1], a.pool.n_pages) * H + h;
                    const int64_t from = ((page * D + row) << shift) + ((k0 + 8 * c) & inside);
                    if (EXACT || row < D)
                        __builtin_amdgcn_global_load_lds((global_void*)((const char*)a.pool.v + from * 2), (lds_void*)(t.v + (wave * CPI + j) * 64), 16, 0, 0);
                }
                name(k0 + TILE);
            }
        };
        // 8 bits: codes and scales in registers until the tile before has been multiplied
        u32x4 raw_k[S8 ? UNITS : 1], raw_v[S8 ? UNITS : 1];
        float k_scale[S8 ? UNITS : 1], lane_k = 0.0f, lane_v = 0.0f;
        f32x4 v_scale[S8 ? 4 : 1];
        constexpr int UPR = DIM / 16;       // units of a key's row
        const auto fetch_codes = [&](const int k0) {
            if constexpr (S8) {
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int row = (tid + THREADS * i) / UPR, d = tid % UPR * 16;
                    const int64_t slot = (page_of(k0 + row) << shift) + ((k0 + row) & inside);
                    raw_k[i] = EXACT || d < D ? *(const u32x4*)((const int8_t*)a.pool.k + slot * D + d) : u32x4{0, 0, 0, 0};
                    k_scale[i] = a.pool.k_scale[slot];
                }
                const int key = k0 + tid % 4 * 16;
                const int64_t page = page_of(key);
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int d = tid / 4 + TILE * i;
                    raw_v[i] = EXACT || d < D ? *(const u32x4*)((const int8_t*)a.pool.v + ((page * D + d) << shift) + (key & inside)) : u32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) v_scale[i] = *(const f32x4*)(a.pool.v_scale + (page << shift) + (key & inside) + 4 * i);
                const int64_t slot = (page_of(k0 + lane) << shift) + ((k0 + lane) & inside);
                lane_k = a.pool.k_scale[slot];
                lane_v = a.pool.v_scale[slot];
            }
        };
        float k_up = 1.0f, k_up_next = 1.0f, v_up = __builtin_bit_cast(float, 2u << 23), v_less = 1.0f;
        const auto widen_codes = [&](Tile<DIM>& t, const int k0) {
            if constexpr (S8) {
                const bool here = k0 + lane >= seen_from && k0 + lane <= seen_to;       // (others' scales may be anything)
                float k_down, up;
                const float k_most = here && fabsf(lane_k) <= 3.4e38f ? fabsf(lane_k) : 0.0f, v_most = here && fabsf(lane_v) <= 3.4e38f ? fabsf(lane_v) : 0.0f;
                float mk = k_most, mv = v_most;
#pragma unroll
                for (int i = 1; i < 64; i <<= 1) {
                    mk = fmaxf(mk, __shfl_xor(mk, i));
                    mv = fmaxf(mv, __shfl_xor(mv, i));
                }
                k_down = to_unit(mk, &k_up_next);
                to_unit(mv, &up);
                up = fmaxf(up, v_up);
                v_less = v_up / up;
                v_up = up;
                const float v_down = __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, up));
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int row = (tid + THREADS * i) / UPR, c = tid % UPR * 2;
                    const _Float16 f = (_Float16)(k0 + row <= seen_to && k0 + row >= seen_from ? k_scale[i] * k_down : 0.0f);
                    const f16x8 by = {f, f, f, f, f, f, f, f};
                    const f16x8 x = widen(raw_k[i][0], raw_k[i][1]) * by, y = widen(raw_k[i][2], raw_k[i][3]) * by;
                    *(f16x8*)(t.k + row * KC + turned<KC>(row, c)) = x;
                    *(f16x8*)(t.k + row * KC + turned<KC>(row, c + 1)) = y;
                }
                f16x8 by[2];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = k0 + tid % 4 * 16 + i;
                    by[i / 8][i % 8] = (_Float16)(key <= seen_to && key >= seen_from ? v_scale[i / 4][i % 4] * v_down : 0.0f);
                }
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int row = tid / 4 + TILE * i, c = tid % 4 * 2;
                    *(f16x8*)(t.v + row * 8 + turned<8>(row, c)) = widen(raw_v[i][0], raw_v[i][1]) * by[0];
                    *(f16x8*)(t.v + row * 8 + turned<8>(row, c + 1)) = widen(raw_v[i][2], raw_v[i][3]) * by[1];
                }
            }
        };

        // ---- a tile multiplied ----
        const auto multiply = [&](Tile<DIM>& t, const int k0) {
            const bool partial = k0 < all_from || k0 + TILE - 1 > all_to;
            if (partial) {
                // What no column sees may hold anything (pages are not cleared): it counts as 0, and so does what is not
                // finite where some columns see it and others do not (store_odd).
                bool mine = false;
                for (int i = tid; i < DIM * 8; i += THREADS) {
                    const int row = i / 8, c = turned<8>(row, i % 8);
                    u32x4 v = __builtin_bit_cast(u32x4, t.v[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = k0 + 8 * c + 2 * j;
                        if (key < seen_from || key > seen_to) v[j] &= 0xffff0000u;
                        if (key + 1 < seen_from || key + 1 > seen_to) v[j] &= 0xffffu;
                    }
                    const u32x4 w = S8 ? finite_half_or_zero(v) : finite_or_zero(v);
                    mine |= (v[0] != w[0]) | (v[1] != w[1]) | (v[2] != w[2]) | (v[3] != w[3]);
                    t.v[i] = __builtin_bit_cast(uint4, w);
                }
                if (mine) odd_found = 1;
                __syncthreads();
            }
            if constexpr (S8) {
                if (v_less != 1.0f) {
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int d = 0; d < DT; ++d) o[c][d] *= v_less;
                }
            }
            f32x16 sc[NC][2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[c][g][i] = 0.0f;
                // row r of a tile of scores is token r with bits 2 and 3 exchanged
                const int row = 32 * g + ((col & 0x13) | (col & 4) << 1 | (col & 8) >> 1);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const u32x4 x = __builtin_bit_cast(u32x4, t.k[row * KC + turned<KC>(row, 2 * k + half)]);
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        if constexpr (S8) sc[c][g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, q[c][k]), sc[c][g], 0, 0, 0);
                        else sc[c][g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, q[c][k]), sc[c][g], 0, 0, 0);
                    }
                }
            }
            u32x4 p[NC][4];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float by = S8 ? unit[c] * k_up : unit[c];
                if (partial) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int key = k0 + 16 * (i / 8) + 8 * half + i % 8;
                        sc[c][i / 16][i % 16] = key >= lo[c] && key <= hi[c] ? sc[c][i / 16][i % 16] : NONE;
                    }
                }
                float top = sc[c][0][0];
#pragma unroll
                for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[c][i / 16][i % 16]);
                top = fmaxf(top, other_half(top)) * by;
                if (__any(top > m[c] + ROOM)) {
                    const float mn = fmaxf(m[c], top), fade = __builtin_amdgcn_exp2f(m[c] - (mn == NONE ? 0.0f : mn));
                    m[c] = mn;
                    l[c] *= fade;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[c][d] *= fade;
                }
                const float ms = m[c] == NONE ? 0.0f : m[c];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[c][e / 2][e % 2 * 8 + j], by, -ms));
                    if constexpr (S8) {
                        f16x8 w;
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = (_Float16)x[j];
                        l[c] = sum_of(w, l[c]);
                        p[c][e] = __builtin_bit_cast(u32x4, w);
                    } else {
                        bf16x8 w;
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = (__bf16)x[j];
                        l[c] = sum_of(w, l[c]);
                        p[c][e] = __builtin_bit_cast(u32x4, w);
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int row = 32 * d + col;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u32x4 x = __builtin_bit_cast(u32x4, t.v[row * 8 + turned<8>(row, 2 * e + half)]);
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        if constexpr (S8) o[c][d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, p[c][e]), o[c][d], 0, 0, 0);
                        else o[c][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, p[c][e]), o[c][d], 0, 0, 0);
                    }
                }
            }
        };

        if (tid == 0) odd_found = 0;
        const int first = (blk.tile0 + u0) * TILE, last = (blk.tile0 + u1) * TILE;
        const int end = min(last, seen_to + 1);        // (what nobody sees has no tiles, but for one where nothing is seen)
        if (first < end) {
            if constexpr (S8) {
                fetch_codes(first);
                widen_codes(tile0, first);
            } else {
                name(first);
                fetch(tile0, first);
            }
        }
        for (int k0 = first; k0 < end; k0 += 2 * TILE) {
            k_up = k_up_next;
            __syncthreads();
            if (k0 + TILE < end) {
                if constexpr (S8) fetch_codes(k0 + TILE);
                else fetch(tile1, k0 + TILE);
            }
            multiply(tile0, k0);
            if (k0 + TILE >= end) break;
            if constexpr (S8) widen_codes(tile1, k0 + TILE);
            k_up = k_up_next;
            __syncthreads();
            if (k0 + 2 * TILE < end) {
                if constexpr (S8) fetch_codes(k0 + 2 * TILE);
                else fetch(tile0, k0 + 2 * TILE);
            }
            multiply(tile1, k0 + TILE);
            if constexpr (S8) {
                if (k0 + 2 * TILE < end) widen_codes(tile0, k0 + 2 * TILE);
            }
        }

        const bool whole = !SPLIT || (u0 == 0 && u1 == blk.tiles);
        float* const slot = SPLIT ? a.work + parts_at((int64_t)a.batch.n_seqs * blocks) + (2 * (int64_t)blockIdx.x + (u0 == 0)) * part_floats(DIM, BLOCK<NC>) : nullptr;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            l[c] += other_half(l[c]);
            int i = blk.c0 + (wave * NC + c) * 32 + col;
            asm volatile("" : "+v"(i));     // (or addresses of results are worked out before the loop, and spilled)
            if (SPLIT && !whole) {
                const int w = (wave * NC + c) * 32;
                if (half == 0) {
                    slot[w + col] = m[c];
                    slot[BLOCK<NC> + w + col] = l[c];
                }
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) slot[2 * BLOCK<NC> + w * DIM + (d * 16 + r) * 64 + lane] = o[c][d][r] * (S8 ? v_up : 1.0f);
            } else if (i < blk.c1) {
                const float inv = l[c] == 0.0f ? 0.0f : (S8 ? v_up : 1.0f) / l[c];
                const int token = i / G, head = h * G + i % G;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
                        if (EXACT || row < D) store_out(a, ((int64_t)head * D + row) * a.ldo + s.first + token, l[c] == 0.0f ? 0.0f : o[c][d][r] * inv);
                    }
            }
        }
        __syncthreads();        // (the results are written; the tiles are filled again)
        if (odd_found) {
            for (int i = tid; i < BLOCK<NC> * DIM; i += THREADS) {
                const int row = i % DIM, c = blk.c0 + i / DIM, token = c / G;
                float sum;
                if (c >= blk.c1 || row >= D || !odd_sum<TYPE, TILE>(a, table, last_page, h, row, max(first, s.first_seen(a, token)), min(end - 1, s.last_seen(a, token)), all_from, all_to, &sum))
                    continue;
                if (SPLIT && !whole) {
                    const int w = i / DIM / 32, r = row % 8;
                    slot[2 * BLOCK<NC> + w * 32 * DIM + (row / 32 * 16 + row % 32 / 8 * 4 + r % 4) * 64 + r / 4 * 32 + i / DIM % 32] = sum;
                } else {
                    store_out(a, ((int64_t)(h * G + c % G) * D + row) * a.ldo + s.first + token, sum);
                }
            }
            __syncthreads();
        }
        done += u1 - u0;
        at += u1 - u0;
        if constexpr (!SPLIT) return;
    }
}

// Joins the parts of a block that several runs had a share of, in the order of the keys: a wave for 32 columns and 32 dims.
template <int DIM, int NC>
__global__ __launch_bounds__(64) void cache_join_many(const AttendArgs a, const int blocks, const int most)
{
    const int lane = threadIdx.x, col = lane % 32, half = lane / 32, h = blockIdx.y, w = blockIdx.x / (DIM / 32), d = blockIdx.x % (DIM / 32);
    const int64_t item = blockIdx.z, items = (int64_t)a.batch.n_seqs * blocks;
    const int64_t* const prefix = (const int64_t*)a.work;
    const int64_t total = prefix[items], first = prefix[item], n = (prefix[item + 1] - first) / a.pool.n_heads;
    if (n <= 0) return;
    const int64_t runs = min((int64_t)most, total);
    const auto run_of = [&](const int64_t x) { return (int)(((x + 1) * runs - 1) / total); };
    const int w0 = run_of(first + h * n), w1 = run_of(first + (h + 1) * n - 1);
    if (w0 == w1) return;
    const Sequence s = sequence(a, (int)(item / blocks));
    const Block blk = block_of(a, s, (int)(item % blocks), BLOCK<NC>);
    const float* const parts = a.work + parts_at(items);
    const auto part_of = [&](const int x) { return parts + (2 * (int64_t)x + (x == w0)) * part_floats(DIM, BLOCK<NC>); };
    float top = NONE;
    for (int x = w0; x <= w1; ++x) top = fmaxf(top, part_of(x)[w * 32 + col]);
    const float ms = top == NONE ? 0.0f : top;
    float all = 0.0f, y[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = 0.0f;
    for (int x = w0; x <= w1; ++x) {
        const float* const p = part_of(x);
        const float share = __builtin_amdgcn_exp2f(p[w * 32 + col] - ms);
        all += p[BLOCK<NC> + w * 32 + col] * share;
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] += p[2 * BLOCK<NC> + w * 32 * DIM + (d * 16 + r) * 64 + lane] * share;
    }
    const int i = blk.c0 + w * 32 + col;
    if (i >= blk.c1) return;
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    const int token = i / a.group, head = h * a.group + i % a.group;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
        if (row < a.pool.head_dim) store_out(a, ((int64_t)head * a.pool.head_dim + row) * a.ldo + s.first + token, all == 0.0f ? 0.0f : y[r] * inv);
    }
}

// Whether there are too few blocks to go round, and how many blocks a sequence has.
template <int NC>
static bool split(const int64_t n_seqs, const int n_heads, const int64_t cols, int* const blocks)
{
    *blocks = (int)((cols + BLOCK<NC> - 1) / BLOCK<NC>);
    return n_seqs * n_heads * *blocks < 2 * CUS * PER_CU<NC>;
}

constexpr int TILES_OF_COLUMNS = 1;     // of a wave

int64_t many_work_bytes(const int64_t n_seqs, const int n_heads, const int dim, const int64_t cols)
{
    int blocks;
    if (!split<TILES_OF_COLUMNS>(n_seqs, n_heads, cols, &blocks)) return 16;
    return 4 * (parts_at(n_seqs * blocks) + (int64_t)2 * CUS * PER_CU<TILES_OF_COLUMNS> * part_floats(dim > 64 ? 128 : 64, BLOCK<TILES_OF_COLUMNS>));
}

static int launch_two(const void* kernel, const dim3 grid, const dim3 block, const AttendArgs& a, int x, int y, void* stream)
{
    void* args[] = {const_cast<AttendArgs*>(&a), &x, &y};
    return (int)hipLaunchKernel(kernel, grid, block, args, 0, (hipStream_t)stream);
}

template <int DIM, spmm_cache_type_t TYPE, int NC>
static int launch_typed(const AttendArgs& a, void* stream)
{
    int blocks;
    const bool parts = split<NC>(a.batch.n_seqs, a.pool.n_heads, (int64_t)a.max_new * a.group, &blocks), exact = a.pool.head_dim == DIM;
    const int64_t all = (int64_t)a.batch.n_seqs * a.pool.n_heads * blocks;
    if (!parts) {
        const dim3 grid((unsigned)((all + XCDS - 1) / XCDS * XCDS));
        return launch_two(exact ? (const void*)cache_attend_many<DIM, TYPE, true, NC, false> : (const void*)cache_attend_many<DIM, TYPE, false, NC, false>, grid,
                          dim3(THREADS), a, blocks, 0, stream);
    }
    constexpr int runs = CUS * PER_CU<NC>;
    const int rc = launch_two(exact ? (const void*)cache_attend_many<DIM, TYPE, true, NC, true> : (const void*)cache_attend_many<DIM, TYPE, false, NC, true>, dim3(runs),
                              dim3(THREADS), a, blocks, 0, stream);
    if (rc) return rc;
    return launch_two((const void*)cache_join_many<DIM, NC>, dim3(WAVES * NC * (DIM / 32), a.pool.n_heads, a.batch.n_seqs * blocks), dim3(64), a, blocks, runs, stream);
}

int launch_attend_many(const AttendArgs& a, const spmm_cache_type_t type, void* stream)
{
    constexpr int NC = TILES_OF_COLUMNS;
    if (a.pool.head_dim > 64) return type == SPMM_CACHE_S8 ? launch_typed<128, SPMM_CACHE_S8, NC>(a, stream) : launch_typed<128, SPMM_CACHE_BF16, NC>(a, stream);
    return type == SPMM_CACHE_S8 ? launch_typed<64, SPMM_CACHE_S8, NC>(a, stream) : launch_typed<64, SPMM_CACHE_BF16, NC>(a, stream);
}

}  // namespace spmm_cache
