// Attention where a key/value head has few columns (up to 32: single tokens, drafts): bound by reading the cache once.
//
// The work is cut into units of STEP keys of a sequence's head, all units are numbered, sequence by sequence and head by
// head, and every workgroup takes an equal run of them, whatever the lengths are: as many as the device runs at a time.  A
// workgroup first sums up the sequences' units to find its run (lengths are known on the device only).  Its four waves take
// the keys of a unit in turn; a wave loads operands straight from the pages to registers, 16 bytes a lane, the next step's
// keys and page numbers while it works on this one's: 64 KB on the way for each workgroup.  Where a run covers a whole head
// the result is written; parts of a head go to scratch and are joined by cache_join, in the order of the keys.  64 tokens on
// contexts of up to 8191, 32 heads on 8 of 128: 227 us, 5.2 TB/s; with a workgroup for each head 574 us, as long as the longest
// takes.  4 x 3 tokens on 131 thousand keys in 8 bits: 216 us and 7 to join.
#include "cache_attend.h"

#include <cfloat>

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;
constexpr int COLS = 16;            // columns of a tile
// workgroups on a CU: two tiles of columns of 128 dims need more registers than half of them
template <int DIM, int NC>
constexpr int PER_CU = DIM > 64 && NC > 1 ? 1 : 2;
constexpr int CUS = 256;
// Keys, and bytes of a head's keys, up to which a workgroup takes the whole head and nothing is joined.  Whole against runs and join,
// one token, one sequence: 8 heads of 128 dims in bfloat16 512 keys 11.2 / 11.6 us, 1024 keys 18.2 / 12.0; in 8 bits 1024 keys
// 13.2 / 13.9, 2048 keys 20.5 / 14.3; 16 heads of 64 in bfloat16 1024 keys 8.1 / 10.3, 2048 keys 12.4 / 11.5, in 8 bits 8.7 / 10.8
// and 13.4 / 11.4; 64 sequences of 512 keys 23.9 / 29.3.
constexpr int64_t SHORT_KEYS = 1024, SHORT_BYTES = 128 << 10;

template <spmm_cache_type_t TYPE>
constexpr int KEYS = TYPE == SPMM_CACHE_S8 ? 64 : 32;       // of a wave's step
template <spmm_cache_type_t TYPE>
constexpr int UNIT = WAVES * KEYS<TYPE>;

// scratch: units before each sequence, then two parts for each run
__host__ __device__ inline int64_t parts_at(const int64_t n_seqs) { return ((n_seqs + 1) * 8 + 15) / 16 * 4; }      // in floats
__host__ __device__ constexpr int part_floats(const int dim, const int tiles) { return tiles * COLS * (dim + 2); }

// units of a head of sequence s, and the first one
template <spmm_cache_type_t TYPE>
__device__ __forceinline__ int units_of(const AttendArgs& a, const Sequence& s, int* const first)
{
    if (s.tokens <= 0) return 0;
    *first = s.first_seen(a, 0) / UNIT<TYPE>;
    return max(s.last_seen(a, s.tokens - 1) / UNIT<TYPE> + 1 - *first, 1);
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

// x / y, and x's share of i of n: in 32 bits where they suffice (a division of 64 takes a hundred instructions)
__device__ __forceinline__ int quotient(const int64_t x, const int64_t y)
{
    return (x | y) >> 32 ? (int)(x / y) : (int)((uint32_t)x / (uint32_t)y);
}
__device__ __forceinline__ int64_t share_of(const int64_t x, const int64_t i, const int64_t n)
{
    return x >> 22 ? x * i / n : (int64_t)((uint32_t)x * (uint32_t)i / (uint32_t)n);       // (i and n are at most 2^10)
}

__device__ __forceinline__ int uniform(const int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(const int64_t v)
{
    return (int64_t)(uint32_t)uniform((int)v) | (int64_t)uniform((int)(v >> 32)) << 32;
}

// What a step loads: DIM / 16 registers of 16 bytes a lane for keys, and for values.
//   bfloat16: rows 4 g + i of score tile t (t < 2) are tokens 8 g + 4 t + i; key register t KS + s holds dims 32 s + 8 g ..;
//   8 bits:   rows 4 g + i of score tile t (t < 4) are tokens 16 g + 4 t + i; key register t KS + s holds dims 64 s + 16 g ..;
// value register d holds, of dim 16 d + lane % 16, the lane group's tokens: 8 g .. 8 g + 7, or 16 g .. 16 g + 15.
template <int DIM, spmm_cache_type_t TYPE>
struct Loads {
    static constexpr int N = DIM / 16, BYTES = TYPE == SPMM_CACHE_S8 ? 1 : 2, TILES = TYPE == SPMM_CACHE_S8 ? 4 : 2, KS = N / TILES;
    static constexpr int CHUNK = KEYS<TYPE> / 4;        // tokens of a lane group
    static constexpr int LANE = 16 / BYTES;             // elements of a register
};

template <int DIM, spmm_cache_type_t TYPE, bool EXACT, int NC, bool WHOLE>
__global__ __launch_bounds__(THREADS, (PER_CU<DIM, NC>)) void cache_attend_few(const AttendArgs a)
{
    using L = Loads<DIM, TYPE>;
    constexpr int N = L::N, TILES = L::TILES, KS = L::KS, CHUNK = L::CHUNK, STEP = KEYS<TYPE>, ROWS = TILES * 4;
    constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    __shared__ float part[WAVES][N * 4][64];
    __shared__ float stat[WAVES][2][NC * COLS];
    __shared__ int odd_found;
    __shared__ int64_t found[2];

    const int tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64), col = lane % 16, g = lane / 16;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int n_seqs = a.batch.n_seqs;

    int b;
    int64_t at, from = 0, to = 1;
    if constexpr (WHOLE) {
        b = (int)(blockIdx.x / (uint32_t)H);
        at = blockIdx.x % (uint32_t)H;      // (the head; its units below)
    } else {
        // the run: units from .. to - 1 of all, beginning `at` units into sequence b
        int64_t* const prefix = (int64_t*)a.work;
        int64_t total = 0, sum = 0;
        int64_t mine = 0, ahead = 0;        // units of this thread's sequence, and before it
        for (int b0 = 0; b0 < n_seqs; b0 += THREADS) {
            int skip;
            mine = b0 + tid < n_seqs ? (int64_t)units_of<TYPE>(a, sequence(a, b0 + tid), &skip) * H : 0;
            int64_t all;
            ahead = total + before(mine, &all);
            if (blockIdx.x == 0 && b0 + tid < n_seqs) prefix[b0 + tid] = ahead;
            total += all;
        }
        if (blockIdx.x == 0 && tid == 0) prefix[n_seqs] = total;
        const int64_t runs = min((int64_t)gridDim.x, total);        // none is empty
        if (blockIdx.x >= runs) return;
        from = share_of(total, blockIdx.x, runs);
        to = share_of(total, blockIdx.x + 1, runs);
        for (int b0 = 0; b0 < n_seqs; b0 += THREADS) {
            if (n_seqs > THREADS) {
                int skip;
                mine = b0 + tid < n_seqs ? (int64_t)units_of<TYPE>(a, sequence(a, b0 + tid), &skip) * H : 0;
                int64_t all;
                ahead = sum + before(mine, &all);
                sum += all;
            } else {
                sum = total;
            }
            if (from >= ahead && from < ahead + mine) {
                found[0] = b0 + tid;
                found[1] = from - ahead;
            }
            if (from < sum) break;
        }
        __syncthreads();
        b = uniform((int)found[0]);
        at = uniform(found[1]);
    }

    for (int64_t done = from; done < to;) {
        const Sequence s = sequence(a, b);
        int u_first = 0;
        const int n = units_of<TYPE>(a, s, &u_first);
        if (WHOLE && n == 0) return;
        if (!WHOLE && (n == 0 || at >= (int64_t)n * H)) {
            ++b;
            at = 0;
            continue;
        }
        const int h = WHOLE ? (int)at : quotient(at, n), u0 = WHOLE ? 0 : (int)(at - (int64_t)h * n), u1 = WHOLE ? n : (int)min((int64_t)n, u0 + (to - done));
        const int32_t* const table = a.batch.table + b * a.batch.ld_table;
        const int rows = s.tokens * G;

        // columns
        int lo[NC], hi[NC], token[NC], head[NC];
        float unit[NC];         // score units: scale * log2(e), and the power of two that the queries were divided by
        u32x4 q[NC][KS * (S8 ? 2 : 1)];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int i = c * COLS + col;
            token[c] = i / G;
            head[c] = h * G + i % G;
            const bool there = i < rows;
            lo[c] = s.first_seen(a, token[c]);
            hi[c] = there ? s.last_seen(a, token[c]) : -1;
            const __bf16* const src = a.q + ((int64_t)(s.first + (there ? token[c] : 0)) * (H * G) + (there ? head[c] : 0)) * D;
            unit[c] = a.scale_log2;
            if constexpr (S8) {
                float most = 0.0f;
                u32x4 raw[KS * 2];
#pragma unroll
                for (int i8 = 0; i8 < KS * 2; ++i8) {
                    const int d = 64 * (i8 / 2) + 16 * g + 8 * (i8 % 2);
                    raw[i8] = there && d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
                    const bf16x8 v = __builtin_bit_cast(bf16x8, raw[i8]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf((float)v[j]));
                }
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                float up;
                const float down = to_unit(most, &up);
                unit[c] = fmaxf(unit[c] * up, FLT_TRUE_MIN);        // (never 0, which what is hidden, -inf, must not be multiplied by)
#pragma unroll
                for (int i8 = 0; i8 < KS * 2; ++i8) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, raw[i8]);
                    f16x8 w;
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = (_Float16)((float)v[j] * down);
                    q[c][i8] = __builtin_bit_cast(u32x4, w);
                }
            } else {
#pragma unroll
                for (int i8 = 0; i8 < KS; ++i8) {
                    const int d = 32 * i8 + 8 * g;
                    q[c][i8] = there && d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
                }
            }
        }
        const int seen_from = s.first_seen(a, 0), seen_to = s.last_seen(a, s.tokens - 1);           // by some column
        const int all_from = s.first_seen(a, s.tokens - 1), all_to = s.last_seen(a, 0);             // by all

        f32x4 o[NC][N];
        float m[NC], l[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m[c] = NONE;
            l[c] = 0.0f;
#pragma unroll
            for (int d = 0; d < N; ++d) o[c][d] = f32x4{0, 0, 0, 0};
        }
        float v_up = __builtin_bit_cast(float, 2u << 23), v_down = __builtin_bit_cast(float, 252u << 23);      // of the values' scales so far

        // (a step's pages are asked for two steps ahead, its keys one; pages beyond the last one are never named)
        const int last_page = max(s.len - 1, 0) >> shift;
        const auto page_of = [&](const int key) { return table[min(key >> shift, last_page)]; };
        const int chunk_k = CHUNK * (col >> 2), chunk_v = CHUNK * g;
        const char* const k_base = (const char*)a.pool.k + ((col & 3) * D + L::LANE * g) * L::BYTES;
        const char* const v_base = (const char*)a.pool.v + ((int64_t)col << shift) * L::BYTES;
        u32x4 k[N], v[N];
        const auto load_k = [&](const int k0, const int page) {
            const int64_t slot = (((int64_t)page_in_pool(page, a.pool.n_pages) * H + h) << shift) + ((k0 + chunk_k) & inside);
            const char* const p = k_base + slot * D * L::BYTES;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int d = (i % KS) * (DIM / KS);
                if (EXACT || d + L::LANE * g < D) k[i] = *(const u32x4*)(p + ((i / KS) * 4 * D + d) * L::BYTES);
                else k[i] = u32x4{0, 0, 0, 0};
            }
        };
        const auto load_v = [&](const int k0, const int page) {
            const int64_t head_row = ((int64_t)page_in_pool(page, a.pool.n_pages) * H + h) * D;
            const char* const p = v_base + ((head_row << shift) + ((k0 + chunk_v) & inside)) * L::BYTES;
#pragma unroll
            for (int d = 0; d < N; ++d) {
                if (EXACT || 16 * d < D) v[d] = *(const u32x4*)(p + (((int64_t)16 * d) << shift) * L::BYTES);
                else v[d] = u32x4{0, 0, 0, 0};
            }
        };

        __syncthreads();
        if (tid == 0) odd_found = 0;
        __syncthreads();
        int k0 = (u_first + u0) * UNIT<TYPE> + wave * STEP;
        const int k_end = min((u_first + u1) * UNIT<TYPE> - 1, seen_to);
        int page_k = 0, page_v = 0, page_v1 = 0;
        if (k0 <= k_end) {
            const int now = page_of(k0 + chunk_k);
            page_v = page_of(k0 + chunk_v);
            page_k = page_of(k0 + UNIT<TYPE> + chunk_k);
            page_v1 = page_of(k0 + UNIT<TYPE> + chunk_v);
            load_k(k0, now);
        }
        for (; k0 <= k_end; k0 += UNIT<TYPE>) {
            float ks[S8 ? ROWS : 1], vs[S8 ? ROWS : 1];
            load_v(k0, page_v);
            if constexpr (S8) {
                const int64_t slot = (((int64_t)page_in_pool(page_v, a.pool.n_pages) * H + h) << shift) + ((k0 + chunk_v) & inside);
#pragma unroll
                for (int i = 0; i < ROWS; i += 4) {
                    *(f32x4*)(ks + i) = *(const f32x4*)(a.pool.k_scale + slot + i);
                    *(f32x4*)(vs + i) = *(const f32x4*)(a.pool.v_scale + slot + i);
                }
            }
            // scores
            f32x4 sc[NC][TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
#pragma unroll
                for (int c = 0; c < NC; ++c) sc[c][t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const u32x4 r = k[t * KS + i];
                    if constexpr (S8) {
                        const f16x8 x = widen(r[0], r[1]), y = widen(r[2], r[3]);
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            sc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, __builtin_bit_cast(f16x8, q[c][2 * i]), sc[c][t], 0, 0, 0);
                            sc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, __builtin_bit_cast(f16x8, q[c][2 * i + 1]), sc[c][t], 0, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < NC; ++c)
                            sc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, q[c][i]), sc[c][t], 0, 0, 0);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (k0 + UNIT<TYPE> <= k_end) {
                load_k(k0 + UNIT<TYPE>, page_k);
                page_k = page_of(k0 + 2 * UNIT<TYPE> + chunk_k);
                page_v = page_v1;
                page_v1 = page_of(k0 + 2 * UNIT<TYPE> + chunk_v);
            }
            __builtin_amdgcn_sched_barrier(0);

            const bool partial = k0 < all_from || k0 + STEP - 1 > all_to;
            if constexpr (S8) {
                // the power of two that weights are divided by follows the largest scale (those that are not seen by
                // anyone may hold anything)
                if (partial) {
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        const int key = k0 + CHUNK * g + i;
                        if (key < seen_from || key > seen_to) vs[i] = 0.0f;
                        if (!(fabsf(vs[i]) <= 3.4e38f)) {
                            odd = true;
                            vs[i] = 0.0f;
                        }
                    }
                    if (__any(odd)) odd_found = 1;
                }
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) most = fmaxf(most, fabsf(vs[i]));
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                if (__any(!(most <= 3.4e38f))) most = FLT_MAX;
                float up;
                const float down = to_unit(most, &up);
                if (__any(up > v_up)) {
                    const float less = v_up * down;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int d = 0; d < N; ++d) o[c][d] *= less;
                    v_up = up;
                    v_down = down;
                }
#pragma unroll
                for (int i = 0; i < ROWS; ++i) vs[i] *= v_down;
            }
            if constexpr (S8) {
                // an infinite scale makes infinities of both signs of a key's codes, whose score is NaN
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) most = fmaxf(most, fabsf(ks[i]));
                if (__any(most > FLT_MAX)) {
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) ks[i] = fabsf(ks[i]) > FLT_MAX ? __builtin_nanf("") : ks[i];
                }
            }
            u32x4 p[NC][S8 ? 2 : 1];
            float x[NC][ROWS];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i) x[c][i] = sc[c][i / 4][i % 4] * (S8 ? ks[S8 ? i : 0] : 1.0f);
                if (partial) {
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        const int key = k0 + CHUNK * g + i;
                        x[c][i] = key >= lo[c] && key <= hi[c] ? x[c][i] : NONE;
                    }
                }
                float top = x[c][0];
#pragma unroll
                for (int i = 1; i < ROWS; ++i) top = fmaxf(top, x[c][i]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float mn = fmaxf(m[c], top), ms = mn == NONE ? 0.0f : mn * unit[c];
                const float fade = __builtin_amdgcn_exp2f(m[c] * unit[c] - ms);
                m[c] = mn;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    x[c][i] = __builtin_amdgcn_exp2f(__fmaf_rn(x[c][i], unit[c], -ms));
                    if constexpr (S8) {
                        sum += x[c][i];
                        x[c][i] *= vs[i];
                    }
                }
                if constexpr (S8) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        f16x8 w;
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = (_Float16)x[c][8 * e + j];
                        p[c][e] = __builtin_bit_cast(u32x4, w);
                    }
                } else {
                    bf16x8 w;
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = (__bf16)x[c][j];
                    p[c][0] = __builtin_bit_cast(u32x4, w);
                    sum = sum_of(w, sum);
                }
                l[c] = l[c] * fade + sum;       // (of this lane's keys)
#pragma unroll
                for (int d = 0; d < N; ++d) o[c][d] *= fade;
            }

            // values.  What no column sees may hold anything (pages are not cleared): it counts as 0, and so does what is
            // not finite where some columns see it and others do not (odd_sum).
            if constexpr (!S8) {
                if (partial) {
                    u32x4 keep;
                    u16x2 most = {0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = k0 + chunk_v + 2 * j;
                        keep[j] = (key >= seen_from && key <= seen_to ? 0xffffu : 0u) | (key + 1 >= seen_from && key + 1 <= seen_to ? 0xffff0000u : 0u);
                    }
#pragma unroll
                    for (int d = 0; d < N; ++d) {
                        v[d] &= keep;
#pragma unroll
                        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[d][j] & 0x7fff7fffu));
                    }
                    if (__any(most[0] >= 0x7f80 || most[1] >= 0x7f80)) {
                        odd_found = 1;
#pragma unroll
                        for (int d = 0; d < N; ++d) v[d] = finite_or_zero(v[d]);
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < N; ++d) {
                if constexpr (S8) {
                    const f16x8 y = widen(v[d][0], v[d][1]), z = widen(v[d][2], v[d][3]);
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, __builtin_bit_cast(f16x8, p[c][0]), o[c][d], 0, 0, 0);
                        o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(z, __builtin_bit_cast(f16x8, p[c][S8 ? 1 : 0]), o[c][d], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, p[c][0]), o[c][d], 0, 0, 0);
                }
            }
        }

        // the waves' parts together: written if they are the whole of the head, else to scratch
        const bool whole = WHOLE || (u0 == 0 && u1 == n);
        int g_out = g;
        asm volatile("" : "+v"(g_out));     // (or the addresses of results are worked out before the loop, and spilled)
        float* const slot = a.work + parts_at(n_seqs) + (2 * (int64_t)blockIdx.x + (u0 == 0)) * part_floats(DIM, NC);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            l[c] += __shfl_xor(l[c], 16);
            l[c] += __shfl_xor(l[c], 32);
            m[c] = m[c] == NONE ? NONE : m[c] * unit[c];
            if (g == 0) {
                stat[wave][0][c * COLS + col] = m[c];
                stat[wave][1][c * COLS + col] = l[c];
            }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float top = NONE, all = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stat[w][0][c * COLS + col]);
            const float ms = top == NONE ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all += stat[w][1][c * COLS + col] * __builtin_amdgcn_exp2f(stat[w][0][c * COLS + col] - ms);
            const float share = __builtin_amdgcn_exp2f(m[c] - ms) * (S8 ? v_up : 1.0f);
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[wave][d * 4 + e][lane] = o[c][d][e] * share;
            __syncthreads();
            if (odd_found) {
                const int k_first = (u_first + u0) * UNIT<TYPE>;
                for (int i = tid; i < N * 4 * 64; i += THREADS) {
                    const int reg = i / 64, row = 16 * (reg / 4) + 4 * (i % 64 / 16) + reg % 4, column = c * COLS + i % COLS, t = column / G;
                    if (column < rows && row < D)
                        part[0][reg][i % 64] += odd_sum<TYPE, STEP>(a, table, last_page, h, row, max(k_first, s.first_seen(a, t)), min(k_end, s.last_seen(a, t)), all_from, all_to);
                }
                __syncthreads();
            }
            if (!whole && tid < COLS) {
                slot[c * COLS + tid] = top;
                slot[(NC + c) * COLS + tid] = all;
            }
            const float inv = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int i = wave + WAVES * j;
                float y = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) y += part[w][i][lane];
                const int row = 16 * (i / 4) + 4 * g_out + i % 4;
                if (!whole) slot[2 * NC * COLS + (c * N * 4 + i) * 64 + lane] = y;
                else if (c * COLS + col < rows && row < D)
                    store_out(a, ((int64_t)head[c] * D + row) * a.ldo + s.first + token[c], all == 0.0f ? of_nothing(lo[c], hi[c]) : y * inv);
            }
            __syncthreads();
        }
        if constexpr (WHOLE) return;
        done += u1 - u0;
        at += u1 - u0;
    }
}

// Joins the parts of a head that several runs had a share of: those runs are w0 .. w1, in the order of the keys.
template <int DIM, int NC>
__global__ __launch_bounds__(THREADS) void cache_join(const AttendArgs a, const int most)
{
    constexpr int N = DIM / 16, ROWS = NC * N * 4, SLICE = ROWS / 4 / WAVES;      // registers of a part; of a wave of a workgroup of 4
    constexpr int PARTS = THREADS / COLS / NC;       // whose statistics are read at a time
    __shared__ float shares[PARTS][NC * COLS], tops[PARTS][NC * COLS], sums[PARTS][NC * COLS];
    const int b = blockIdx.y, h = blockIdx.x / 4, slice = blockIdx.x % 4, tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, g = lane / 16;
    const int64_t* const prefix = (const int64_t*)a.work;
    const int64_t total = prefix[a.batch.n_seqs], first = prefix[b], next = prefix[b + 1];
    const Sequence s = sequence(a, b);
    if (next <= first) return;
    const int64_t n = quotient(next - first, a.pool.n_heads), runs = min((int64_t)most, total);
    // the run that unit x lies in is the last one that begins at or before it
    const auto run_of = [&](const int64_t x) { return quotient((x + 1) * runs - 1, total); };
    const int w0 = run_of(first + h * n), w1 = run_of(first + (h + 1) * n - 1);
    if (w0 == w1) return;
    const int D = a.pool.head_dim, rows = s.tokens * a.group;
    const float* const parts = a.work + parts_at(a.batch.n_seqs);
    const auto part_of = [&](const int w) { return parts + (2 * (int64_t)w + (w == w0)) * part_floats(DIM, NC); };

    // statistics of all parts: a thread has a column of every PARTS-th
    const int c16 = tid % (NC * COLS), p0 = tid / (NC * COLS);
    float top = NONE, sum = 0.0f;
    for (int w = w0 + p0; w <= w1; w += PARTS) {
        const float* const p = part_of(w);
        const float m = p[c16], l = p[NC * COLS + c16], mn = fmaxf(top, m), ms = mn == NONE ? 0.0f : mn;
        sum = sum * __builtin_amdgcn_exp2f(top - ms) + l * __builtin_amdgcn_exp2f(m - ms);
        top = mn;
    }
    tops[p0][c16] = top;
    sums[p0][c16] = sum;
    __syncthreads();
    top = NONE;
    for (int i = 0; i < PARTS; ++i) top = fmaxf(top, tops[i][c16]);
    const float ms = top == NONE ? 0.0f : top;
    sum = 0.0f;
    for (int i = 0; i < PARTS; ++i) sum += sums[i][c16] * __builtin_amdgcn_exp2f(tops[i][c16] - ms);
    __syncthreads();
    if (p0 == 0) sums[0][c16] = sum;

    float y[SLICE];
#pragma unroll
    for (int i = 0; i < SLICE; ++i) y[i] = 0.0f;
    const int r0 = (slice * WAVES + wave) * SLICE, c = r0 / (N * 4);        // the wave's registers: all of one tile of columns
    for (int w = w0; w <= w1; w += PARTS) {
        if (w + p0 <= w1) shares[p0][c16] = __builtin_amdgcn_exp2f(part_of(w + p0)[c16] - ms);
        __syncthreads();
#pragma unroll 4
        for (int x = w; x <= min(w + PARTS - 1, w1); ++x) {
            const float* const p = part_of(x) + 2 * NC * COLS + r0 * 64 + lane;
            const float share = shares[x - w][c * COLS + col];
#pragma unroll
            for (int i = 0; i < SLICE; ++i) y[i] += p[i * 64] * share;
        }
        __syncthreads();
    }
    const float all = sums[0][c * COLS + col], inv = all == 0.0f ? 0.0f : 1.0f / all;
    const int i0 = c * COLS + col, token = i0 / a.group, head = h * a.group + i0 % a.group;
    if (i0 >= rows) return;
    const float nothing = of_nothing(s.first_seen(a, token), s.last_seen(a, token));
#pragma unroll
    for (int i = 0; i < SLICE; ++i) {
        const int j = r0 % (N * 4) + i, row = 16 * (j / 4) + 4 * g + j % 4;
        if (row < D) store_out(a, ((int64_t)head * D + row) * a.ldo + s.first + token, all == 0.0f ? nothing : y[i] * inv);
    }
}

int64_t few_work_bytes(const int64_t n_seqs, const int dim, const int64_t cols)
{
    return 4 * (parts_at(n_seqs) + (int64_t)2 * CUS * 2 * part_floats(dim > 64 ? 128 : 64, cols > COLS ? 2 : 1));
}

template <int DIM, spmm_cache_type_t TYPE, int NC, bool WHOLE>
static int launch_exact(const AttendArgs& a, const int runs, void* stream)
{
    return a.pool.head_dim == DIM ? launch(cache_attend_few<DIM, TYPE, true, NC, WHOLE>, dim3(runs), dim3(THREADS), a, stream)
                                  : launch(cache_attend_few<DIM, TYPE, false, NC, WHOLE>, dim3(runs), dim3(THREADS), a, stream);
}

template <int DIM, spmm_cache_type_t TYPE, int NC>
static int launch_typed(const AttendArgs& a, void* stream)
{
    const int64_t keys = a.batch.ld_table << a.pool.page_shift, heads = (int64_t)a.batch.n_seqs * a.pool.n_heads;
    if (keys <= SHORT_KEYS && keys * DIM * Loads<DIM, TYPE>::BYTES <= SHORT_BYTES) return launch_exact<DIM, TYPE, NC, true>(a, (int)heads, stream);
    // no more runs than units, as far as the host can say
    const int64_t most = heads * ((keys + UNIT<TYPE> - 1) / UNIT<TYPE>), full = CUS * PER_CU<DIM, NC>;
    const int runs = (int)(most < full ? most : full);
    if (const int rc = launch_exact<DIM, TYPE, NC, false>(a, runs, stream)) return rc;
    void* args[] = {const_cast<AttendArgs*>(&a), const_cast<int*>(&runs)};
    return (int)hipLaunchKernel((const void*)cache_join<DIM, NC>, dim3(4 * a.pool.n_heads, a.batch.n_seqs), dim3(THREADS), args, 0, (hipStream_t)stream);
}

template <int DIM, int NC>
static int launch_dim(const AttendArgs& a, const spmm_cache_type_t type, void* stream)
{
    return type == SPMM_CACHE_S8 ? launch_typed<DIM, SPMM_CACHE_S8, NC>(a, stream) : launch_typed<DIM, SPMM_CACHE_BF16, NC>(a, stream);
}

int launch_attend_few(const AttendArgs& a, const spmm_cache_type_t type, void* stream)
{
    const bool two = a.max_new * a.group > COLS;
    if (a.pool.head_dim > 64) return two ? launch_dim<128, 2>(a, type, stream) : launch_dim<128, 1>(a, type, stream);
    return two ? launch_dim<64, 2>(a, type, stream) : launch_dim<64, 1>(a, type, stream);
}

}  // namespace spmm_cache
