// What the kernels of attention over lists of pages share: a list's pages in LDS, and the queries of a token's heads as operands.
#pragma once

#include "cache_attend.h"

#include <cfloat>

namespace spmm_cache {

constexpr int SELECTED_WAVES = 4;
constexpr int SELECTED_THREADS = 64 * SELECTED_WAVES;
constexpr int SELECTED_COLS = 16;           // columns of a tile
constexpr int LISTED = 1024;                // pages of a list, or of a part of one, that a workgroup has in LDS

template <spmm_cache_type_t TYPE>
constexpr int SELECTED_KEYS = TYPE == SPMM_CACHE_S8 ? 64 : 32;      // of a wave's step

// A wave's operands: DIM / 16 registers of 16 bytes a lane for keys, and for values (which tokens and dims they hold: Loads in cache_attend_few.hip).
template <int DIM, spmm_cache_type_t TYPE>
struct Selected {
    static constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    static constexpr int N = DIM / 16, BYTES = S8 ? 1 : 2, TILES = S8 ? 4 : 2, KS = N / TILES, STEP = SELECTED_KEYS<TYPE>, CHUNK = STEP / 4, ROWS = TILES * 4,
                         LANE = 16 / BYTES, QUERIES = KS * (S8 ? 2 : 1),
                         TERMS = S8 ? 2 : 3, HALVES = S8 ? 2 : 1, WEIGHTS = TERMS * HALVES;     // of a weight; registers of weights of a term
};

// Waves that a list of an 8-bit cache has in launch_attend_lists, 1 or 4, or 0: it goes to the workgroups of cache_attend_selected.  One wave / four / those, us,
// 16 pages of 64 of 15 thousand tokens: 32 heads on 8 of 128 dims 128 lists 39 / 15 / 17, 256 39 / 16 / 22, 768 41 / 34 / 38, 1024 42 / 42 / 47, 1280 65 / 51 / 58,
// 2048 66 / 75 / 83, 2056 91 / 79 / 88, 4096 117 / 134 / 150, 8192 222 / 258 / 290; 64 pages 128 lists 117 / 35 / 30, 256 118 / 37 / 45, 2056 302 / 236 / 264; 16 heads of 64
// dims 256 lists 22 / 11 / 15, 1024 24 / 24 / 28, 2048 33 / 40 / 48; 32 heads on 2, which leave no columns free, 256 lists 42 / 18 / 24, 4096 162 / 183 / 177.  Waves of 128 dims
// come in rounds of 1024 lists (one on each SIMD) of 24 us after 16, workgroups take 32 ns a list after 9.  (In bfloat16, where no codes are
// widened, a wave each gained nothing: 2048 lists 127 / - / 121, 8192 472 / - / 466, measured with one term a weight.)
inline int waves_of(const spmm_cache_type_t type, const int dim, const int64_t lists, const int64_t pages)
{
    const int64_t rounds = (lists + 1023) / 1024;
    if (type != SPMM_CACHE_S8) return 0;
    if (lists >= 960 && pages <= LISTED / SELECTED_WAVES && (dim <= 64 || lists > 736 * rounds + 215)) return 1;
    return lists >= 256 && pages <= LISTED ? SELECTED_WAVES : 0;
}
int launch_attend_lists(const SelectedArgs& a, int64_t lists, bool shared, void* stream);

#if defined(__HIPCC__)

// What a column sees, none of it where a window begins behind its last token.
__device__ __forceinline__ Span seen_span(const AttendArgs& a, const int b, const int t)
{
    const Span s = span_of(a.batch, b, t, a.pool.page_shift, a.causal, a.window);
    return s.from <= s.to ? s : Span{0, -1};
}

// Page `id` of a row: its number in the pool and the position of its first token, -1 where there is no such page; *visible: whether
// some token of it is.
__device__ __forceinline__ int2 listed_page(const AttendArgs& a, const int32_t* const table, const int id, const Span span, bool* const visible)
{
    const int shift = a.pool.page_shift;
    *visible = false;
    if (id < 0 || id >= a.batch.ld_table) return int2{0, -1};
    const int first = id << shift;
    *visible = first <= span.to && first + (1 << shift) - 1 >= span.from;
    return int2{page_in_pool(table[id], a.pool.n_pages), first};
}

// The operand of a column's queries; returns what scores are multiplied by.
template <int DIM, spmm_cache_type_t TYPE, int QUERIES>
__device__ __forceinline__ float load_queries(const AttendArgs& a, const __bf16* const src, const bool there, const int D, const int g, u32x4 (&q)[QUERIES])
{
    using L = Selected<DIM, TYPE>;
    if constexpr (L::S8) {
        // (brought to [1, 2) by a power of two, as binary16 holds them)
        float most = 0.0f;
        u32x4 raw[QUERIES];
#pragma unroll
        for (int i = 0; i < QUERIES; ++i) {
            const int d = 64 * (i / 2) + 16 * g + 8 * (i % 2);
            raw[i] = there && d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
            const bf16x8 v = __builtin_bit_cast(bf16x8, raw[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf((float)v[j]));
        }
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        float up;
        const float down = to_unit(most, &up);
#pragma unroll
        for (int i = 0; i < QUERIES; ++i) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, raw[i]);
            f16x8 w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = (_Float16)((float)v[j] * down);
            q[i] = __builtin_bit_cast(u32x4, w);
        }
        return fmaxf(a.scale_log2 * up, FLT_TRUE_MIN);      // (never 0, which what is hidden, -inf, must not be multiplied by)
    } else {
#pragma unroll
        for (int i = 0; i < QUERIES; ++i) {
            const int d = 32 * i + 8 * g;
            q[i] = there && d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
        }
        return a.scale_log2;
    }
}

// A step's scores, of tokens 16 g + 4 t + i (8 bits) or 8 g + 4 t + i (bfloat16) of it.
template <int DIM, spmm_cache_type_t TYPE, int QUERIES>
__device__ __forceinline__ void selected_scores(const u32x4 (&k)[DIM / 16], const u32x4 (&q)[QUERIES], f32x4 (&sc)[Selected<DIM, TYPE>::TILES])
{
    using L = Selected<DIM, TYPE>;
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
        sc[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < L::KS; ++i) {
            const u32x4 r = k[t * L::KS + i];
            if constexpr (L::S8) {
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(r[0], r[1]), __builtin_bit_cast(f16x8, q[2 * i]), sc[t], 0, 0, 0);
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(r[2], r[3]), __builtin_bit_cast(f16x8, q[2 * i + 1]), sc[t], 0, 0, 0);
            } else {
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, q[i]), sc[t], 0, 0, 0);
            }
        }
        if constexpr (L::S8) __builtin_amdgcn_sched_barrier(0);     // (or all codes are widened first, and their registers spilled)
    }
}

// A step's values times its weights, the small terms first.
template <int DIM, spmm_cache_type_t TYPE>
__device__ __forceinline__ void selected_values(const u32x4 (&v)[DIM / 16], const u32x4 (&w)[Selected<DIM, TYPE>::WEIGHTS], f32x4 (&o)[DIM / 16])
{
    using L = Selected<DIM, TYPE>;
#pragma unroll
    for (int d = 0; d < DIM / 16; ++d) {
        if constexpr (L::S8) {
            const f16x8 low = widen(v[d][0], v[d][1]), high = widen(v[d][2], v[d][3]);
#pragma unroll
            for (int x = L::TERMS - 1; x >= 0; --x) {
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(low, __builtin_bit_cast(f16x8, w[2 * x]), o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(high, __builtin_bit_cast(f16x8, w[2 * x + 1]), o[d], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int x = L::TERMS - 1; x >= 0; --x)
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, w[x]), o[d], 0, 0, 0);
        }
        if (L::S8 && d % 2) __builtin_amdgcn_sched_barrier(0);
    }
}

// Values of tokens that are hidden, from position `first` on, which may hold anything, as 0.
template <int N>
__device__ __forceinline__ void hide_values(u32x4 (&v)[N], const int first, const Span span)
{
    u32x4 keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = first + 2 * j;
        keep[j] = (i >= span.from && i <= span.to ? 0xffffu : 0u) | (i + 1 >= span.from && i + 1 <= span.to ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int d = 0; d < N; ++d) v[d] &= keep;
}

// Weights as operands: sums of terms of 16 bits, each the rest of those before it, which hold all 24 bits of a weight in bfloat16, and 22 in binary16.  Reading
// keys and values, or widening codes, bounds these kernels, and the further terms are products with operands that are there: with one term alone, which a result is 2^-9 of the
// weights' sum off by (2^-12 in binary16), 440 lists of 32 pages in bfloat16 take 93.4 us instead of 93.3, 2048 of 16 124.7 instead of 127, 2056 of 16 in 8 bits 80.5 instead of 83.9,
// 8192 230 instead of 240.  `infinite`: whether one of the wave's weights may be (there is no rest of these).
template <typename E, int TERMS, int HALVES>
__device__ __forceinline__ void pack_terms(const float (&y)[8 * HALVES], const bool infinite, u32x4 (&w)[TERMS * HALVES])
{
    typedef E E8 __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int e = 0; e < HALVES; ++e) {
        float rest[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[j] = y[8 * e + j];
#pragma unroll
        for (int x = 0; x < TERMS; ++x) {
            E8 f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (E)rest[j];
            w[HALVES * x + e] = __builtin_bit_cast(u32x4, f);
            if (x + 1 == TERMS) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] -= (float)f[j];
            if (infinite) {
#pragma unroll
                for (int j = 0; j < 8; ++j) rest[j] = fabsf((float)f[j]) > FLT_MAX ? 0.0f : rest[j];
            }
        }
    }
}

// The power of two that weights are divided by, which follows the largest of the values' scales.
struct ValueUnit {
    bool infinite = false;      // whether one of the last ones was, of the wave's
    float up = __builtin_bit_cast(float, 2u << 23), down = __builtin_bit_cast(float, 252u << 23);
    // returns what results so far are multiplied by; vs: scales of what is visible, 0 of what is not
    template <int ROWS>
    __device__ __forceinline__ float follow(const float (&vs)[ROWS])
    {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) most = fmaxf(most, fabsf(vs[i]));
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        infinite = __any(most > FLT_MAX);
        most = fminf(most, FLT_MAX);
        float new_up;
        const float new_down = to_unit(most, &new_up);
        if (!(new_up > up)) return 1.0f;
        const float less = up * new_down;
        up = new_up;
        down = new_down;
        return less;
    }
};

// An infinite scale makes infinities of both signs of a key's codes, whose score is NaN.
template <int ROWS>
__device__ __forceinline__ void key_scales(float (&ks)[ROWS])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) most = fmaxf(most, fabsf(ks[i]));
    if (__any(most > FLT_MAX)) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) ks[i] = fabsf(ks[i]) > FLT_MAX ? __builtin_nanf("") : ks[i];
    }
}

#endif

}  // namespace spmm_cache
