// What the attention kernels share: which keys a column sees, operands of the matrix instructions from either type of cache,
// and the stores of results.
//
// o = sum_j softmax_j(scale q.k_j) v_j in one pass over the keys with a running maximum and sum.  Columns are the query heads
// of one key/value head, token by token (column c: token c / group, head c % group), so that a key that is read once serves
// all heads that share it.  Scores are computed transposed, S^T = K Q^T, with keys as the rows of the matrix instruction: a
// lane then holds scores of one column, which are, rounded to 16 bits, already its operand of O^T = V^T P^T, and nothing
// passes through LDS in between.  Which token a row of K stands for is free, and is chosen so that the consecutive k of that
// operand are consecutive tokens, which V, whose tokens are contiguous, is loaded in 16 bytes at a time.
//
// bfloat16 caches are multiplied as they are, with weights in bfloat16; the sum of the weights is that of the rounded ones, so
// that one that outweighs all others is exactly 1 (and half of the rounding's error cancels).  Codes of 8 bits are widened to
// binary16, which holds weights 8 times as exactly: for few columns by themselves, which is exact, with the keys' scales on the scores and the
// values' on the weights; for many columns times their scales, rounded once (results come out 1.07 times as far off as with one
// rounding at the end): a product for each code, where scales on scores and weights would cost one for each column.  Queries are brought to [1, 2) by a power
// of two for each column before they are narrowed to binary16, and scales, or weights times scales, by a power of two that
// follows the largest scale, so that neither leaves its range; what is small beside the largest loses at most 2^-24 of that.
#pragma once

#include "cache_internal.h"

namespace spmm_cache {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float NONE = -__builtin_inff();       // score of what is not seen

// A sequence's new tokens, and what they see.
struct Sequence {
    int first, tokens;      // first column of the batch, number of columns that are computed
    int past, len;          // position of the first new token (it may be negative, from -2^30 on); tokens in the cache
    __host__ __device__ __forceinline__ int last_seen(const AttendArgs& a, const int token) const
    {
        const int at = past + token;
        return at < 0 ? -1 : a.causal ? min(at, len - 1) : len - 1;
    }
    __host__ __device__ __forceinline__ int first_seen(const AttendArgs& a, const int token) const
    {
        // 0 .. len: a window may be as wide as an int, and positions may lie far beyond the table's width
        return a.window ? min(max((int)((uint32_t)past + token + 1), a.window) - a.window, len) : 0;
    }
};

__host__ __device__ __forceinline__ Sequence sequence(const AttendArgs& a, const int b)
{
    Sequence s;
    s.first = a.batch.q_start[b];
    const int end = a.batch.q_start[b + 1];
    s.tokens = s.first < 0 || end <= s.first ? 0 : max(min(min(end, a.T) - s.first, a.max_new), 0);     // (no difference overflows)
    s.len = tokens_of(a.batch, b, a.pool.page_shift);
    s.past = (int)max((int64_t)a.batch.kv_len[b] - ((int64_t)end - s.first), (int64_t)-(1 << 30));     // (there are at most 2^27 columns)
    return s;
}

__device__ __forceinline__ u32x4 finite_or_zero(u32x4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
    }
    return v;
}

__device__ __forceinline__ u32x4 finite_half_or_zero(u32x4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7c00u) == 0x7c00u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7c000000u) == 0x7c000000u) v[i] &= 0xffffu;
    }
    return v;
}

// four codes to binary16: 0x6400 + n is 1024 + n
__device__ __forceinline__ u32x2 widen4(uint32_t v)
{
    v ^= 0x80808080u;
    const f16x2 middle = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, v, 0x04010400u)) + middle;
    const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, v, 0x04030402u)) + middle;
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

__device__ __forceinline__ f16x8 widen(const uint32_t a, const uint32_t b)
{
    const u32x2 x = widen4(a), y = widen4(b);
    return __builtin_bit_cast(f16x8, u32x4{x[0], x[1], y[0], y[1]});
}

__device__ __forceinline__ float sum_of(const bf16x8 p, float sum)
{
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[2 * i], p[2 * i + 1]}, one, sum, false);
    return sum;
}

__device__ __forceinline__ float sum_of(const f16x8 p, float sum)
{
    const f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2(f16x2{p[2 * i], p[2 * i + 1]}, one, sum, false);
    return sum;
}

// 2^-e of the largest magnitude (exponent e), as a factor; *up: 2^e.  Both stay normal numbers.
__device__ __forceinline__ float to_unit(const float most, float* const up)
{
    const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23 & 255), 2), 252);
    *up = __builtin_bit_cast(float, (uint32_t)e << 23);
    return __builtin_bit_cast(float, (uint32_t)(254 - e) << 23);
}

// Values that are not finite, in steps of keys that not all columns see in full (all_from .. all_to are seen by all), are left
// out of the products, where they would reach all columns.  This is their sum over the keys from .. to, of one dim, which is added to the
// column's own: it is not finite if there are any (and their weights, which are positive, make no difference), else 0.
template <spmm_cache_type_t TYPE, int STEP>
__device__ __forceinline__ float odd_sum(const AttendArgs& a, const int32_t* table, const int last_page, const int h, const int row, const int from, const int to,
                                         const int all_from, const int all_to)
{
    const int shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int full_from = (all_from + STEP - 1) / STEP * STEP, full_to = (all_to + 1) / STEP * STEP - 1;
    float sum = 0.0f;
#pragma unroll 1
    for (int key = from; key <= to; ++key) {
        if (key >= full_from && key <= full_to) {
            key = full_to;
            continue;
        }
        const int64_t page = (int64_t)page_in_pool(table[min(key >> shift, last_page)], a.pool.n_pages) * a.pool.n_heads + h;
        const int64_t at = ((page * a.pool.head_dim + row) << shift) + (key & inside);
        float v;
        if constexpr (TYPE == SPMM_CACHE_S8) v = (float)((const int8_t*)a.pool.v)[at] * a.pool.v_scale[(page << shift) + (key & inside)];
        else v = (float)((const __bf16*)a.pool.v)[at];
        if (!(fabsf(v) <= 3.4e38f)) sum += v;
    }
    return sum;
}

// The result where the sum of the weights is 0: nothing is visible, or what is (from .. to) has scores of -inf alone, whose softmax is NaN.
__device__ __forceinline__ float of_nothing(const int from, const int to) { return from <= to ? __builtin_nanf("") : 0.0f; }

// store(pointer to results of the call's type, function that makes one of a value)
template <typename F>
__device__ __forceinline__ void store_type(const AttendArgs& a, const F& store)
{
    const float inv = a.out_inv, zero = (float)a.out_zero_point;
    if (a.out_type == SPMM_OUT_BF16) store((__bf16*)a.out, [](const float o) { return (__bf16)o; });
    else if (a.out_type == SPMM_OUT_F32) store((float*)a.out, [](const float o) { return o; });
    else if (a.out_type == SPMM_OUT_S8) store((int8_t*)a.out, [=](const float o) { return (int8_t)fminf(fmaxf(rintf(o * inv) + zero, -128.0f), 127.0f); });
    else store((uint8_t*)a.out, [=](const float o) { return (uint8_t)fminf(fmaxf(rintf(o * inv) + zero, 0.0f), 255.0f); });
}

__device__ __forceinline__ void store_out(const AttendArgs& a, const int64_t at, const float o)
{
    store_type(a, [&](auto* out, auto encode) { out[at] = encode(o); });
}

}  // namespace spmm_cache
