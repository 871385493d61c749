// Attention of new tokens over a paged cache.
//
// o = sum_j softmax_j(scale q.k_j) v_j in one pass over the keys with a running maximum and sum.  Columns are the query
// heads of one key/value head, token by token (column c: token c / group, head c % group), so that a key that is read once
// serves all heads that share it.  Scores are computed transposed, S^T = K Q^T, with keys as the rows of the matrix
// instruction: a lane then holds scores of one column, which are, rounded to bfloat16, already the operand of O^T = V^T P^T:
// nothing passes through LDS, and a column's maximum and sum are those of 4 lanes.  Which token a row of K stands for is
// free, and is chosen so that the operand's 8 consecutive k are 8 consecutive tokens (see key_row), which V, with its tokens
// contiguous, is loaded in 16 bytes at a time.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int COLS = 16;        // columns of a workgroup
constexpr int KEYS = 32;        // keys of a wave's step

// Rows 4 g + i of score tile t (t < 2) are tokens 8 g + 4 t + i of a step: lane group g of the result holds tokens
// 8 g .. 8 g + 7 in its two tiles, which is what it has to supply of P^T.
__device__ __forceinline__ int key_row(const int row, const int t) { return 8 * (row >> 2) + 4 * t + (row & 3); }

__device__ __forceinline__ bf16x8 widen(const u32x2 v)
{
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)(float)(int8_t)(v[i / 4] >> 8 * (i % 4));
    return r;
}

template <spmm_cache_type_t TYPE>
__device__ __forceinline__ bf16x8 load8(const void* p, const int64_t at)
{
    if constexpr (TYPE == SPMM_CACHE_S8) return widen(*(const u32x2*)((const int8_t*)p + at));
    else return *(const bf16x8*)((const __bf16*)p + at);
}

__device__ __forceinline__ bool not_finite(const __bf16 v)
{
    const float f = (float)v;
    return !(fabsf(f) <= 3.4e38f);
}

__device__ __forceinline__ float sum_of(const bf16x8 p, float sum)
{
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[2 * i], p[2 * i + 1]}, one, sum, false);
    return sum;
}

__device__ __forceinline__ void store_out(const AttendArgs& a, const int64_t at, const float o)
{
    if (a.out_type == SPMM_OUT_F32) ((float*)a.out)[at] = o;
    else if (a.out_type == SPMM_OUT_BF16) ((__bf16*)a.out)[at] = (__bf16)o;
    else {
        const float q = rintf(o * a.out_inv) + (float)a.out_zero_point;
        if (a.out_type == SPMM_OUT_S8) ((int8_t*)a.out)[at] = (int8_t)fminf(fmaxf(q, -128.0f), 127.0f);
        else ((uint8_t*)a.out)[at] = (uint8_t)fminf(fmaxf(q, 0.0f), 255.0f);
    }
}

template <int DIM, spmm_cache_type_t TYPE>
__global__ __launch_bounds__(64 * WAVES) void cache_attend(const AttendArgs a)
{
    constexpr int DT = DIM / 16, KS = DIM / 32;
    __shared__ float part[WAVES][DT * 4][64];
    __shared__ float stat[WAVES][2][COLS];
    __shared__ float weights[WAVES][KEYS][COLS];

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, g = lane / 16;
    const int b = blockIdx.z, h = blockIdx.y, D = a.pool.head_dim, G = a.group, shift = a.pool.page_shift;
    const int first = a.batch.q_start[b], end = min(a.batch.q_start[b + 1], a.T);
    const int len = tokens_of(a.batch, b, shift);
    const int past = a.batch.kv_len[b] - (a.batch.q_start[b + 1] - first);      // position of the first new token
    const int rows = min(end - first, a.max_new) * G;
    const int c0 = blockIdx.x * COLS;
    if (first < 0 || c0 >= rows) return;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;

    // what a column sees: lo .. hi
    const int c = c0 + col, token = c / G, head = h * G + c % G;
    const bool there = c < rows;
    const auto last_seen = [&](int token) { const int at = past + token; return at < 0 ? -1 : a.causal ? min(at, len - 1) : len - 1; };
    const auto first_seen = [&](int token) { return a.window ? max(past + token - a.window + 1, 0) : 0; };
    const int lo = first_seen(token), hi = there ? last_seen(token) : -1;
    const int t_first = c0 / G, t_last = (min(c0 + COLS, rows) - 1) / G;
    const int from = first_seen(t_first), to = last_seen(t_last);                      // seen by some column
    const int all_from = first_seen(t_last), all_to = last_seen(t_first);              // seen by all

    bf16x8 q[KS];
    const bf16x8 zero8 = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = 32 * s + 8 * g;
        q[s] = there && d < D ? *(const bf16x8*)(a.q + ((int64_t)(first + token) * (a.pool.n_heads * G) + head) * D + d) : zero8;
    }

    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0, 0, 0, 0};
    float m = -__builtin_inff(), l = 0.0f;

    for (int k0 = from / KEYS * KEYS + wave * KEYS; k0 <= to; k0 += WAVES * KEYS) {
        // scores
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = min(k0 + key_row(col, t), len - 1);
            const int64_t page = page_in_pool(table[key >> shift], a.pool.n_pages);
            const int64_t at = (((page * a.pool.n_heads + h) << shift) + (key & ((1 << shift) - 1))) * D;
            s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const int d = 32 * i + 8 * g;
                const bf16x8 k = d < D ? load8<TYPE>(a.pool.k, at + d) : zero8;
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[i], s[t], 0, 0, 0);
            }
        }
        // the lane's 8 tokens
        const int k8 = min(k0 + 8 * g, (len - 1) & ~7);
        const int64_t page = page_in_pool(table[k8 >> shift], a.pool.n_pages);
        const int off = k8 & ((1 << shift) - 1);
        const int64_t slot = ((page * a.pool.n_heads + h) << shift) + off;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = s[j / 4][j % 4];
            if constexpr (TYPE == SPMM_CACHE_S8) x[j] *= a.pool.k_scale[slot + j];
        }
        const bool partial = k0 < all_from || k0 + KEYS - 1 > all_to;
        uint32_t seen = 0xff;
        if (partial) {
            seen = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = k0 + 8 * g + j;
                const bool yes = key >= lo && key <= hi;
                seen |= (uint32_t)yes << j;
                x[j] = yes ? x[j] : -__builtin_inff();
            }
        }
        // running maximum and sum
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top), ms = mn == -__builtin_inff() ? 0.0f : mn * a.scale_log2;
        const float fade = __builtin_amdgcn_exp2f(m * a.scale_log2 - ms);
        m = mn;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = __builtin_amdgcn_exp2f(__fmaf_rn(x[j], a.scale_log2, -ms));
            if constexpr (TYPE == SPMM_CACHE_S8) {
                sum += x[j];
                x[j] = seen >> j & 1 ? x[j] * a.pool.v_scale[slot + j] : 0.0f;
            }
        }
        bf16x8 p;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = (__bf16)x[j];
        // the weights as they are multiplied: one that outweighs all others is then exactly 1
        if constexpr (TYPE == SPMM_CACHE_BF16) sum = sum_of(p, sum);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        l = l * fade + sum;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= fade;

        // values.  What no column sees may hold anything (pages are not cleared): it counts as 0, and so does what is not
        // finite where some columns see it and others do not; it is then added to those that do, key by key.
        bool odd = false;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int row = 16 * d + col;
            bf16x8 v = row < D ? load8<TYPE>(a.pool.v, (((page * a.pool.n_heads + h) * D + row) << shift) + off) : zero8;
            if (partial) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool is = k0 + 8 * g + j <= to && k0 + 8 * g + j >= from;
                    if (is && not_finite(v[j])) odd = true;
                    v[j] = is && !not_finite(v[j]) ? v[j] : (__bf16)0.0f;
                }
            }
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o[d], 0, 0, 0);
        }
        if (TYPE == SPMM_CACHE_BF16 && partial && __any(odd)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) weights[wave][8 * g + j][col] = seen >> j & 1 ? x[j] : -1.0f;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int i = 0; i < KEYS; ++i) {
                const float w = weights[wave][i][col];
                if (!(w < 0.0f)) {
                    const int key = k0 + i;
                    const int64_t page = page_in_pool(table[key >> shift], a.pool.n_pages);
                    const __bf16* const v = (const __bf16*)a.pool.v + (((page * a.pool.n_heads + h) * D) << shift) + (key & ((1 << shift) - 1));
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int row = 16 * d + 4 * g + e;
                            if (row < D && not_finite(v[(int64_t)row << shift])) o[d][e] += w * (float)v[(int64_t)row << shift];
                        }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }

    // the waves' parts
    if (g == 0) {
        stat[wave][0][col] = m;
        stat[wave][1][col] = l;
    }
    __syncthreads();
    float top = stat[0][0][col];
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, stat[w][0][col]);
    const float ms = top == -__builtin_inff() ? 0.0f : top * a.scale_log2;
    float total = 0.0f;
    for (int w = 0; w < WAVES; ++w) total += stat[w][1][col] * __builtin_amdgcn_exp2f(stat[w][0][col] * a.scale_log2 - ms);
    const float share = __builtin_amdgcn_exp2f(m * a.scale_log2 - ms);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][d * 4 + e][lane] = o[d][e] * share;
    __syncthreads();
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    for (int i = wave; i < DT * 4; i += WAVES) {
        const int row = 16 * (i / 4) + 4 * g + i % 4;
        float v = 0.0f;
        for (int w = 0; w < WAVES; ++w) v += part[w][i][lane];
        if (there && row < D) store_out(a, ((int64_t)head * D + row) * a.ldo + first + token, total == 0.0f ? 0.0f : v * inv);
    }
}

int64_t attend_work_bytes(int64_t, int64_t, int32_t, int32_t, int32_t, int64_t) { return 16; }

int launch_attend(const AttendArgs& a, spmm_cache_type_t type, void* stream)
{
    const dim3 grid((unsigned)(((int64_t)a.max_new * a.group + COLS - 1) / COLS), a.pool.n_heads, a.batch.n_seqs), block(64 * WAVES);
    const bool wide = a.pool.head_dim > 64;
    if (type == SPMM_CACHE_S8)
        return wide ? launch(cache_attend<128, SPMM_CACHE_S8>, grid, block, a, stream) : launch(cache_attend<64, SPMM_CACHE_S8>, grid, block, a, stream);
    return wide ? launch(cache_attend<128, SPMM_CACHE_BF16>, grid, block, a, stream) : launch(cache_attend<64, SPMM_CACHE_BF16>, grid, block, a, stream);
}

}  // namespace spmm_cache
