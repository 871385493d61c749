// New tokens into the cache: norms of the query and key heads, rotation by position, rounding, and the stores to q and to
// the pages, in one pass over the projection's output.
//
// y = x rsqrt(mean x^2 + eps) w, then pairs (a, b) -> (a c - b s, b c + a s): one read of x, one write of q, k and v, about
// ten operations a value, so memory bounds it.  x has its tokens contiguous and q and k have a head's dims contiguous, so a
// workgroup turns a tile of TOKENS tokens x one head over in LDS (binary32, 17 KB at 128 dims: 8 workgroups on a CU); the
// norm, the largest value (8-bit caches) and the rotation are then worked out by 16 lanes a token of 8 dims each, whose sums
// stay inside a row of 16 lanes.  Values keep the order of x.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int TOKENS = 32;          // of a workgroup
constexpr int THREADS = 256;
constexpr int PITCH = TOKENS + 1;   // floats of a dim's row in LDS

constexpr int NOWHERE = -1, PADDING = -2;

struct Place {      // of a new token
    int32_t turn;       // the position it is rotated to
    int32_t offset;     // in its page
    int64_t page;       // NOWHERE: not stored, PADDING: a column of no token
};

template <typename X>
__device__ __forceinline__ float value_of(const AppendArgs& a, const X x)
{
    if constexpr (sizeof(X) == 4) return x;
    else return (float)((int)x - a.x_zero_point) * a.x_scale;
}

// largest and sum over the 16 lanes of a row
__device__ __forceinline__ float row_sum(float v)
{
    for (int i = 1; i < 16; i <<= 1) v += __shfl_xor(v, i);
    return v;
}
__device__ __forceinline__ float row_max(float v)
{
    for (int i = 1; i < 16; i <<= 1) v = fmaxf(v, __shfl_xor(v, i));
    return v;
}

template <typename X, spmm_cache_type_t TYPE>
__global__ __launch_bounds__(THREADS) void cache_append(const AppendArgs a)
{
    __shared__ float tile[HEAD_DIM_MAX * PITCH];
    __shared__ Place places[TOKENS];
    __shared__ float inverse[TOKENS];       // 127 / amax, of values in 8 bits

    const int D = a.pool.head_dim, t0 = blockIdx.x * TOKENS, head = blockIdx.y, tid = threadIdx.x;
    const X* const x = (const X*)a.x + (int64_t)head * D * a.ldx;
    for (int i = tid; i < D * TOKENS; i += THREADS) {
        const int d = i / TOKENS, t = i % TOKENS;
        tile[d * PITCH + t] = t0 + t < a.T ? value_of(a, x[(int64_t)d * a.ldx + t0 + t]) : 0.0f;
    }
    if (tid < TOKENS) {
        Place p = {-1, 0, PADDING};
        const int t = t0 + tid, b = t < a.T ? sequence_of(a.batch, t) : -1;
        if (b >= 0) {
            const int at = a.batch.kv_len[b] - (a.batch.q_start[b + 1] - t);
            if (at >= 0) {
                p.turn = a.positions ? a.positions[t] : at;
                p.page = NOWHERE;
                p.offset = at & ((1 << a.pool.page_shift) - 1);
                const int i = at >> a.pool.page_shift;
                if (i < a.batch.ld_table) {
                    const int page = a.batch.table[b * a.batch.ld_table + i];
                    if ((uint32_t)page < (uint32_t)a.pool.n_pages) p.page = page;
                }
            }
        }
        places[tid] = p;
    }
    __syncthreads();

    const int q_heads = a.q_heads, kv_heads = a.pool.n_heads, shift = a.pool.page_shift;
    if (head < q_heads + kv_heads) {
        const bool is_q = head < q_heads;
        const float* const weight = is_q ? a.q_weight : a.k_weight;
        const int c = tid % 16, d0 = 8 * c, half = a.rope_dim / 2;
        const bool mine = d0 < D;
        float w[8], pw[8];       // weights of the lane's dims, and of those they are paired with
        int pair[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int d = d0 + j;
            pair[j] = !a.rope || d >= a.rope_dim ? d : a.interleaved ? d ^ 1 : d < half ? d + half : d - half;
            w[j] = mine && weight ? weight[d] : 1.0f;
            pw[j] = mine && weight ? weight[pair[j]] : 1.0f;
        }
        for (int t = tid / 16; t < TOKENS && t0 + t < a.T; t += THREADS / 16) {
            const Place p = places[t];
            float y[8], sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = mine ? tile[(d0 + j) * PITCH + t] : 0.0f;
                sum = __fmaf_rn(y[j], y[j], sum);
            }
            const float norm = weight ? 1.0f / sqrtf(row_sum(sum) / (float)D + a.eps) : 1.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = y[j] * norm * w[j];
            if (a.rope && mine) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int d = d0 + j;
                    if (d >= a.rope_dim) continue;
                    const int i = a.interleaved ? d >> 1 : d < half ? d : d - half;
                    float cs = __builtin_nanf(""), sn = cs;
                    if (p.turn >= 0 && p.turn < a.rope_len) {
                        const float* const r = a.rope + ((int64_t)p.turn * half + i) * 2;
                        cs = r[0];
                        sn = r[1];
                    }
                    const float other = tile[pair[j] * PITCH + t] * norm * pw[j];
                    y[j] = pair[j] > d ? y[j] * cs - other * sn : y[j] * cs + other * sn;
                }
            }
            if (is_q) {
                bf16x8 o;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = (__bf16)(p.page == PADDING ? 0.0f : y[j]);
                if (mine) *(bf16x8*)(a.q + ((int64_t)(t0 + t) * q_heads + head) * D + d0) = o;
            } else {
                const int64_t slot = ((p.page * kv_heads + (head - q_heads)) << shift) + p.offset;
                if constexpr (TYPE == SPMM_CACHE_S8) {
                    float most = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(y[j]));
                    most = row_max(most);
                    const float inv = most > 0.0f ? 127.0f / most : 0.0f;
                    uint32_t o[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j / 4] |= (uint32_t)(uint8_t)(int8_t)rintf(y[j] * inv) << 8 * (j % 4);
                    if (p.page >= 0) {
                        if (mine) *(u32x2*)((int8_t*)a.pool.k + slot * D + d0) = u32x2{o[0], o[1]};
                        if (c == 0) a.pool.k_scale[slot] = most / 127.0f;
                    }
                } else {
                    bf16x8 o;
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = (__bf16)y[j];
                    if (p.page >= 0 && mine) *(bf16x8*)((__bf16*)a.pool.k + slot * D + d0) = o;
                }
            }
        }
        return;
    }

    const int kv = head - q_heads - kv_heads;
    if constexpr (TYPE == SPMM_CACHE_S8) {
        for (int t = tid / 16; t < TOKENS; t += THREADS / 16) {
            float most = 0.0f;
            for (int d = tid % 16; d < D; d += 16) most = fmaxf(most, fabsf(tile[d * PITCH + t]));
            most = row_max(most);
            if (tid % 16 == 0) {
                const Place p = places[t];
                inverse[t] = most > 0.0f ? 127.0f / most : 0.0f;
                if (p.page >= 0) a.pool.v_scale[((p.page * kv_heads + kv) << shift) + p.offset] = most / 127.0f;
            }
        }
        __syncthreads();
    }
    for (int i = tid; i < D * TOKENS; i += THREADS) {
        const int d = i / TOKENS, t = i % TOKENS;
        const Place p = places[t];
        if (p.page < 0) continue;
        const int64_t at = (((p.page * kv_heads + kv) * D + d) << shift) + p.offset;
        const float y = tile[d * PITCH + t];
        if constexpr (TYPE == SPMM_CACHE_S8) ((int8_t*)a.pool.v)[at] = (int8_t)rintf(y * inverse[t]);
        else ((__bf16*)a.pool.v)[at] = (__bf16)y;
    }
}

template <typename X>
static int launch_typed(const AppendArgs& a, spmm_cache_type_t type, void* stream)
{
    const dim3 grid((a.T + TOKENS - 1) / TOKENS, a.q_heads + 2 * a.pool.n_heads);
    return type == SPMM_CACHE_S8 ? launch(cache_append<X, SPMM_CACHE_S8>, grid, dim3(THREADS), a, stream)
                                 : launch(cache_append<X, SPMM_CACHE_BF16>, grid, dim3(THREADS), a, stream);
}

int launch_append(const AppendArgs& a, spmm_out_t x_type, spmm_cache_type_t type, void* stream)
{
    switch (x_type) {
    case SPMM_OUT_F32: return launch_typed<float>(a, type, stream);
    case SPMM_OUT_S8: return launch_typed<int8_t>(a, type, stream);
    default: return launch_typed<uint8_t>(a, type, stream);
    }
}

}  // namespace spmm_cache
