// New tokens into the cache: norms of the query and key heads, rotation by position, rounding, and the stores to q and to
// the pages, in one pass over the projection's output.
//
// y = x rsqrt(mean x^2 + eps) w, then pairs (a, b) -> (a c - b s, b c + a s): one read of x, one write of q, k and v, about
// ten operations a value, so memory bounds it.
//
// cache_append_rows (heads of 64 or 128 dims, rotated in all of them or in none): a lane has a token, as x has its tokens
// contiguous, and a wave two sets of consecutive dims that lie half a head apart, so that either form of rotation pairs values
// of one lane; only the sum of the squares, and the largest value for 8 bits, go through LDS.  All loads of a head are under way
// at once (32 a lane).  q and k take 16 or 32 bytes of each token at a time.  Prompts of up to 1100 tokens, 3712 in all, 32 heads on
// 8 of 128: 36 us, 3.8 TB/s (43 us with inputs that come from HBM); 8 single tokens, 12 heads of 64: 4.2 us.
// cache_append (any other head): a workgroup turns a tile of TOKENS tokens x one head over in LDS (binary32, 17 KB at 128
// dims); 16 lanes a token of 8 dims each then work on it, whose sums stay inside a row of 16 lanes.  It took 90 us for the same
// prompts: two reads of LDS for each value are what the other form saves.
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

// the larger of two magnitudes: NaN where one of them is
__device__ __forceinline__ float larger(const float a, const float b) { return __builtin_elementwise_maximum(a, b); }

// Values whose largest is below TINY are brought up by UP first: 127 over the largest would overflow.
constexpr float TINY = 0x1p-120f, UP = 0x1p100f;

// What a token's head's values become codes by.
__device__ __forceinline__ float codes_by(const float most)
{
    return most > 0.0f ? 127.0f / (most < TINY ? most * UP : most) : 0.0f;
}

// The code of a value of a token's head; 0 where the head's values are not all finite, and so the scale is not (code times scale is NaN).
__device__ __forceinline__ int8_t code_of(const float y, const float inv)
{
    const float c = rintf(y * inv);
    return (int8_t)(fabsf(c) <= 127.0f ? c : 0.0f);
}

// largest and sum over the 16 lanes of a row
__device__ __forceinline__ float row_sum(float v)
{
    for (int i = 1; i < 16; i <<= 1) v += __shfl_xor(v, i);
    return v;
}
__device__ __forceinline__ float row_max(float v)
{
    for (int i = 1; i < 16; i <<= 1) v = larger(v, __shfl_xor(v, i));
    return v;
}

template <typename X, spmm_cache_type_t TYPE>
__global__ __launch_bounds__(THREADS) void cache_append(const AppendArgs a)
{
    __shared__ float tile[HEAD_DIM_MAX * PITCH];
    __shared__ Place places[TOKENS];
    __shared__ float inverse[TOKENS];       // of codes_by, for values in 8 bits

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
                    for (int j = 0; j < 8; ++j) most = larger(most, fabsf(y[j]));
                    most = row_max(most);
                    const float inv = codes_by(most);
                    if (most < TINY) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] *= UP;
                    }
                    uint32_t o[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j / 4] |= (uint32_t)(uint8_t)code_of(y[j], inv) << 8 * (j % 4);
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
            for (int d = tid % 16; d < D; d += 16) most = larger(most, fabsf(tile[d * PITCH + t]));
            most = row_max(most);
            if (most < TINY) {
                for (int d = tid % 16; d < D; d += 16) tile[d * PITCH + t] *= UP;
            }
            if (tid % 16 == 0) {
                const Place p = places[t];
                inverse[t] = codes_by(most);
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
        if constexpr (TYPE == SPMM_CACHE_S8) ((int8_t*)a.pool.v)[at] = code_of(y, inverse[t]);
        else ((__bf16*)a.pool.v)[at] = (__bf16)y;
    }
}

typedef const __attribute__((address_space(4))) float scalar_float;     // (read alike by all lanes: scalar loads)

constexpr int MANY = 64;            // tokens of a workgroup of cache_append_rows
constexpr int FEW_SEQS = 256;       // sequences whose columns are searched for in LDS

// y: DIM / 8 consecutive values of head `kv`'s token at `slot` (dims from d0 on), as the cache holds keys
template <spmm_cache_type_t TYPE, int N>
__device__ __forceinline__ void store_key(const AppendArgs& a, const int64_t at, const float* const y, const float inv)
{
    if constexpr (TYPE == SPMM_CACHE_S8) {
        uint32_t o[N / 4] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) o[i / 4] |= (uint32_t)(uint8_t)code_of(y[i], inv) << 8 * (i % 4);
        if constexpr (N == 16) *(u32x4*)((int8_t*)a.pool.k + at) = u32x4{o[0], o[1], o[2], o[3]};
        else *(u32x2*)((int8_t*)a.pool.k + at) = u32x2{o[0], o[1]};
    } else {
#pragma unroll
        for (int j = 0; j < N; j += 8) {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (__bf16)y[j + i];
            *(bf16x8*)((__bf16*)a.pool.k + at + j) = o;
        }
    }
}

// ROPE: 0 none, 1 pairs half a head apart, 2 neighbours
template <typename X, spmm_cache_type_t TYPE, int DIM, int ROPE>
__global__ __launch_bounds__(THREADS) void cache_append_rows(const AppendArgs a)
{
    constexpr int N = DIM / 8;          // dims of a set: wave w has N w .. and DIM / 2 + N w ..
    constexpr int WAVES = THREADS / 64;
    __shared__ int starts[FEW_SEQS + 1], lens[FEW_SEQS];
    __shared__ float part[WAVES][MANY];

    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int head = blockIdx.y, t = blockIdx.x * MANY + lane, q_heads = a.q_heads, kv_heads = a.pool.n_heads, shift = a.pool.page_shift;
    const bool turned = head < q_heads + kv_heads;

    // everything of x, and where the token goes
    const X* const x = (const X*)a.x + ((int64_t)head * DIM + N * wave) * a.ldx + min(t, a.T - 1);
    X raw[2][N];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < N; ++i) raw[s][i] = x[(int64_t)(DIM / 2 * s + i) * a.ldx];
    const int n_seqs = a.batch.n_seqs;
    const bool few = n_seqs <= FEW_SEQS;
    if (few) {
        for (int i = tid; i <= n_seqs; i += THREADS) starts[i] = a.batch.q_start[i];
        for (int i = tid; i < n_seqs; i += THREADS) lens[i] = a.batch.kv_len[i];
        __syncthreads();
    }
    Place p = {-1, 0, PADDING};
    int b = -1;
    if (t < a.T) {
        if (few) {
            int lo = 0, hi = n_seqs;        // (as in sequence_of)
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (starts[mid + 1] > t) hi = mid;
                else lo = mid + 1;
            }
            if (lo < n_seqs && t >= starts[lo]) b = lo;
        } else {
            b = sequence_of(a.batch, t);
        }
    }
    if (b >= 0) {
        const int at = (few ? lens[b] : a.batch.kv_len[b]) - ((few ? starts[b + 1] : a.batch.q_start[b + 1]) - t);
        if (at >= 0) {
            p.turn = at;
            if (ROPE && turned && a.positions) p.turn = a.positions[t];
            p.page = NOWHERE;
            p.offset = at & ((1 << shift) - 1);
            if (head >= q_heads && at >> shift < a.batch.ld_table) {
                const int page = a.batch.table[b * a.batch.ld_table + (at >> shift)];
                if ((uint32_t)page < (uint32_t)a.pool.n_pages) p.page = page;
            }
        }
    }
    // angles of the lane's pairs: N w .. of the head's, or N / 2 of each set
    float2 angle[ROPE ? N : 1];
    if constexpr (ROPE != 0) {
        if (turned) {
            const bool known = p.turn >= 0 && p.turn < a.rope_len;
            const float2* const r = (const float2*)a.rope + (int64_t)(known ? p.turn : 0) * (DIM / 2);
#pragma unroll
            for (int i = 0; i < N; ++i) angle[i] = r[ROPE == 1 ? N * wave + i : i < N / 2 ? N / 2 * wave + i : DIM / 4 + N / 2 * wave + i - N / 2];
            if (!known) {
#pragma unroll
                for (int i = 0; i < N; ++i) angle[i] = make_float2(__builtin_nanf(""), __builtin_nanf(""));
            }
        }
    }
    float y[2][N];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < N; ++i) y[s][i] = value_of(a, raw[s][i]);

    if (turned) {
        const bool is_q = head < q_heads;
        const float* const weight = is_q ? a.q_weight : a.k_weight;
        if (weight) {
            float sum = 0.0f;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < N; ++i) sum = __fmaf_rn(y[s][i], y[s][i], sum);
            part[wave][lane] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += part[w][lane];
            const float norm = 1.0f / sqrtf(sum / (float)DIM + a.eps);
            scalar_float* const w = (scalar_float*)(uintptr_t)weight + N * wave;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < N; ++i) y[s][i] = y[s][i] * norm * w[DIM / 2 * s + i];
        }
        if constexpr (ROPE == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float u = y[0][i], v = y[1][i];
                y[0][i] = u * angle[i].x - v * angle[i].y;
                y[1][i] = v * angle[i].x + u * angle[i].y;
            }
        } else if constexpr (ROPE == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int s = 2 * i / N, j = 2 * i % N;
                const float u = y[s][j], v = y[s][j + 1];
                y[s][j] = u * angle[i].x - v * angle[i].y;
                y[s][j + 1] = v * angle[i].x + u * angle[i].y;
            }
        }
        if (is_q) {
            if (t >= a.T) return;
            __bf16* const q = a.q + ((int64_t)t * q_heads + head) * DIM + N * wave;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < N; j += 8) {
                    bf16x8 o;
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = (__bf16)(p.page == PADDING ? 0.0f : y[s][j + i]);
                    *(bf16x8*)(q + DIM / 2 * s + j) = o;
                }
            return;
        }
    }
    const int kv = head - q_heads - (turned ? 0 : kv_heads);
    float inv = 0.0f;
    if constexpr (TYPE == SPMM_CACHE_S8) {
        float most = 0.0f;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i) most = larger(most, fabsf(y[s][i]));
        __syncthreads();        // (the sums have been read)
        part[wave][lane] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = larger(most, part[w][lane]);
        inv = codes_by(most);
        if (most < TINY) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < N; ++i) y[s][i] *= UP;
        }
        if (wave == 0 && p.page >= 0) (turned ? a.pool.k_scale : a.pool.v_scale)[((p.page * kv_heads + kv) << shift) + p.offset] = most / 127.0f;
    }
    if (p.page < 0) return;
    if (turned) {
        const int64_t at = (((p.page * kv_heads + kv) << shift) + p.offset) * DIM + N * wave;
        store_key<TYPE, N>(a, at, y[0], inv);
        store_key<TYPE, N>(a, at + DIM / 2, y[1], inv);
        return;
    }
    const int64_t at = (((p.page * kv_heads + kv) * DIM + N * wave) << shift) + p.offset;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t to = at + ((int64_t)(DIM / 2 * s + i) << shift);
            if constexpr (TYPE == SPMM_CACHE_S8) ((int8_t*)a.pool.v)[to] = code_of(y[s][i], inv);
            else ((__bf16*)a.pool.v)[to] = (__bf16)y[s][i];
        }
}

template <typename X, spmm_cache_type_t TYPE, int DIM>
static int launch_rows(const AppendArgs& a, void* stream)
{
    const dim3 grid((a.T + MANY - 1) / MANY, a.q_heads + 2 * a.pool.n_heads), block(THREADS);
    if (!a.rope) return launch(cache_append_rows<X, TYPE, DIM, 0>, grid, block, a, stream);
    return a.interleaved ? launch(cache_append_rows<X, TYPE, DIM, 2>, grid, block, a, stream) : launch(cache_append_rows<X, TYPE, DIM, 1>, grid, block, a, stream);
}

template <typename X, spmm_cache_type_t TYPE>
static int launch_dims(const AppendArgs& a, void* stream)
{
    if (!a.rope || a.rope_dim == a.pool.head_dim) {
        if (a.pool.head_dim == 128) return launch_rows<X, TYPE, 128>(a, stream);
        if (a.pool.head_dim == 64) return launch_rows<X, TYPE, 64>(a, stream);
    }
    return launch(cache_append<X, TYPE>, dim3((a.T + TOKENS - 1) / TOKENS, a.q_heads + 2 * a.pool.n_heads), dim3(THREADS), a, stream);
}

template <typename X>
static int launch_typed(const AppendArgs& a, spmm_cache_type_t type, void* stream)
{
    return type == SPMM_CACHE_S8 ? launch_dims<X, SPMM_CACHE_S8>(a, stream) : launch_dims<X, SPMM_CACHE_BF16>(a, stream);
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
