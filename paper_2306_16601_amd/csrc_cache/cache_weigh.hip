// Attention that each token gets from the new ones, added up.
//
// The softmax of a column (a new token's query head) needs the largest of its scores and the sum of their powers before any key can be
// given its share, so there are two passes over the keys.  cache_weigh_stats: a workgroup has columns in its registers and a part of
// the keys goes by, with a running maximum and sum; cache_weigh_join puts the parts' statistics together; cache_weigh_add: a wave has keys in its
// registers, the columns go by, and each key's shares are summed up, first in a lane, then over the lanes of its row: every weight is
// one wave's, so that there are no atomics, and sums have one order.  Products are exact: queries are bfloat16, and so are codes of 8 bits
// once they are widened (integers up to 256 have 8 bits).
#include "cache_attend.h"

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;
constexpr int COLS = 16;            // columns of a tile
constexpr int KEYS = 32;            // of a wave's step
constexpr int STEP = KEYS * WAVES;

// A sequence's columns that count, and its tokens.
struct Counted {
    int first, tokens;      // first column of the batch, number of new tokens that count
    int len;                // tokens in the cache
    int fresh;              // first of them that is new
};

__device__ __forceinline__ Counted counted(const WeighArgs& a, const int b)
{
    const int64_t begin = a.batch.q_start[b], end = a.batch.q_start[b + 1];
    Counted s = {0, 0, tokens_of(a.batch, b, a.pool.page_shift), 0};
    if (begin < 0 || end <= begin) return s;
    const int64_t from = end - a.max_new > begin ? end - a.max_new : begin, to = end < a.T ? end : a.T;
    if (from >= to) return s;
    s.first = (int)from;
    s.tokens = (int)(to - from);
    const int64_t past = (int64_t)a.batch.kv_len[b] - (end - begin);
    s.fresh = past > 0 ? past < s.len ? (int)past : s.len : 0;
    return s;
}

__device__ __forceinline__ Span span_of(const WeighArgs& a, const int b, const int t) { return span_of(a.batch, b, t, a.pool.page_shift, a.causal, a.window); }

// Another part's largest score and sum of powers into m and l.
__device__ __forceinline__ void join(float& m, float& l, const float mo, const float lo)
{
    const float mn = fmaxf(m, mo), ms = mn == NONE ? 0.0f : mn;
    l = l * __builtin_amdgcn_exp2f(m - ms) + lo * __builtin_amdgcn_exp2f(mo - ms);
    m = mn;
}

// statistics: of column (t, query head) and part; behind them, of columns
__device__ __forceinline__ float* stat_of(const WeighArgs& a, const int64_t column, const int part) { return a.work + (column * a.parts + part) * 2; }
__device__ __forceinline__ float* joined_of(const WeighArgs& a, const int64_t column)
{
    return a.work + ((int64_t)a.T * a.group * a.pool.n_heads * a.parts + column) * 2;
}

// Operands of 32 dims of a product: queries' and keys'.  bfloat16: step s holds dims 32 s + 8 g ..; 8 bits: dims 64 (s / 2) + 16 g + 8 (s % 2) ..
template <spmm_cache_type_t TYPE>
__device__ __forceinline__ int dim_of(const int s, const int g)
{
    return TYPE == SPMM_CACHE_S8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
}

template <int KS, spmm_cache_type_t TYPE>
__device__ __forceinline__ void load_q(const WeighArgs& a, const int64_t column, const int g, bf16x8 (&q)[KS])
{
    const __bf16* const src = a.q + column * a.pool.head_dim;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = dim_of<TYPE>(s, g);
        q[s] = d < a.pool.head_dim ? *(const bf16x8*)(src + d) : bf16x8{};
    }
}

__device__ __forceinline__ bf16x8 codes(const uint32_t lo, const uint32_t hi)
{
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)(float)(int8_t)((j < 4 ? lo : hi) >> (8 * (j % 4)));
    return v;
}

// Keys k0 + 16 t + row of tile t, in registers; their scales (8 bits) for the rows that the lane has scores of.
template <int KS, spmm_cache_type_t TYPE>
struct Keys {
    bf16x8 v[2][KS];
    float scale[2][4];
    __device__ __forceinline__ void load(const WeighArgs& a, const int32_t* const table, const int h, const int k0, const int last)
    {
        const int lane = threadIdx.x % 64, row = lane % 16, g = lane / 16, shift = a.pool.page_shift, inside = (1 << shift) - 1, D = a.pool.head_dim;
        const auto slot_of = [&](const int at) {
            const int key = min(at, last);
            return (((int64_t)page_in_pool(table[key >> shift], a.pool.n_pages) * a.pool.n_heads + h) << shift) + (key & inside);
        };
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t slot = slot_of(k0 + 16 * t + row);
            if constexpr (TYPE == SPMM_CACHE_S8) {
                const int8_t* const src = (const int8_t*)a.pool.k + slot * D;
#pragma unroll
                for (int s = 0; s < KS; s += 2) {
                    const int d = dim_of<TYPE>(s, g);
                    const u32x4 x = d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
                    v[t][s] = codes(x[0], x[1]);
                    v[t][s + 1] = codes(x[2], x[3]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = a.pool.k_scale[slot_of(k0 + 16 * t + 4 * g + i)];
                    scale[t][i] = fabsf(f) <= 3.4028235e38f ? f : __builtin_nanf("");
                }
            } else {
                const __bf16* const src = (const __bf16*)a.pool.k + slot * D;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int d = dim_of<TYPE>(s, g);
                    v[t][s] = d < D ? *(const bf16x8*)(src + d) : bf16x8{};
                }
            }
        }
    }
    // scores of the lane's column: of key k0 + 16 t + 4 g + i
    __device__ __forceinline__ void scores(const bf16x8 (&q)[KS], float (&x)[2][4]) const
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 sc = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[t][s], q[s], sc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = TYPE == SPMM_CACHE_S8 ? sc[i] * scale[t][i] : sc[i];
        }
    }
};

template <int KS, spmm_cache_type_t TYPE, int TILES>
__global__ __launch_bounds__(THREADS) void cache_weigh_stats(const WeighArgs a)
{
    __shared__ float stat[WAVES][2][TILES * COLS];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, G = a.group, part = blockIdx.x % a.parts, h = blockIdx.x / a.parts, b = blockIdx.y;
    const Counted s = counted(a, b);
    const int cols = s.tokens * G;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    for (int c0 = blockIdx.z * TILES * COLS; c0 < cols; c0 += gridDim.z * TILES * COLS) {
        const int token_last = min(c0 + TILES * COLS, cols) - 1;
        const Span first = span_of(a, b, s.first + c0 / G), last = span_of(a, b, s.first + token_last / G);
        // keys that some column of these sees, and this part of them
        const int from = first.from <= first.to ? min(first.from, last.from) : last.from, to = last.to;
        const int steps = to < from ? 0 : to / STEP + 1 - from / STEP, step0 = from / STEP + (int)((int64_t)steps * part / a.parts),
                  step1 = from / STEP + (int)((int64_t)steps * (part + 1) / a.parts);
        bf16x8 q[TILES][KS];
        Span span[TILES];
        float m[TILES], l[TILES];
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
            const int c = min(c0 + x * COLS + col, cols - 1), t = s.first + c / G;
            load_q<KS, TYPE>(a, ((int64_t)t * H + h) * G + c % G, g, q[x]);
            span[x] = span_of(a, b, t);
            m[x] = NONE;
            l[x] = 0.0f;
        }
        for (int k0 = step0 * STEP + wave * KEYS; k0 < step1 * STEP && k0 <= to; k0 += STEP) {
            Keys<KS, TYPE> k;
            k.load(a, table, h, k0, max(s.len - 1, 0));
#pragma unroll
            for (int x = 0; x < TILES; ++x) {
                float sc[2][4];
                k.scores(q[x], sc);
                float top = NONE;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = k0 + 16 * t + 4 * g + i;
                        sc[t][i] = key >= span[x].from && key <= span[x].to ? sc[t][i] : NONE;
                        top = fmaxf(top, sc[t][i]);
                    }
                const float mn = fmaxf(m[x], top), ms = mn == NONE ? 0.0f : mn * a.scale_log2;
                float sum = 0.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum += __builtin_amdgcn_exp2f(__fmaf_rn(sc[t][i], a.scale_log2, -ms));
                l[x] = l[x] * __builtin_amdgcn_exp2f(m[x] * a.scale_log2 - ms) + sum;
                m[x] = mn;
            }
        }
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
            // over the lanes of a column; from here on in units of the exponent, as the powers were taken
            m[x] = m[x] == NONE ? NONE : m[x] * a.scale_log2;
#pragma unroll
            for (int o = 16; o < 64; o <<= 1) join(m[x], l[x], __shfl_xor(m[x], o), __shfl_xor(l[x], o));
            if (g == 0) {
                stat[wave][0][x * COLS + col] = m[x];
                stat[wave][1][x * COLS + col] = l[x];
            }
        }
        __syncthreads();
        for (int c = tid; c < TILES * COLS && c0 + c < cols; c += THREADS) {
            float top = NONE, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) join(top, sum, stat[w][0][c], stat[w][1][c]);
            const int i = c0 + c;
            float* const out = stat_of(a, ((int64_t)(s.first + i / G) * H + h) * G + i % G, part);
            out[0] = top;
            out[1] = sum;
        }
        __syncthreads();
    }
}

// A column's largest score, in units of the exponent, and 1 / the sum of powers.
__global__ __launch_bounds__(THREADS) void cache_weigh_join(const WeighArgs a)
{
    const int64_t column = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    if (column >= (int64_t)a.T * a.group * a.pool.n_heads) return;
    float top = NONE, sum = 0.0f;
    for (int p = 0; p < a.parts; ++p) {
        const float* const in = stat_of(a, column, p);
        join(top, sum, in[0], in[1]);
    }
    float* const out = joined_of(a, column);
    out[0] = top;
    out[1] = 1.0f / sum;
}

template <int KS, spmm_cache_type_t TYPE>
__global__ __launch_bounds__(THREADS) void cache_weigh_add(const WeighArgs a)
{
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, G = a.group, part = blockIdx.x % a.parts, h = blockIdx.x / a.parts, b = blockIdx.y;
    const int shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const Counted s = counted(a, b);
    const int cols = s.tokens * G;
    if (cols <= 0) return;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    const int steps = (s.len + STEP - 1) / STEP, step0 = (int)((int64_t)steps * part / a.parts), step1 = (int)((int64_t)steps * (part + 1) / a.parts);
    for (int k0 = step0 * STEP + wave * KEYS; k0 < step1 * STEP && k0 < s.len; k0 += STEP) {
        Keys<KS, TYPE> k;
        k.load(a, table, h, k0, s.len - 1);
        float sum[2][4] = {};
        for (int c0 = 0; c0 < cols; c0 += COLS) {
            const int c = min(c0 + col, cols - 1), t = s.first + c / G;
            const int64_t column = ((int64_t)t * H + h) * G + c % G;
            bf16x8 q[KS];
            load_q<KS, TYPE>(a, column, g, q);
            const Span span = span_of(a, b, t);
            const float* const joined = joined_of(a, column);
            const float most = joined[0], inv = joined[1];
            float sc[2][4];
            k.scores(q, sc);
#pragma unroll
            for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 16 * t2 + 4 * g + i;
                    const float p = __builtin_amdgcn_exp2f(__fmaf_rn(sc[t2][i], a.scale_log2, -most)) * inv;
                    if (key >= span.from && key <= span.to && c0 + col < cols) sum[t2][i] += p;
                }
        }
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                for (int o = 1; o < 16; o <<= 1) sum[t2][i] += __shfl_xor(sum[t2][i], o);
                const int key = k0 + 16 * t2 + 4 * g + i;
                if (col == 0 && key < s.len) {
                    const int page = table[key >> shift];
                    if ((uint32_t)page >= (uint32_t)a.pool.n_pages) continue;
                    float* const w = a.pool.weight + (((int64_t)page * H + h) << shift) + (key & inside);
                    *w = (key >= s.fresh || a.decay == 0.0f ? 0.0f : a.decay * *w) + sum[t2][i];
                }
            }
    }
}

constexpr int MANY = 4;             // tiles of columns of a workgroup, where there are many

static int64_t blocks_of(const int64_t cols) { return cols <= COLS ? 1 : (cols + MANY * COLS - 1) / (MANY * COLS); }

static int parts_of(const int page_tokens, const int64_t n_seqs, const int64_t ld_table, const int n_heads, const int64_t cols)
{
    const int64_t most = (ld_table * page_tokens + STEP - 1) / STEP, want = 2048 / (n_seqs * n_heads * blocks_of(cols));
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

int64_t weigh_work_bytes(const int page_tokens, const int64_t n_seqs, const int64_t ld_table, const int n_heads, const int64_t cols)
{
    return 8 * (int64_t)(parts_of(page_tokens, n_seqs, ld_table, n_heads, cols) + 1);     // of a column
}

template <int KS, spmm_cache_type_t TYPE>
static int launch_steps(const WeighArgs& a, const int64_t blocks, void* stream)
{
    const dim3 grid((unsigned)(a.parts * a.pool.n_heads), (unsigned)a.batch.n_seqs, (unsigned)(blocks < 65535 ? blocks : 65535));
    const bool few = (int64_t)a.max_new * a.group <= COLS;
    if (const int rc = few ? launch(cache_weigh_stats<KS, TYPE, 1>, grid, dim3(THREADS), a, stream) : launch(cache_weigh_stats<KS, TYPE, MANY>, grid, dim3(THREADS), a, stream)) return rc;
    const int64_t columns = (int64_t)a.T * a.group * a.pool.n_heads;
    if (const int rc = launch(cache_weigh_join, dim3((unsigned)((columns + THREADS - 1) / THREADS)), dim3(THREADS), a, stream)) return rc;
    return launch(cache_weigh_add<KS, TYPE>, dim3(grid.x, grid.y), dim3(THREADS), a, stream);
}

int launch_weigh(const WeighArgs& args, const spmm_cache_type_t type, void* stream)
{
    WeighArgs a = args;
    const int64_t cols = (int64_t)a.max_new * a.group, blocks = blocks_of(cols);
    a.parts = parts_of(1 << a.pool.page_shift, a.batch.n_seqs, a.batch.ld_table, a.pool.n_heads, cols);
    const int dim = a.pool.head_dim;
    if (type == SPMM_CACHE_S8) return dim > 64 ? launch_steps<4, SPMM_CACHE_S8>(a, blocks, stream) : launch_steps<2, SPMM_CACHE_S8>(a, blocks, stream);
    return dim > 96 ? launch_steps<4, SPMM_CACHE_BF16>(a, blocks, stream)
         : dim > 64 ? launch_steps<3, SPMM_CACHE_BF16>(a, blocks, stream)
         : dim > 32 ? launch_steps<2, SPMM_CACHE_BF16>(a, blocks, stream) : launch_steps<1, SPMM_CACHE_BF16>(a, blocks, stream);
}

}  // namespace spmm_cache
