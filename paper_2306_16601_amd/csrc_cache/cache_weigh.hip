// Attention that each token gets from the new ones, added up.
//
// The softmax of a column (a new token's query head) needs the largest of its scores and the sum of their powers before any key can be
// given its share, so there are two passes over the keys.  cache_weigh_stats: a workgroup has columns in its registers and a part of
// the keys goes by, with a running maximum and sum.  Where a key/value head has up to 16 columns (single tokens, drafts) that pass reads the
// cache once and memory bounds it; it keeps the scores, four bytes where the key has 2 head_dim, and cache_weigh_kept makes shares of them.  With
// more columns the scores would be more than the keys are: cache_weigh_join puts the parts' statistics together, and in
// cache_weigh_add a wave has keys in its registers, the columns go by, and each key's shares are summed up, first in a lane, then over the lanes of
// its row.  Every weight is one thread's, so that there are no atomics, and sums have one order.  Where rows share pages, as forks leave them, a page is one row's: cache_weigh_stats
// notes one of the rows that name it, whichever is last; in the next kernel the others find that it is not they, and say so; and the one row's workgroups add the shares of
// all of them, in the order of the rows (64 single tokens of 8 thousand each 162.6 us, 159.4 if no row could share: a launch; 32 tokens of two prompts 56.4, 54.8).  Products are exact: queries are bfloat16, and so are
// codes of 8 bits once they are widened (integers up to 256 have 8 bits).
//
// 64 sequences of up to 8192 tokens, 32 heads on 8 of 128 dims, a new token each: 142.6 us for the statistics (4.2 TB/s of keys; in 8 bits 121, 2.5 TB/s) and 16.4 for the
// kept scores' shares; 32 tokens of 2 prompts of 16 thousand (256 columns): 21.7 + 4.7 + 29.3 (in 8 bits 31.5 + 4.3 + 33.6), where the keys are read twice (14 us each time at the
// rate of a copy), and latencies, not the instructions, are what is left.
#include "cache_attend.h"

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;
constexpr int COLS = 16;            // columns of a tile
constexpr int MANY = 4;             // tiles of columns of a workgroup of cache_weigh_stats, where there are many
constexpr int NEAR = 2;             // tiles of 16 keys of a wave's step in cache_weigh_stats
constexpr int STEP = 16 * NEAR * WAVES;
constexpr int LISTED = 128;         // columns that are in LDS at a time
constexpr double KEPT = 1 << 30;    // most bytes of scores that are kept: a limit of scratch, beyond which a call of few columns takes the other way too

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

__device__ __forceinline__ int uniform(const int v) { return __builtin_amdgcn_readfirstlane(v); }

// Another part's largest score and sum of powers into m and l.
__device__ __forceinline__ void join(float& m, float& l, const float mo, const float lo)
{
    const float mn = fmaxf(m, mo), ms = mn == NONE ? 0.0f : mn;
    l = l * __builtin_amdgcn_exp2f(m - ms) + lo * __builtin_amdgcn_exp2f(mo - ms);
    m = mn;
}

// Of a column: its largest score, in units of the exponent, 1 / the sum of powers, and what it sees.
struct Joined {
    float most, inv;
    Span span;
};

// scratch: statistics of column (t, query head) and part; behind them scores that are kept, or statistics of columns
__device__ __forceinline__ float* stat_of(const WeighArgs& a, const int64_t column, const int part) { return a.work + (column * a.parts + part) * 2; }
__device__ __forceinline__ float* behind_stats(const WeighArgs& a) { return a.work + ((int64_t)a.T * a.group * a.pool.n_heads * a.parts + 1) / 2 * 4; }
__device__ __forceinline__ Joined* joined_of(const WeighArgs& a, const int64_t column) { return (Joined*)behind_stats(a) + column; }
__host__ __device__ __forceinline__ int64_t kept_keys(const int64_t keys) { return (keys + STEP - 1) / STEP * STEP; }
// scores of column c of a sequence's head, all keys
__device__ __forceinline__ float* kept_of(const WeighArgs& a, const int b, const int h, const int c)
{
    return behind_stats(a) + (((int64_t)b * a.pool.n_heads + h) * (a.max_new * a.group) + c) * kept_keys(a.batch.ld_table << a.pool.page_shift);
}
__device__ __forceinline__ int64_t column_of(const WeighArgs& a, const Counted& s, const int h, const int c)
{
    return ((int64_t)(s.first + c / a.group) * a.pool.n_heads + h) * a.group + c % a.group;
}

// A page's owner, by one of the threads from .. of each row that names it; then whether there are others.
__device__ __forceinline__ void own_pages(const WeighArgs& a, const int b, const Counted& s, const int from, const int step)
{
    if (s.tokens <= 0) return;
    for (int i = from; i << a.pool.page_shift < s.len; i += step) {
        const int page = a.batch.table[b * a.batch.ld_table + i];
        if ((uint32_t)page < (uint32_t)a.pool.n_pages) a.owner[page] = b;
    }
}
__device__ __forceinline__ int owner_of(const int mark) { return mark < 0 ? ~mark : mark; }
__device__ __forceinline__ void find_shared(const WeighArgs& a)
{
    const uint32_t width = (uint32_t)a.batch.ld_table, all = width * a.batch.n_seqs;        // (less than 2^31)
    for (uint32_t e = blockIdx.x * THREADS + threadIdx.x; e < all; e += gridDim.x * THREADS) {
        const int b = e / width, i = e % width, page = a.batch.table[e];
        const Counted s = counted(a, b);
        if (s.tokens <= 0 || i << a.pool.page_shift >= s.len || (uint32_t)page >= (uint32_t)a.pool.n_pages) continue;
        const int owner = owner_of(a.owner[page]);
        if (owner != b) a.owner[page] = ~owner;     // (as all that find it so write)
    }
}
__global__ __launch_bounds__(THREADS) void cache_weigh_shared(const WeighArgs a) { find_shared(a); }
// The end of what a row's workgroups go through: of its last page, where it may be another row's too, whose tokens there may be more.
__device__ __forceinline__ int end_of(const WeighArgs& a, const Counted& s)
{
    const int inside = (1 << a.pool.page_shift) - 1;
    return a.owner ? (s.len + inside) & ~inside : s.len;
}
// Whether row r, of tokens s, has page number i of a row too.
__device__ __forceinline__ bool has_page(const WeighArgs& a, const int r, const Counted& s, const int i, const int page)
{
    return s.tokens > 0 && i << a.pool.page_shift < s.len && a.batch.table[r * a.batch.ld_table + i] == page;
}

// Parts from, from + step, .. of a column's statistics, put together in their order; AHEAD of them are loaded together (behind the last one nothing).
template <int AHEAD>
__device__ __forceinline__ void join_parts(const WeighArgs& a, const int64_t column, const int from, const int step, float& top, float& sum)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    for (int p0 = from; p0 < a.parts; p0 += AHEAD * step) {
        f32x2 x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k] = *(const f32x2*)stat_of(a, column, min(p0 + k * step, a.parts - 1));
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (p0 + k * step < a.parts) join(top, sum, x[k][0], x[k][1]);
    }
}

// Operands of 32 dims of a product: queries' and keys'.  bfloat16: step s holds dims 32 s + 8 g ..; 8 bits: dims 64 (s / 2) + 16 g + 8 (s % 2) ..
template <spmm_cache_type_t TYPE>
__device__ __forceinline__ int dim_of(const int s, const int g)
{
    return TYPE == SPMM_CACHE_S8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
}

template <int KS, spmm_cache_type_t TYPE, bool EXACT>
__device__ __forceinline__ void load_q(const WeighArgs& a, const int64_t column, const int g, bf16x8 (&q)[KS])
{
    const int D = EXACT ? 32 * KS : a.pool.head_dim;
    const __bf16* const src = a.q + column * D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = dim_of<TYPE>(s, g);
        q[s] = *(const bf16x8*)(src + (EXACT || d < D ? d : 0));
        if (!EXACT && d >= D) q[s] = bf16x8{};
    }
}

__device__ __forceinline__ bf16x8 codes(const uint32_t lo, const uint32_t hi)
{
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)(float)(int8_t)((j < 4 ? lo : hi) >> (8 * (j % 4)));
    return v;
}

// Keys k0 + 16 t + row of tile t < N, as they lie in the cache; their scales (8 bits) for the rows that the lane has scores of.
template <int KS, spmm_cache_type_t TYPE, bool EXACT, int N>
struct Keys {
    static constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    static constexpr int PARTS = S8 ? (KS + 1) / 2 : KS;       // of 16 bytes
    u32x4 v[N][PARTS];
    f32x4 scale[S8 ? N : 1];
    __device__ __forceinline__ void load(const WeighArgs& a, const int32_t* const table, const int h, const int k0, const int last)
    {
        const int lane = threadIdx.x % 64, row = lane % 16, g = lane / 16, shift = a.pool.page_shift, inside = (1 << shift) - 1, D = EXACT ? 32 * KS : a.pool.head_dim;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            // (16 tokens that start at a multiple of 16 are in one page; those beyond the last lie in its page too)
            const int at = min(k0 + 16 * t, last) & ~15;
            const int64_t slot = (((int64_t)page_in_pool(table[at >> shift], a.pool.n_pages) * a.pool.n_heads + h) << shift) + (at & inside);
            const char* const src = (const char*)a.pool.k + (slot + row) * D * (S8 ? 1 : 2) + (EXACT || 16 * g < D * (S8 ? 1 : 2) ? 16 * g : 0);
#pragma unroll
            for (int s = 0; s < PARTS; ++s) {
                const bool there = EXACT || 64 * s + 16 * g < D * (S8 ? 1 : 2);
                v[t][s] = *(const u32x4*)(src + (there ? 64 * s : 0));
                if (!there) v[t][s] = u32x4{0, 0, 0, 0};
            }
            if constexpr (S8) scale[t] = *(const f32x4*)(a.pool.k_scale + slot + 4 * g);
        }
    }
    // what is not finite among the scales makes scores NaN
    __device__ __forceinline__ void ready()
    {
        if constexpr (S8)
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) scale[t][i] = fabsf(scale[t][i]) <= 3.4028235e38f ? scale[t][i] : __builtin_nanf("");
    }
    __device__ __forceinline__ bf16x8 operand(const int t, const int s) const
    {
        if constexpr (S8) return s % 2 ? codes(v[t][s / 2][2], v[t][s / 2][3]) : codes(v[t][s / 2][0], v[t][s / 2][1]);
        else return __builtin_bit_cast(bf16x8, v[t][s]);
    }
};

// Scores of TILES tiles of columns: of the lane's column and key k0 + 16 t + 4 g + i.
template <int KS, spmm_cache_type_t TYPE, bool EXACT, int N, int TILES>
__device__ __forceinline__ void scores_of(const Keys<KS, TYPE, EXACT, N>& k, const bf16x8 (&q)[TILES][KS], f32x4 (&x)[TILES][N])
{
#pragma unroll
    for (int t = 0; t < N; ++t) {
#pragma unroll
        for (int c = 0; c < TILES; ++c) x[c][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const bf16x8 w = k.operand(t, s);
#pragma unroll
            for (int c = 0; c < TILES; ++c) x[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, q[c][s], x[c][t], 0, 0, 0);
        }
        if constexpr (TYPE == SPMM_CACHE_S8)
#pragma unroll
            for (int c = 0; c < TILES; ++c) x[c][t] *= k.scale[t];
    }
}

template <int KS, spmm_cache_type_t TYPE, bool EXACT, int TILES>
__global__ __launch_bounds__(THREADS, 2) void cache_weigh_stats(const WeighArgs a)
{
    constexpr int KEYS = 16 * NEAR;     // of a wave's step
    __shared__ float stat[WAVES][2][TILES * COLS];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, G = a.group, part = blockIdx.x % a.parts, h = blockIdx.x / a.parts, b = blockIdx.y;
    const Counted s = counted(a, b);
    const int cols = s.tokens * G;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    for (int c0 = blockIdx.z * TILES * COLS; c0 < cols; c0 += gridDim.z * TILES * COLS) {
        const Span first = span_of(a, b, s.first + c0 / G), last = span_of(a, b, s.first + (min(c0 + TILES * COLS, cols) - 1) / G);
        // keys that some column of these sees, and this part of them; keys that all see
        const int from = first.from <= first.to ? min(first.from, last.from) : last.from, to = last.to;
        const int steps = to < from ? 0 : to / STEP + 1 - from / STEP;
        const int key0 = (from / STEP + (int)((int64_t)steps * part / a.parts)) * STEP, key1 = (from / STEP + (int)((int64_t)steps * (part + 1) / a.parts)) * STEP;
        const int all_from = last.from, all_to = first.to;
        bf16x8 q[TILES][KS];
        Span span[TILES];
        float m[TILES], l[TILES];
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
            const int c = min(c0 + x * COLS + col, cols - 1);
            load_q<KS, TYPE, EXACT>(a, column_of(a, s, h, c), g, q[x]);
            span[x] = span_of(a, b, s.first + c / G);
            m[x] = NONE;
            l[x] = 0.0f;
        }
        const int end = min(key1 - 1, to), last_key = max(s.len - 1, 0);
        int k0 = key0 + wave * KEYS;
        Keys<KS, TYPE, EXACT, NEAR> k, next;
        if (k0 <= end) next.load(a, table, h, k0, last_key);
        for (; k0 <= end; k0 += STEP) {
            k = next;
            if (k0 + STEP <= end) next.load(a, table, h, k0 + STEP, last_key);
            __builtin_amdgcn_sched_barrier(0);
            k.ready();
            f32x4 sc[TILES][NEAR];
            scores_of(k, q, sc);
            if (k0 < all_from || k0 + KEYS - 1 > all_to) {
#pragma unroll
                for (int x = 0; x < TILES; ++x)
#pragma unroll
                    for (int t = 0; t < NEAR; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = k0 + 16 * t + 4 * g + i;
                            sc[x][t][i] = key >= span[x].from && key <= span[x].to ? sc[x][t][i] : NONE;
                        }
            }
            if (TILES == 1 && a.keep && c0 + col < cols) {
#pragma unroll
                for (int t = 0; t < NEAR; ++t) *(f32x4*)(kept_of(a, b, h, c0 + col) + k0 + 16 * t + 4 * g) = sc[0][t];
            }
#pragma unroll
            for (int x = 0; x < TILES; ++x) {
                float top = NONE;
#pragma unroll
                for (int t = 0; t < NEAR; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[x][t][i]);
                const float mn = fmaxf(m[x], top), ms = mn == NONE ? 0.0f : mn * a.scale_log2;
                float sum = 0.0f;
#pragma unroll
                for (int t = 0; t < NEAR; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum += __builtin_amdgcn_exp2f(__fmaf_rn(sc[x][t][i], a.scale_log2, -ms));
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
            float* const out = stat_of(a, column_of(a, s, h, c0 + c), part);
            out[0] = top;
            out[1] = sum;
        }
        __syncthreads();
    }
    if (a.owner && h == 0 && blockIdx.z == 0) own_pages(a, b, s, part * THREADS + tid, a.parts * THREADS);
}

// What a key's weight is before this call's shares.
__device__ __forceinline__ float faded(const WeighArgs& a, const bool fresh, const float weight) { return fresh || a.decay == 0.0f ? 0.0f : a.decay * weight; }

// LDS of cache_weigh_kept: statistics of a row's columns, of all parts, and put together
struct alignas(16) KeptColumns {
    static constexpr int EACH = THREADS / COLS;
    float tops[EACH][COLS], sums[EACH][COLS], most[COLS], inv[COLS];
    Span spans[COLS];
    bool shared[WAVES];
};
// What the columns of row r are multiplied by and see, and whether shared() is true of any thread (it is asked once the statistics have been loaded).
template <int AHEAD, bool ASK, typename F>
__device__ __forceinline__ bool join_row(const WeighArgs& a, const int r, const Counted& s, const int h, KeptColumns& lds, const F& shared)
{
    const int tid = threadIdx.x, c = tid % COLS, p0 = tid / COLS;
    float top = NONE, sum = 0.0f;
    if (c < s.tokens * a.group) {
        join_parts<AHEAD>(a, column_of(a, s, h, c), p0, KeptColumns::EACH, top, sum);
        if (p0 == 0) lds.spans[c] = span_of(a, r, s.first + c / a.group);
    }
    lds.tops[p0][c] = top;
    lds.sums[p0][c] = sum;
    if constexpr (ASK) {
        const bool any = __any(shared());
        if (tid % 64 == 0) lds.shared[tid / 64] = any;
    }
    __syncthreads();
    if (tid < COLS) {
        for (int i = 1; i < KeptColumns::EACH; ++i) join(top, sum, lds.tops[i][c], lds.sums[i][c]);
        lds.most[c] = top;
        lds.inv[c] = 1.0f / sum;
    }
    bool all = false;
    for (int w = 0; w < (ASK ? WAVES : 0); ++w) all |= lds.shared[w];
    __syncthreads();
    return all;
}
// The shares of row r's columns at four keys; AHEAD: columns whose scores are loaded together.
template <int AHEAD>
__device__ __forceinline__ void add_kept(const WeighArgs& a, const int r, const Counted& s, const int h, const int key, const KeptColumns& lds, f32x4& add)
{
    const int cols = s.tokens * a.group;
    for (int i0 = 0; i0 < cols; i0 += AHEAD) {
        f32x4 x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k] = *(const f32x4*)(kept_of(a, r, h, min(i0 + k, cols - 1)) + key);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            // (a column behind the last one is that once more and adds nothing: were it left out, its scores would not be loaded before it is known that it is there)
            const int i = min(i0 + k, cols - 1), from = i0 + k < cols ? lds.spans[i].from : INT32_MAX, to = lds.spans[i].to;
            const float m = lds.most[i], f = lds.inv[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = __builtin_amdgcn_exp2f(__fmaf_rn(x[k][j], a.scale_log2, -m)) * f;
                add[j] += key + j >= from && key + j <= to ? p : 0.0f;
            }
        }
    }
}

// Shares of kept scores: a thread has four keys, in one page.  ROWS: there are several, which may share pages.
template <bool ROWS>
__global__ __launch_bounds__(THREADS, ROWS ? 8 : 1) void cache_weigh_kept(const WeighArgs a)
{
    __shared__ KeptColumns lds;
    const int h = blockIdx.y, b = blockIdx.z, shift = a.pool.page_shift;
    const Counted own = counted(a, b);
    const int end = end_of(a, own), first = blockIdx.x * THREADS * 4, key = first + threadIdx.x * 4;
    if (own.tokens <= 0 || first >= end) return;
    const int page = key < end ? a.batch.table[b * a.batch.ld_table + (key >> shift)] : -1;
    bool mine = (uint32_t)page < (uint32_t)a.pool.n_pages, shared = false;
    const bool several = join_row<8, ROWS>(a, b, own, h, lds, [&] {
        if (mine) {
            const int mark = a.owner[page];
            mine = owner_of(mark) == b;
            shared = mine && mark < 0;
        }
        return shared;
    });
    float* const out = a.pool.weight + (((int64_t)page * a.pool.n_heads + h) << shift) + (key & ((1 << shift) - 1));
    f32x4 add = {0, 0, 0, 0};
    if (!ROWS || !several) {
        if (!mine || key >= own.len) return;
        f32x4 w = *(const f32x4*)out;
        add_kept<4>(a, b, own, h, key, lds, add);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = key + j < own.len ? faded(a, key + j >= own.fresh, w[j]) + add[j] : w[j];
        *(f32x4*)out = w;
        return;
    }
    int held = 0, fresh = 0;        // a bit a key
#pragma unroll 1
    for (int r = 0; r < a.batch.n_seqs; ++r) {
        const Counted s = counted(a, r);
        const bool takes = mine && (r == b || (shared && has_page(a, r, s, key >> shift, page)));
        if (!__syncthreads_or(takes)) continue;     // (and the last row's numbers have been read)
        join_row<2, false>(a, r, s, h, lds, [] { return false; });
        if (!takes) continue;
        add_kept<2>(a, r, s, h, key, lds, add);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            held |= (key + j < s.len) << j;
            fresh |= (key + j < s.len && key + j >= s.fresh) << j;
        }
    }
    if (!mine) return;
    f32x4 w = *(const f32x4*)out;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = held >> j & 1 ? faded(a, fresh >> j & 1, w[j]) + add[j] : w[j];
    *(f32x4*)out = w;
}

__global__ __launch_bounds__(THREADS) void cache_weigh_join(const WeighArgs a)
{
    if (a.owner) find_shared(a);
    const int64_t column = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    if (column >= (int64_t)a.T * a.group * a.pool.n_heads) return;
    const int t = (int)(column / (a.group * a.pool.n_heads)), b = sequence_near(a.batch, t);
    if (b < 0) return;
    float top = NONE, sum = 0.0f;
    join_parts<8>(a, column, 0, 1, top, sum);
    *joined_of(a, column) = Joined{top, 1.0f / sum, span_of(a, b, t)};
}

// What columns go by with, in LDS: queries (16 bytes between rows, so that the lanes of a tile read from all banks), and numbers.
template <int KS>
struct Columns {
    static constexpr int PITCH = 32 * KS + 8;
    __bf16 q[LISTED][PITCH];
    Joined joined[LISTED];
    int64_t id[LISTED];
};

// FAR: tiles of 16 keys of a wave's step
template <int KS, spmm_cache_type_t TYPE, bool EXACT, int FAR>
__global__ __launch_bounds__(THREADS, 2) void cache_weigh_add(const WeighArgs a)
{
    constexpr int KEYS = 16 * FAR;      // of a wave's step
    constexpr int TILES = FAR == 1 ? 4 : 1, TILED = TILES * COLS;      // tiles of columns that are multiplied together
    __shared__ Columns<KS> columns;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, G = a.group, h = blockIdx.y, b = blockIdx.z, shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int D = EXACT ? 32 * KS : a.pool.head_dim;
    const Counted own = counted(a, b);
    if (own.tokens <= 0 || own.len == 0) return;       // (keys are loaded ahead: of a row without tokens there would be none, nor a page)
    const int end = end_of(a, own);
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    const int stride = gridDim.x * KEYS * WAVES;
    int in_lds = -1;        // the row whose columns are in LDS, where all of them are
    // whose a block's pages are, a lane a page, the same in all waves: looked up two blocks ahead, and one
    const auto page_of = [&](const int block) {
        const int at = (block >> shift) + lane;
        return a.owner && lane < max((KEYS * WAVES) >> shift, 1) && at << shift < end ? table[at] : -1;
    };
    const auto mark_of = [&](const int page) { return (uint32_t)page < (uint32_t)a.pool.n_pages && a.owner ? a.owner[page] : ~(1 << 30); };     // (no row's)
    int page = page_of(blockIdx.x * KEYS * WAVES), mark = mark_of(page);
    page = page_of(blockIdx.x * KEYS * WAVES + stride);
    Keys<KS, TYPE, EXACT, FAR> k, next;
    next.load(a, table, h, blockIdx.x * KEYS * WAVES + wave * KEYS, end - 1);
    for (int block = blockIdx.x * KEYS * WAVES; block < end; block += stride) {
        const int k0 = block + wave * KEYS;
        k = next;
        next.load(a, table, h, block + stride < end ? k0 + stride : k0, end - 1);
        __builtin_amdgcn_sched_barrier(0);
        // which of the block's pages are this row's to write, and which of these are others' too
        const int first_page = block >> shift;
        const uint64_t mine = a.owner ? __ballot(owner_of(mark) == b) : ~0ull, shared = __ballot(owner_of(mark) == b && mark < 0);
        mark = mark_of(page);
        page = page_of(block + 2 * stride);
        if (mine == 0) continue;
        // the lane's key, once the sums are over the lanes (worked out where it is asked for: it would be kept over all columns)
        constexpr int SHARED = COLS / (4 * FAR);        // lanes that are left with the same
        const auto key_of = [&] {
            int l = lane;
            asm volatile("" : "+v"(l));
            const int j = l % 16 / SHARED;
            return k0 + 16 * (j / 4) + 4 * (l / 16) + j % 4;
        };
        float add = 0.0f;
        bool held = false, fresh = false;
        for (int r = shared ? 0 : b; r < (shared ? a.batch.n_seqs : b + 1); ++r) {
            const Counted s = shared ? counted(a, r) : own;
            uint64_t takes = mine;
            if (shared) {
                int l = lane;
                asm volatile("" : "+v"(l));
                takes = r == b ? mine : __ballot((shared >> l & 1) && has_page(a, r, s, first_page + l, table[first_page + l]));
                if (takes == 0) continue;
            }
            const int cols = s.tokens * G;
            float sum[4 * FAR] = {};
            for (int c0 = 0; c0 < cols; c0 += LISTED) {
                const int n = min(cols - c0, LISTED), rounded = (n + TILED - 1) / TILED * TILED;
                if (cols > LISTED || in_lds != r) {
                    // (columns that fill the last tile up are the last one, with no share)
                    in_lds = cols > LISTED ? -1 : r;
                    int own_tid = tid;
                    asm volatile("" : "+v"(own_tid));       // (what is worked out of it is not kept over the loops)
                    __syncthreads();        // (the last ones have been read)
                    if (own_tid < rounded) {
                        const int64_t id = column_of(a, s, h, c0 + min(own_tid, n - 1));
                        Joined x = *joined_of(a, id);
                        if (own_tid >= n) x.inv = 0.0f;
                        columns.joined[own_tid] = x;
                        columns.id[own_tid] = id;
                    }
                    __syncthreads();
                    constexpr int PIECES = 4 * KS;
                    const int d = own_tid % PIECES * 8;
                    for (int row = own_tid / PIECES; row < rounded; row += THREADS / PIECES)
                        *(bf16x8*)&columns.q[row][d] = EXACT || d < D ? *(const bf16x8*)(a.q + columns.id[row] * D + d) : bf16x8{};
                    __syncthreads();
                }
                if (c0 == 0) k.ready();
                for (int i = 0; i < rounded; i += TILED) {
                    // what the first and the last column see (no column sees less far than one before it)
                    const int first_from = uniform(columns.joined[i].span.from), first_to = uniform(columns.joined[i].span.to);
                    const int last_from = uniform(columns.joined[i + TILED - 1].span.from), last_to = uniform(columns.joined[i + TILED - 1].span.to);
                    if (k0 > last_to || k0 + KEYS <= first_from) continue;      // (no column of the tiles sees any of the keys)
                    bf16x8 q[TILES][KS];
#pragma unroll
                    for (int c = 0; c < TILES; ++c)
#pragma unroll
                        for (int x = 0; x < KS; ++x) q[c][x] = *(const bf16x8*)&columns.q[i + c * COLS + col][dim_of<TYPE>(x, g)];
                    f32x4 sc[TILES][FAR];
                    scores_of(k, q, sc);
                    const bool whole = k0 >= last_from && k0 + KEYS - 1 <= first_to;
#pragma unroll
                    for (int c = 0; c < TILES; ++c) {
                        const Joined& column = columns.joined[i + c * COLS + col];
                        const float most = column.most, inv = column.inv;
                        if (whole) {
#pragma unroll
                            for (int t = 0; t < FAR; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    sum[4 * t + e] = __fmaf_rn(__builtin_amdgcn_exp2f(__fmaf_rn(sc[c][t][e], a.scale_log2, -most)), inv, sum[4 * t + e]);
                        } else {
                            const Span span = column.span;
#pragma unroll
                            for (int t = 0; t < FAR; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int at_key = k0 + 16 * t + 4 * g + e;
                                    const bool sees = at_key >= span.from && at_key <= span.to;
                                    const float p = __builtin_amdgcn_exp2f(__fmaf_rn(sc[c][t][e], a.scale_log2, -most));
                                    sum[4 * t + e] = __fmaf_rn(sees ? p : 0.0f, sees ? inv : 0.0f, sum[4 * t + e]);
                                }
                        }
                    }
                }
            }
            // over the 16 lanes of a key: each hands another half of what it has, until it is left with the sum of one key
#pragma unroll
            for (int o = COLS / 2; o > 0; o >>= 1) {
                if (o >= SHARED) {
#pragma unroll
                    for (int e = 0; e < o / SHARED; ++e) {
                        const bool high = col & o;
                        const float give = high ? sum[e] : sum[e + o / SHARED], keep = high ? sum[e + o / SHARED] : sum[e];
                        sum[e] = keep + __shfl_xor(give, o);
                    }
                } else {
                    sum[0] += __shfl_xor(sum[0], o);
                }
            }
            const int key = key_of();
            if (takes >> ((key >> shift) - first_page) & 1) {
                add += sum[0];
                held |= key < s.len;
                fresh |= key < s.len && key >= s.fresh;
            }
        }
        if (held && col % SHARED == 0) {
            const int key = key_of(), number = table[key >> shift];
            if ((uint32_t)number < (uint32_t)a.pool.n_pages) {
                float* const w = a.pool.weight + (((int64_t)number * H + h) << shift) + (key & inside);
                *w = faded(a, fresh, *w) + add;
            }
        }
    }
}

// How a call is cut up: parts of the keys that statistics are taken of, and whether scores are kept.
struct WeighShape {
    int parts, keep;
    int64_t owners, bytes;      // offset of the pages' owners; all scratch
};
static WeighShape shape_of(const int page_tokens, const int64_t n_pages, const int64_t n_seqs, const int64_t ld_table, const int n_heads, const int64_t cols, const int64_t columns)
{
    const int64_t keys = ld_table * page_tokens, most = (keys + STEP - 1) / STEP, blocks = cols <= COLS ? 1 : (cols + MANY * COLS - 1) / (MANY * COLS);
    // Workgroups in all.  Few columns: 64 sequences of up to 8192 tokens of all lengths 142 us with 2048, 162 with 1024; 4 tokens of one of 60 thousand 42
    // and 39 (more parts, more to join).  Many: 128 columns a head of 2 times 16 thousand 27 us (with the join) with 256, 29 with 512, 37 with 1024, 43 with 2048.
    const int64_t want = (cols <= COLS ? 2048 : 256) / (n_seqs * n_heads * blocks);
    WeighShape f;
    f.parts = (int)(want < 1 ? 1 : want < most ? want : most);
    const double kept = 4.0 * n_seqs * n_heads * cols * kept_keys(keys);
    // (with kept scores against without, us: 64 single tokens of 8 thousand each 163 / 303, one 12 / 22, 4 of 60 thousand 42 / 87)
    f.keep = cols <= COLS && kept <= KEPT;
    f.owners = (columns * f.parts + 1) / 2 * 16 + (f.keep ? (int64_t)kept : (int64_t)sizeof(Joined) * columns);
    f.bytes = f.owners + (n_seqs > 1 ? 4 * n_pages : 0);
    return f;
}

int64_t weigh_work_bytes(const int page_tokens, const int64_t n_pages, const int64_t n_seqs, const int64_t ld_table, const int n_heads, const int64_t cols, const int64_t columns)
{
    return shape_of(page_tokens, n_pages, n_seqs, ld_table, n_heads, cols, columns).bytes;
}

template <int KS, spmm_cache_type_t TYPE, bool EXACT>
static int launch_exact(const WeighArgs& a, const int64_t cols, void* stream)
{
    const int64_t blocks = cols <= COLS ? 1 : (cols + MANY * COLS - 1) / (MANY * COLS), keys = a.batch.ld_table << a.pool.page_shift;
    const dim3 grid((unsigned)(a.parts * a.pool.n_heads), (unsigned)a.batch.n_seqs, (unsigned)(blocks < 65535 ? blocks : 65535)), threads(THREADS);
    if (const int rc = cols <= COLS ? launch(cache_weigh_stats<KS, TYPE, EXACT, 1>, grid, threads, a, stream)
                                    : launch(cache_weigh_stats<KS, TYPE, EXACT, MANY>, grid, threads, a, stream))
        return rc;
    const auto blocks_of = [&](const int each) { return dim3((unsigned)((keys + each - 1) / each), (unsigned)a.pool.n_heads, (unsigned)a.batch.n_seqs); };
    // threads for the entries of the table, where there is more than one row
    const int64_t entries = a.owner ? a.batch.n_seqs * a.batch.ld_table : 0, looked = (entries < 1 << 18 ? entries : 1 << 18) + THREADS - 1;
    if (a.keep) {
        if (a.owner)
            if (const int rc = launch(cache_weigh_shared, dim3((unsigned)(looked / THREADS)), threads, a, stream)) return rc;
        return launch(a.owner ? cache_weigh_kept<true> : cache_weigh_kept<false>, blocks_of(4 * THREADS), threads, a, stream);
    }
    const int64_t columns = (int64_t)a.T * a.group * a.pool.n_heads, joined = columns + THREADS - 1;
    if (const int rc = launch(cache_weigh_join, dim3((unsigned)((joined > looked ? joined : looked) / THREADS)), threads, a, stream)) return rc;
    // A workgroup takes several blocks of keys with the columns it has put together, where there are more blocks than it takes to fill the device (128
    // columns a head of 2 times 16 thousand keys: 30 us with 512 workgroups, 37 with 256, 38 with 2048); where there are fewer it takes blocks of 64 keys, and
    // multiplies four tiles of columns together (1024 tokens on 2048 keys 138 us against 235, 32 on 4000 9.0 against 13.4; with 288 blocks they are
    // level, 18 against 19).
    dim3 all = blocks_of(16 * 4 * WAVES);
    const int64_t others = (int64_t)all.y * all.z, enough = (512 + others - 1) / others;
    if (all.x * others < 256) return launch(cache_weigh_add<KS, TYPE, EXACT, 1>, blocks_of(16 * WAVES), threads, a, stream);
    if (all.x > enough) all.x = (unsigned)enough;
    return launch(cache_weigh_add<KS, TYPE, EXACT, 4>, all, threads, a, stream);
}

template <int KS, spmm_cache_type_t TYPE>
static int launch_steps(const WeighArgs& a, const int64_t cols, void* stream)
{
    return a.pool.head_dim == 32 * KS ? launch_exact<KS, TYPE, true>(a, cols, stream) : launch_exact<KS, TYPE, false>(a, cols, stream);
}

int launch_weigh(const WeighArgs& args, const spmm_cache_type_t type, void* stream)
{
    WeighArgs a = args;
    const int64_t cols = (int64_t)a.max_new * a.group;
    const WeighShape f = shape_of(1 << a.pool.page_shift, a.pool.n_pages, a.batch.n_seqs, a.batch.ld_table, a.pool.n_heads, cols, (int64_t)a.T * a.group * a.pool.n_heads);
    a.parts = f.parts;
    a.keep = f.keep;
    if (a.batch.n_seqs > 1) a.owner = (int32_t*)((char*)a.work + f.owners);
    if (type == SPMM_CACHE_S8) return a.pool.head_dim > 64 ? launch_steps<4, SPMM_CACHE_S8>(a, cols, stream) : launch_steps<2, SPMM_CACHE_S8>(a, cols, stream);
    return a.pool.head_dim > 64 ? launch_steps<4, SPMM_CACHE_BF16>(a, cols, stream) : launch_steps<2, SPMM_CACHE_BF16>(a, cols, stream);
}

}  // namespace spmm_cache
