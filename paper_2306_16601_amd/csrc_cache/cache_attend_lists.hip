// Attention over lists of pages of an 8-bit cache where there are enough of them for a wave each, or for four: chunks of prompts, whose tokens have lists
// of their own.
//
// What the waves read is in the L2 then, and the vector unit bounds them: widening codes, and the softmax, which would be computed for 16 columns
// of the matrix instruction whether they are there or not.  So the columns that a token's heads leave free take other keys: with G heads (padded to
// a power of two) 16 / G steps of keys, streams, are multiplied one after the other, each column picks its own stream's scores, and one softmax serves all of
// them.  Streams have maxima and sums of their own, and values are multiplied stream by stream, by weights that are 0 in the other
// streams' columns (a value that is not finite reaches them as NaN, but they are the same heads, which see it too).  At the end
// the streams of a head are joined by shuffles, and the waves of a list in LDS.  Keys and values of the next step are on their way while a wave works on this one's; the workgroups are
// dealt out so that lists of the same head run on the same XCD, whose cache they share.
#include "cache_selected.h"

namespace spmm_cache {

constexpr int WAVES = SELECTED_WAVES, THREADS = SELECTED_THREADS, COLS = SELECTED_COLS;
constexpr int XCDS = 8;

// STREAMS: an even number of them, else one; SHARE: waves of a list, 1 or all of a workgroup
template <int DIM, bool EXACT, bool STREAMS, int SHARE>
__global__ __launch_bounds__(THREADS, 2) void cache_attend_lists(const SelectedArgs args, const int log_group)
{
    constexpr spmm_cache_type_t TYPE = SPMM_CACHE_S8;
    using L = Selected<DIM, TYPE>;
    constexpr int N = L::N, KS = L::KS, STEP = L::STEP, CHUNK = L::CHUNK, ROWS = L::ROWS, LANE = L::LANE;
    __shared__ int2 all_listed[WAVES / SHARE][LISTED / WAVES * SHARE];

    const AttendArgs& a = args.attend;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int tiles = (G + COLS - 1) / COLS;
    // lists head by head; the device deals workgroups to the XCDs in turn
    const int each = gridDim.x / XCDS, list = (int)(blockIdx.x % XCDS * each + blockIdx.x / XCDS) * (WAVES / SHARE) + wave / SHARE;
    if (list >= a.T * H * tiles) return;
    const int t = list % a.T, h = list / a.T % H, tile = list / a.T / H;
    const int b = sequence_near(a.batch, t);
    if (b < 0) return;
    const Span span = seen_span(a, b, t);

    int2* const listed = all_listed[wave / SHARE];      // (waves that share a list all write the same)
    const int32_t* const ids = args.lists + ((int64_t)t * H + h) * args.pages;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    int end = 0;
    for (int i = lane; i < args.pages; i += 64) {
        bool visible;
        listed[i] = listed_page(a, table, ids[i], span, &visible);
        if (visible) end = i + 1;
    }
    for (int i = 1; i < 64; i <<= 1) end = max(end, __shfl_xor(end, i));
    end = __builtin_amdgcn_readfirstlane(end);

    // a column's head and its stream
    const int stream = col >> log_group, column = tile * COLS + (col & ((1 << log_group) - 1));
    const bool there = column < G;
    u32x4 q[L::QUERIES];
    const float unit = load_queries<DIM, TYPE>(a, a.q + ((int64_t)t * (H * G) + h * G + (there ? column : 0)) * D, there, D, g, q);
    f32x4 o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = f32x4{0, 0, 0, 0};
    float m = NONE, l = 0.0f;
    ValueUnit values;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    const int k_end = end << shift, last = max(end - 1, 0), steps = (k_end + STEP - 1) / STEP;
    // steps of keys that share a softmax (behind the last one there are steps of nothing)
    const int width = STREAMS ? min(COLS >> log_group, ((steps + SHARE - 1) / SHARE + 1) & ~1) : 1;
    const int chunk_k = CHUNK * (col >> 2), chunk_v = CHUNK * g;
    // (lanes whose dims are not there load the first ones of the token: what lies 16 g bytes behind them may be behind the last token of the pool)
    const char* const k_base = (const char*)a.pool.k + (col & 3) * D + (EXACT || LANE * g < D ? LANE * g : 0);
    const char* const v_base = (const char*)a.pool.v + ((int64_t)col << shift);
    // a step's keys, or its values: the same loads, other addresses and strides
    const auto load = [&](const int step, const bool are_values, u32x4 (&r)[N]) {
        const int at = step * STEP + (are_values ? chunk_v : chunk_k), page = listed[min(at >> shift, last)].x, off = at & inside;
        const int64_t head = (int64_t)page * H + h;
        const char* const from = are_values ? v_base + ((head * D) << shift) + off : k_base + ((head << shift) + off) * D;
        const int major = are_values ? 16 * KS << shift : 4 * D, minor = are_values ? 16 << shift : 64;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int by = i / KS * major + i % KS * minor;
            if (!EXACT && (are_values ? 16 * i >= D : i % KS * (DIM / KS) + LANE * g >= D)) by = are_values ? 0 : i / KS * major;       // (not used)
            r[i] = *(const u32x4*)(from + by);
        }
    };
    // position of the first of a lane's tokens of a step (past all, where there is no page)
    const auto first_of = [&](const int step, int* const page, int* const off) {
        const int at = step * STEP + chunk_v;
        const int2 x = listed[min(at >> shift, last)];
        *page = x.x;
        *off = at & inside;
        return at < k_end && x.y >= 0 ? x.y + (at & inside) : 0x40000000;
    };

    u32x4 even[N], odd[N];
    const int begin = SHARE > 1 ? wave * width : 0;
    if (begin < steps) load(begin, false, even);
    for (int base = begin; base < steps; base += SHARE * width) {
        // the lane's own tokens of these steps
        int page, off;
        int first = first_of(base + stream, &page, &off);
        if (stream >= width) first = 0x40000000;
        const bool partial = __any(!(first >= span.from && first + CHUNK - 1 <= span.to));
        const int64_t slot = (((int64_t)page * H + h) << shift) + off;
        float y[ROWS], ks[ROWS], vs[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; i += 4) *(f32x4*)(ks + i) = *(const f32x4*)(a.pool.k_scale + slot + i);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) y[i] = 0.0f;
        u32x4 w[L::WEIGHTS];

        const auto softmax = [&]() {
#pragma unroll
            for (int i = 0; i < ROWS; i += 4) *(f32x4*)(vs + i) = *(const f32x4*)(a.pool.v_scale + slot + i);
            key_scales(ks);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) y[i] *= ks[i];
            if (partial) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const bool seen = first + i >= span.from && first + i <= span.to;
                    y[i] = seen ? y[i] : NONE;
                    vs[i] = seen ? vs[i] : 0.0f;
                }
            }
            float top = y[0];
#pragma unroll
            for (int i = 1; i < ROWS; ++i) top = fmaxf(top, y[i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float mn = fmaxf(m, top), ms = mn == NONE ? 0.0f : mn * unit, fade = __builtin_amdgcn_exp2f(m * unit - ms), less = fade * values.follow(vs);
            m = mn;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                y[i] = __builtin_amdgcn_exp2f(__fmaf_rn(y[i], unit, -ms));
                sum += y[i];
                y[i] *= vs[i] * values.down;
            }
            pack_terms<_Float16, L::TERMS, L::HALVES>(y, values.infinite, w);
            l = l * fade + sum;
            if (__any(less != 1.0f)) {
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] *= less;
            }
        };
        const auto keys = [&](const int x, u32x4 (&k)[N]) {
            if constexpr (!EXACT) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i % KS * (DIM / KS) + LANE * g >= D) k[i] = u32x4{0, 0, 0, 0};
            }
            f32x4 sc[L::TILES];
            selected_scores<DIM, TYPE>(k, q, sc);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) y[i] = !STREAMS || stream == x ? sc[i / 4][i % 4] : y[i];
        };
        const auto products = [&](const int x, u32x4 (&v)[N]) {
            u32x4 mine[L::WEIGHTS];
#pragma unroll
            for (int e = 0; e < L::WEIGHTS; ++e) mine[e] = !STREAMS || stream == x ? w[e] : u32x4{0, 0, 0, 0};
            selected_values<DIM, TYPE>(v, mine, o);
        };
        const int after = base + SHARE * width < steps ? base + SHARE * width : 0;      // (behind the last one something that is there, and not used)
        if constexpr (STREAMS) {
#pragma unroll 1
            for (int x = 0; x < width; x += 2) {
                load(base + x + 1, false, odd);
                __builtin_amdgcn_sched_barrier(0);
                keys(x, even);
                load(x + 2 < width ? base + x + 2 : base, x + 2 == width, even);
                __builtin_amdgcn_sched_barrier(0);
                keys(x + 1, odd);
            }
            softmax();
#pragma unroll 1
            for (int x = 0; x < width; x += 2) {
                load(base + x + 1, true, odd);
                __builtin_amdgcn_sched_barrier(0);
                products(x, even);
                load(x + 2 < width ? base + x + 2 : after, x + 2 < width, even);
                __builtin_amdgcn_sched_barrier(0);
                products(x + 1, odd);
            }
        } else {
            load(base, true, odd);
            __builtin_amdgcn_sched_barrier(0);
            keys(0, even);
            load(after, false, even);
            __builtin_amdgcn_sched_barrier(0);
            softmax();
            products(0, odd);
        }
    }

    // over the lanes of a column, then the streams of a head
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    m = m == NONE ? NONE : m * unit;
    float top = m;
    for (int i = 1 << log_group; i < COLS; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float share = __builtin_amdgcn_exp2f(m - (top == NONE ? 0.0f : top));
    l *= share;
    for (int i = 1 << log_group; i < COLS; i <<= 1) l += __shfl_xor(l, i);
    const float nothing = of_nothing(0, end - 1), mine = share * values.up;
    if constexpr (SHARE == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y = o[d][e] * mine;
                for (int i = 1 << log_group; i < COLS; i <<= 1) y += __shfl_xor(y, i);
                const int row = 16 * d + 4 * g + e;
                if (there && stream == 0 && row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, l == 0.0f ? nothing : y * inv);
            }
    } else {
        // then the waves
        __shared__ float part[WAVES][N * 4][64], stat[WAVES][2][COLS];
        if (g == 0) {
            stat[wave][0][col] = top;
            stat[wave][1][col] = l;
        }
        __syncthreads();
        float most = NONE, all = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) most = fmaxf(most, stat[i][0][col]);
        const float ms = most == NONE ? 0.0f : most;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += stat[i][1][col] * __builtin_amdgcn_exp2f(stat[i][0][col] - ms);
        const float scaled = mine * __builtin_amdgcn_exp2f(top - ms);
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][d * 4 + e][lane] = o[d][e] * scaled;
        __syncthreads();
        const float inv = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = wave + WAVES * j, row = 16 * (i / 4) + 4 * g + i % 4;
            float y = 0.0f;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) y += part[x][i][lane];
            for (int k = 1 << log_group; k < COLS; k <<= 1) y += __shfl_xor(y, k);
            if (there && stream == 0 && row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, all == 0.0f ? nothing : y * inv);
        }
    }
}

template <int DIM, int SHARE>
static int launch_dim(const SelectedArgs& a, const int64_t lists, void* stream)
{
    int log_group = 0;
    while (1 << log_group < a.attend.group && 1 << log_group < COLS) ++log_group;
    const int64_t groups = (lists + WAVES / SHARE - 1) / (WAVES / SHARE);
    void* args[] = {const_cast<SelectedArgs*>(&a), &log_group};
    const bool streams = 2 << log_group <= COLS;
    const void* const kernel = a.attend.pool.head_dim == DIM
                                   ? streams ? (const void*)cache_attend_lists<DIM, true, true, SHARE> : (const void*)cache_attend_lists<DIM, true, false, SHARE>
                                   : streams ? (const void*)cache_attend_lists<DIM, false, true, SHARE> : (const void*)cache_attend_lists<DIM, false, false, SHARE>;
    return (int)hipLaunchKernel(kernel, dim3((unsigned)((groups + XCDS - 1) / XCDS * XCDS)), dim3(THREADS), args, 0, (hipStream_t)stream);
}

int launch_attend_lists(const SelectedArgs& a, const int64_t lists, const bool shared, void* stream)
{
    if (shared) return a.attend.pool.head_dim > 64 ? launch_dim<128, WAVES>(a, lists, stream) : launch_dim<64, WAVES>(a, lists, stream);
    return a.attend.pool.head_dim > 64 ? launch_dim<128, 1>(a, lists, stream) : launch_dim<64, 1>(a, lists, stream);
}

}  // namespace spmm_cache
