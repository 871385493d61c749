// Attention over the pages of a list for each new token and key/value head: bound by reading those pages.
//
// Columns are the query heads of one token that share a key/value head, up to 16 of them, and as in attention over all pages
// (cache_attend.h) scores are computed transposed and weights go from registers to registers, as sums of terms that hold all of them (pack_terms).  A workgroup has a list, or a part of
// one: it first writes where the listed pages are, and what positions they hold, to LDS; its four waves then take the keys of the
// list in turn, next step's keys on their way while a wave works on this one's.  All columns see the same keys, so that what is hidden is
// hidden from all: its scores are -inf and its values 0.  Parts of a list are joined by cache_join_selected, in their order.
#include "cache_selected.h"

namespace spmm_cache {

constexpr int WAVES = SELECTED_WAVES, THREADS = SELECTED_THREADS, COLS = SELECTED_COLS;
constexpr int CUS = 256, PER_CU = 2;

// a part's statistics (largest score, sum of powers, whether anything is visible), then its results
__host__ __device__ constexpr int part_floats(const int dim) { return COLS * (dim + 3); }

template <int DIM, spmm_cache_type_t TYPE, bool EXACT>
__global__ __launch_bounds__(THREADS, PER_CU) void cache_attend_selected(const SelectedArgs args)
{
    using L = Selected<DIM, TYPE>;
    constexpr bool S8 = L::S8;
    constexpr int N = L::N, BYTES = L::BYTES, KS = L::KS, STEP = L::STEP, CHUNK = L::CHUNK, ROWS = L::ROWS, LANE = L::LANE, UNIT = WAVES * STEP;
    __shared__ float part[WAVES][N * 4][64];
    __shared__ float stat[WAVES][2][COLS];
    __shared__ int2 listed[LISTED];
    __shared__ int listed_end;

    const AttendArgs& a = args.attend;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % 16, g = lane / 16;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int tiles = (G + COLS - 1) / COLS;
    const int list = blockIdx.x / (uint32_t)(tiles * args.parts), rest = blockIdx.x % (uint32_t)(tiles * args.parts);
    const int tile = rest / args.parts, p = rest % args.parts, t = list / H, h = list % H;
    const int b = sequence_near(a.batch, t);
    if (b < 0) return;
    const Span span = seen_span(a, b, t);

    // the part of the list, in pages, and what lies in them
    const int e0 = (int)((int64_t)args.pages * p / args.parts), e1 = (int)((int64_t)args.pages * (p + 1) / args.parts);
    const int32_t* const ids = args.lists + (int64_t)list * args.pages + e0;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    if (tid == 0) listed_end = 0;
    __syncthreads();
    int end = 0;
    for (int i = tid; i < e1 - e0; i += THREADS) {
        bool visible;
        listed[i] = listed_page(a, table, ids[i], span, &visible);
        if (visible) end = i + 1;
    }
    if (end) __hip_atomic_fetch_max(&listed_end, end, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);

    // columns
    const int column = tile * COLS + col;
    const bool there = column < G;
    u32x4 q[L::QUERIES];
    const float unit = load_queries<DIM, TYPE>(a, a.q + ((int64_t)t * (H * G) + h * G + (there ? column : 0)) * D, there, D, g, q);
    f32x4 o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = f32x4{0, 0, 0, 0};
    float m = NONE, l = 0.0f;
    ValueUnit values;
    __syncthreads();

    // (a page is counted if some token of it is visible, so that a list with any page has something visible)
    end = listed_end;
    const int k_end = end << shift, last = end - 1;
    const int chunk_k = CHUNK * (col >> 2), chunk_v = CHUNK * g;
    const char* const k_base = (const char*)a.pool.k + ((col & 3) * D + LANE * g) * BYTES;
    const char* const v_base = (const char*)a.pool.v + ((int64_t)col << shift) * BYTES;
    u32x4 k[N], v[N];
    const auto load_k = [&](const int k0) {
        const int at = k0 + chunk_k, page = listed[min(at >> shift, last)].x;
        const int64_t slot = (((int64_t)page * H + h) << shift) + (at & inside);
        const char* const from = k_base + slot * D * BYTES;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = (i % KS) * (DIM / KS);
            if (EXACT || d + LANE * g < D) k[i] = *(const u32x4*)(from + ((i / KS) * 4 * D + d) * BYTES);
            else k[i] = u32x4{0, 0, 0, 0};
        }
    };
    int k0 = wave * STEP;
    if (k0 < k_end) load_k(k0);
    for (; k0 < k_end; k0 += UNIT) {
        // the lane's tokens of the step, as scores and as values: CHUNK in a row of one page
        const int at = k0 + chunk_v;
        const int2 x = listed[min(at >> shift, last)];
        const int64_t head_slot = ((int64_t)x.x * H + h) << shift;
        const int first = at < k_end && x.y >= 0 ? x.y + (at & inside) : 0x40000000;      // position (past all, where there is no page)
        const bool partial = __any(!(first >= span.from && first + CHUNK - 1 <= span.to));
        {
            const char* const from = v_base + (head_slot * D + (at & inside)) * BYTES;
#pragma unroll
            for (int d = 0; d < N; ++d) {
                if (EXACT || 16 * d < D) v[d] = *(const u32x4*)(from + (((int64_t)16 * d) << shift) * BYTES);
                else v[d] = u32x4{0, 0, 0, 0};
            }
        }
        float ks[S8 ? ROWS : 1], vs[S8 ? ROWS : 1];
        if constexpr (S8) {
            const int64_t slot = head_slot + (at & inside);
#pragma unroll
            for (int i = 0; i < ROWS; i += 4) {
                *(f32x4*)(ks + i) = *(const f32x4*)(a.pool.k_scale + slot + i);
                *(f32x4*)(vs + i) = *(const f32x4*)(a.pool.v_scale + slot + i);
            }
        }
        f32x4 sc[L::TILES];
        selected_scores<DIM, TYPE>(k, q, sc);
        __builtin_amdgcn_sched_barrier(0);
        if (k0 + UNIT < k_end) load_k(k0 + UNIT);
        __builtin_amdgcn_sched_barrier(0);

        if constexpr (S8) {
            if (partial) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    if (first + i < span.from || first + i > span.to) vs[i] = 0.0f;
            }
            const float less = values.follow(vs);
            if (__any(less != 1.0f)) {
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] *= less;
            }
            key_scales(ks);
        }
        float y[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) y[i] = sc[i / 4][i % 4] * (S8 ? ks[S8 ? i : 0] : 1.0f);
        if (partial) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i) y[i] = first + i >= span.from && first + i <= span.to ? y[i] : NONE;
        }
        float top = y[0];
#pragma unroll
        for (int i = 1; i < ROWS; ++i) top = fmaxf(top, y[i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top), ms = mn == NONE ? 0.0f : mn * unit;
        const float fade = __builtin_amdgcn_exp2f(m * unit - ms);
        m = mn;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            y[i] = __builtin_amdgcn_exp2f(__fmaf_rn(y[i], unit, -ms));
            sum += y[i];
            if constexpr (S8) y[i] *= vs[i] * values.down;
        }
        u32x4 w[L::WEIGHTS];
        if constexpr (S8) pack_terms<_Float16, L::TERMS, L::HALVES>(y, values.infinite, w);
        else pack_terms<__bf16, L::TERMS, L::HALVES>(y, false, w);
        l = l * fade + sum;
        if (__any(fade != 1.0f)) {
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] *= fade;
        }
        if (!S8 && partial) hide_values(v, first, span);
        selected_values<DIM, TYPE>(v, w, o);
    }

    // the waves' parts together: written if they are the whole of the list, else to scratch
    const bool alone = args.parts == 1;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    m = m == NONE ? NONE : m * unit;
    if (g == 0) {
        stat[wave][0][col] = m;
        stat[wave][1][col] = l;
    }
    __syncthreads();
    float top = NONE, all = 0.0f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, stat[i][0][col]);
    const float ms = top == NONE ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) all += stat[i][1][col] * __builtin_amdgcn_exp2f(stat[i][0][col] - ms);
    const float share = __builtin_amdgcn_exp2f(m - ms) * (S8 ? values.up : 1.0f);
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][d * 4 + e][lane] = o[d][e] * share;
    __syncthreads();
    float* const slot = a.work + (int64_t)blockIdx.x * part_floats(DIM);
    if (!alone && tid < COLS) {
        slot[tid] = top;
        slot[COLS + tid] = all;
        slot[2 * COLS + tid] = end ? 1.0f : 0.0f;
    }
    const float inv = all == 0.0f ? 0.0f : 1.0f / all, nothing = of_nothing(0, end - 1);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = wave + WAVES * j;
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) sum += part[x][i][lane];
        const int row = 16 * (i / 4) + 4 * g + i % 4;
        if (!alone) slot[3 * COLS + i * 64 + lane] = sum;
        else if (there && row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, all == 0.0f ? nothing : sum * inv);
    }
}

// Joins the parts of a list.
template <int DIM>
__global__ __launch_bounds__(THREADS) void cache_join_selected(const SelectedArgs args)
{
    constexpr int N = DIM / 16, ROWS = N * 4, SLICE = ROWS / WAVES;
    const AttendArgs& a = args.attend;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, g = lane / 16;
    const int H = a.pool.n_heads, G = a.group, D = a.pool.head_dim, tiles = (G + COLS - 1) / COLS;
    const int64_t list = blockIdx.x / (uint32_t)tiles;
    const int tile = blockIdx.x % (uint32_t)tiles, t = (int)(list / H), h = (int)(list % H);
    if (sequence_near(a.batch, t) < 0) return;
    const float* const parts = a.work + (int64_t)blockIdx.x * args.parts * part_floats(DIM);
    float top = NONE, all = 0.0f, seen = 0.0f;
    constexpr int AHEAD = 4;        // parts that are loaded together (behind the last one it again, and nothing of it counts)
    for (int p0 = 0; p0 < args.parts; p0 += 4 * AHEAD) {
        float x[4 * AHEAD];
#pragma unroll
        for (int k = 0; k < 4 * AHEAD; ++k) x[k] = parts[min(p0 + k, args.parts - 1) * part_floats(DIM) + col];
#pragma unroll
        for (int k = 0; k < 4 * AHEAD; ++k) top = fmaxf(top, x[k]);
    }
    const float ms = top == NONE ? 0.0f : top;
    float y[SLICE] = {};
    for (int p0 = 0; p0 < args.parts; p0 += AHEAD) {
        float x[AHEAD][3 + SLICE];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float* const in = parts + min(p0 + k, args.parts - 1) * part_floats(DIM);
#pragma unroll
            for (int i = 0; i < 3; ++i) x[k][i] = in[i * COLS + col];
#pragma unroll
            for (int i = 0; i < SLICE; ++i) x[k][3 + i] = in[3 * COLS + (wave * SLICE + i) * 64 + lane];
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (p0 + k >= args.parts) break;
            const float share = __builtin_amdgcn_exp2f(x[k][0] - ms);
            all += x[k][1] * share;
            seen += x[k][2];
#pragma unroll
            for (int i = 0; i < SLICE; ++i) y[i] += x[k][3 + i] * share;
        }
    }
    const int column = tile * COLS + col;
    if (column >= G) return;
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
    for (int i = 0; i < SLICE; ++i) {
        const int j = wave * SLICE + i, row = 16 * (j / 4) + 4 * g + j % 4;
        if (row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, all == 0.0f ? of_nothing(0, (int)seen - 1) : y[i] * inv);
    }
}

// Workgroups that share a list: as many as fill the device, two on a CU, but none without a unit of keys.  Of 170 calls of 1 to 31 tokens on 8 to 512 pages, two on a
// CU against one: 64 lists of 512 pages 60 us / 77, 128 of 128 34 / 42, 64 of 128 24 / 26 (8 bits, 64 dims); but where few lists have many parts, joining them costs more than
// they gain: 8 lists of 128 pages in bfloat16 39 / 25, 2 of 512 114 / 63; the mean of all is 6 % in favour of one.  Four take 35 where two take 25 (32 lists of 64).
static int parts_of(const spmm_cache_type_t type, const int dim, const int page_tokens, const int64_t lists, const int64_t pages)
{
    if (waves_of(type, dim, lists, pages)) return 1;
    const int unit = WAVES * (type == SPMM_CACHE_S8 ? SELECTED_KEYS<SPMM_CACHE_S8> : SELECTED_KEYS<SPMM_CACHE_BF16>);
    const int64_t units = (pages * page_tokens + unit - 1) / unit, want = CUS * PER_CU / lists, least = (pages + LISTED - 1) / LISTED;
    const int64_t most = units < pages ? units : pages, n = want < 1 ? 1 : want < most ? want : most;
    return (int)(n < least ? least : n);
}

int64_t selected_work_bytes(const spmm_cache_type_t type, const int page_tokens, const int64_t T, const int n_heads, const int group, const int dim, const int64_t pages)
{
    const int64_t lists = T * n_heads * ((group + COLS - 1) / COLS), parts = parts_of(type, dim, page_tokens, lists, pages);
    if (lists * parts >= (int64_t)1 << 24) return -1;       // (a grid has less than 2^32 threads)
    return parts == 1 ? 16 : 4 * lists * parts * part_floats(dim > 64 ? 128 : 64);
}

template <int DIM, spmm_cache_type_t TYPE>
static int launch_dim(const SelectedArgs& a, const int64_t lists, void* stream)
{
    const dim3 grid((unsigned)(lists * a.parts));
    const int rc = a.attend.pool.head_dim == DIM ? launch(cache_attend_selected<DIM, TYPE, true>, grid, dim3(THREADS), a, stream)
                                                 : launch(cache_attend_selected<DIM, TYPE, false>, grid, dim3(THREADS), a, stream);
    return rc || a.parts == 1 ? rc : launch(cache_join_selected<DIM>, dim3((unsigned)lists), dim3(THREADS), a, stream);
}

int launch_attend_selected(const SelectedArgs& args, const spmm_cache_type_t type, void* stream)
{
    SelectedArgs a = args;
    const int64_t lists = (int64_t)a.attend.T * a.attend.pool.n_heads * ((a.attend.group + COLS - 1) / COLS);
    const int dim = a.attend.pool.head_dim;
    if (const int waves = waves_of(type, dim, lists, a.pages)) return launch_attend_lists(a, lists, waves > 1, stream);
    a.parts = parts_of(type, dim, 1 << a.attend.pool.page_shift, lists, a.pages);
    if (dim > 64)
        return type == SPMM_CACHE_S8 ? launch_dim<128, SPMM_CACHE_S8>(a, lists, stream) : launch_dim<128, SPMM_CACHE_BF16>(a, lists, stream);
    return type == SPMM_CACHE_S8 ? launch_dim<64, SPMM_CACHE_S8>(a, lists, stream) : launch_dim<64, SPMM_CACHE_BF16>(a, lists, stream);
}

}  // namespace spmm_cache
