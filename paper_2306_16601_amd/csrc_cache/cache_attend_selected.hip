// Attention over the pages of a list for each new token and key/value head: bound by reading those pages.
//
// Columns are the query heads of one token that share a key/value head, up to 16 of them, and as in attention over all pages
// (cache_attend.h) scores are computed transposed and weights go from registers to registers.  A workgroup has a list, or a part of
// one: it first writes where the listed pages are, and what positions they hold, to LDS; its four waves then take the keys of the
// list in turn, next step's keys on their way while a wave works on this one's.  All columns see the same keys, so that what is hidden is
// hidden from all: its scores are -inf and its values 0.  Parts of a list are joined by cache_join_selected, in their order.
#include "cache_attend.h"

#include <cfloat>

namespace spmm_cache {

constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;
constexpr int COLS = 16;
constexpr int CUS = 256, PER_CU = 2;
constexpr int LISTED = 1024;        // pages of a part, at most
constexpr int XCDS = 8;

template <spmm_cache_type_t TYPE>
constexpr int KEYS = TYPE == SPMM_CACHE_S8 ? 64 : 32;       // of a wave's step
template <spmm_cache_type_t TYPE>
constexpr int UNIT = WAVES * KEYS<TYPE>;        // of a step of all waves

// a part's statistics (largest score, sum of powers, whether anything is visible), then its results
__host__ __device__ constexpr int part_floats(const int dim) { return COLS * (dim + 3); }

// What the waves of a list tell each other, and a wave of its own list.
template <int DIM, int TEAM>
struct Shared {
    float part[WAVES][DIM / 4][64];
    float stat[WAVES][2][COLS];
    int2 listed[LISTED];            // number in the pool, position of the first token (-1: no page)
    int end, any;
};
template <int DIM>
struct Shared<DIM, 1> {
    int2 listed[LISTED / WAVES];
};

// TEAM: waves of a list: all of the workgroup, which may have a part of the list, or one
template <int DIM, spmm_cache_type_t TYPE, bool EXACT, int TEAM>
__global__ __launch_bounds__(THREADS, PER_CU) void cache_attend_selected(const SelectedArgs args)
{
    constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    constexpr int N = DIM / 16, BYTES = S8 ? 1 : 2, TILES = S8 ? 4 : 2, KS = N / TILES, STEP = KEYS<TYPE>, CHUNK = STEP / 4, ROWS = TILES * 4, LANE = 16 / BYTES;
    constexpr int AHEAD = TEAM * STEP;      // keys from a wave's step to its next
    constexpr bool LATE = false;        // keys and values are not asked for before the others are done with: three waves fit a SIMD, and what they read is in the L2
    __shared__ Shared<DIM, TEAM> shared[TEAM == 1 ? WAVES : 1];

    const AttendArgs& a = args.attend;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % 16, g = lane / 16;
    const int D = EXACT ? DIM : a.pool.head_dim, G = a.group, H = a.pool.n_heads, shift = a.pool.page_shift, inside = (1 << shift) - 1;
    const int tiles = (G + COLS - 1) / COLS;
    int t, h, tile, p = 0;
    if constexpr (TEAM == 1) {
        // lists of the same head side by side on the same XCD, whose cache they share: the device deals workgroups to the XCDs in turn
        const int each = (gridDim.x + XCDS - 1) / XCDS, at = (blockIdx.x % XCDS * each + blockIdx.x / XCDS) * WAVES + wave;
        if (blockIdx.x / XCDS >= each || at >= a.T * H * tiles) return;
        t = at % a.T;
        h = at / a.T % H;
        tile = at / a.T / H;
    } else {
        const int list = blockIdx.x / (uint32_t)(tiles * args.parts), rest = blockIdx.x % (uint32_t)(tiles * args.parts);
        tile = rest / args.parts;
        p = rest % args.parts;
        t = list / H;
        h = list % H;
    }
    const int b = sequence_of(a.batch, t);
    if (b < 0) return;
    Span span = span_of(a.batch, b, t, shift, a.causal, a.window);
    if (span.from > span.to) span = Span{0, -1};
    auto& own = shared[TEAM == 1 ? wave : 0];

    // the part of the list, in pages, and what lies in them
    const int e0 = (int)((int64_t)args.pages * p / args.parts), e1 = (int)((int64_t)args.pages * (p + 1) / args.parts);
    const int32_t* const ids = args.lists + ((int64_t)t * H + h) * args.pages + e0;
    const int32_t* const table = a.batch.table + b * a.batch.ld_table;
    if constexpr (TEAM > 1) {
        if (tid == 0) own.end = own.any = 0;
        __syncthreads();
    }
    int listed_end = 0;
    for (int i = TEAM == 1 ? lane : tid; i < e1 - e0; i += 64 * TEAM) {
        const int id = ids[i];
        int2 x = {0, -1};
        if (id >= 0 && id < a.batch.ld_table) {
            x = int2{page_in_pool(table[id], a.pool.n_pages), id << shift};
            if (x.y <= span.to && x.y + inside >= span.from) listed_end = i + 1;
        }
        own.listed[i] = x;
    }
    if constexpr (TEAM > 1) {
        if (listed_end) __hip_atomic_fetch_max(&own.end, listed_end, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    } else {
        for (int i = 1; i < 64; i <<= 1) listed_end = max(listed_end, __shfl_xor(listed_end, i));
        listed_end = __builtin_amdgcn_readfirstlane(listed_end);
    }

    // columns
    const int column = tile * COLS + col;
    const bool there = column < G;
    const __bf16* const src = a.q + ((int64_t)t * (H * G) + h * G + (there ? column : 0)) * D;
    float unit = a.scale_log2;
    u32x4 q[KS * (S8 ? 2 : 1)];
    if constexpr (S8) {
        // (brought to [1, 2) by a power of two, as binary16 holds them)
        float most = 0.0f;
        u32x4 raw[KS * 2];
#pragma unroll
        for (int i = 0; i < KS * 2; ++i) {
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
        unit = fmaxf(unit * up, FLT_TRUE_MIN);
#pragma unroll
        for (int i = 0; i < KS * 2; ++i) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, raw[i]);
            f16x8 w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = (_Float16)((float)v[j] * down);
            q[i] = __builtin_bit_cast(u32x4, w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const int d = 32 * i + 8 * g;
            q[i] = there && d < D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
        }
    }
    f32x4 o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = f32x4{0, 0, 0, 0};
    float m = NONE, l = 0.0f;
    float v_up = __builtin_bit_cast(float, 2u << 23), v_down = __builtin_bit_cast(float, 252u << 23);      // of the values' scales so far
    if constexpr (TEAM > 1) {
        __syncthreads();
        listed_end = own.end;
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // (a page is counted if some token of it is visible, so that a list with any page has something visible)
    const int k_end = listed_end << shift, last = listed_end - 1;
    const int chunk_k = CHUNK * (col >> 2), chunk_v = CHUNK * g;
    const char* const k_base = (const char*)a.pool.k + ((col & 3) * D + LANE * g) * BYTES;
    const char* const v_base = (const char*)a.pool.v + ((int64_t)col << shift) * BYTES;
    u32x4 k[N], v[N];
    const auto load_k = [&](const int k0) {
        const int at = k0 + chunk_k, page = own.listed[min(at >> shift, last)].x;
        const int64_t slot = (((int64_t)page * H + h) << shift) + (at & inside);
        const char* const from = k_base + slot * D * BYTES;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = (i % KS) * (DIM / KS);
            if (EXACT || d + LANE * g < D) k[i] = *(const u32x4*)(from + ((i / KS) * 4 * D + d) * BYTES);
            else k[i] = u32x4{0, 0, 0, 0};
        }
    };
    int k0 = TEAM == 1 ? 0 : wave * STEP;
    if (k0 < k_end) load_k(k0);
    for (; k0 < k_end; k0 += AHEAD) {
        // the lane's tokens of the step, as scores and as values: CHUNK in a row of one page; -1 where there are none
        const int at = k0 + chunk_v;
        const int2 x = own.listed[min(at >> shift, last)];
        const int64_t head_slot = ((int64_t)x.x * H + h) << shift;
        const int first = at < k_end && x.y >= 0 ? x.y + (at & inside) : 0x40000000;      // position (past all, where there is no page)
        const bool whole = first >= span.from && first + CHUNK - 1 <= span.to;
        const bool partial = __any(!whole);
        float ks[S8 ? ROWS : 1], vs[S8 ? ROWS : 1];
        const auto load_scales = [&](const float* const scales, float* const to) {
            if constexpr (S8)
#pragma unroll
                for (int i = 0; i < ROWS; i += 4) *(f32x4*)(to + i) = *(const f32x4*)(scales + head_slot + (at & inside) + i);
        };
        const auto load_v = [&]() {
            const char* const from = v_base + (head_slot * D + (at & inside)) * BYTES;
#pragma unroll
            for (int d = 0; d < N; ++d) {
                if (EXACT || 16 * d < D) v[d] = *(const u32x4*)(from + (((int64_t)16 * d) << shift) * BYTES);
                else v[d] = u32x4{0, 0, 0, 0};
            }
            load_scales(a.pool.v_scale, vs);
        };
        load_scales(a.pool.k_scale, ks);
        if constexpr (!LATE) load_v();
        // scores
        f32x4 sc[TILES];
#pragma unroll
        for (int tl = 0; tl < TILES; ++tl) {
            sc[tl] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const u32x4 r = k[tl * KS + i];
                if constexpr (S8) {
                    sc[tl] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(r[0], r[1]), __builtin_bit_cast(f16x8, q[2 * i]), sc[tl], 0, 0, 0);
                    sc[tl] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(r[2], r[3]), __builtin_bit_cast(f16x8, q[2 * i + 1]), sc[tl], 0, 0, 0);
                } else {
                    sc[tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, q[i]), sc[tl], 0, 0, 0);
                }
            }
        }
        float y[ROWS];
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
#pragma unroll
        for (int i = 0; i < ROWS; ++i) y[i] = sc[i / 4][i % 4] * (S8 ? ks[S8 ? i : 0] : 1.0f);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (LATE) load_v();
        else if (k0 + AHEAD < k_end) load_k(k0 + AHEAD);
        __builtin_amdgcn_sched_barrier(0);

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
            if constexpr (S8) sum += y[i];
        }
        if constexpr (S8) {
            // the power of two that weights are divided by follows the largest scale of what is visible
            if (partial) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    if (first + i < span.from || first + i > span.to) vs[i] = 0.0f;
            }
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) most = fmaxf(most, fabsf(vs[i]));
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (__any(!(most <= FLT_MAX))) most = FLT_MAX;
            float up;
            const float down = to_unit(most, &up);
            if (__any(up > v_up)) {
                const float less = v_up * down;
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] *= less;
                v_up = up;
                v_down = down;
            }
#pragma unroll
            for (int i = 0; i < ROWS; ++i) y[i] *= vs[i] * v_down;
        }
        u32x4 w[S8 ? 2 : 1];
        if constexpr (S8) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f16x8 f;
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = (_Float16)y[8 * e + j];
                w[e] = __builtin_bit_cast(u32x4, f);
            }
        } else {
            bf16x8 f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (__bf16)y[j];
            w[0] = __builtin_bit_cast(u32x4, f);
            sum = sum_of(f, sum);
        }
        l = l * fade + sum;
        if (__any(fade != 1.0f)) {
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] *= fade;
        }

        // values (what is hidden may hold anything: it counts as 0; codes do, by their scales)
        if constexpr (!S8) {
            if (partial) {
                u32x4 keep;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = first + 2 * j;
                    keep[j] = (i >= span.from && i <= span.to ? 0xffffu : 0u) | (i + 1 >= span.from && i + 1 <= span.to ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int d = 0; d < N; ++d) v[d] &= keep;
            }
        }
#pragma unroll
        for (int d = 0; d < N; ++d) {
            if constexpr (S8) {
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(v[d][0], v[d][1]), __builtin_bit_cast(f16x8, w[0]), o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(v[d][2], v[d][3]), __builtin_bit_cast(f16x8, w[S8 ? 1 : 0]), o[d], 0, 0, 0);
            } else {
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, w[0]), o[d], 0, 0, 0);
            }
        }
        if constexpr (LATE) {
            __builtin_amdgcn_sched_barrier(0);
            if (k0 + AHEAD < k_end) load_k(k0 + AHEAD);
        }
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const float nothing = listed_end ? __builtin_nanf("") : 0.0f;     // (scores of -inf alone, or nothing visible)
    if constexpr (TEAM == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l * (S8 ? v_up : 1.0f);
        if (there)
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = 16 * d + 4 * g + e;
                    if (row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, l == 0.0f ? nothing : o[d][e] * inv);
                }
        return;
    } else {
        // the waves' parts together: written if they are the whole of the list, else to scratch
        const bool alone = args.parts == 1;
        m = m == NONE ? NONE : m * unit;
        if (g == 0) {
            own.stat[wave][0][col] = m;
            own.stat[wave][1][col] = l;
        }
        __syncthreads();
        float top = NONE, all = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = fmaxf(top, own.stat[i][0][col]);
        const float ms = top == NONE ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += own.stat[i][1][col] * __builtin_amdgcn_exp2f(own.stat[i][0][col] - ms);
        const float share = __builtin_amdgcn_exp2f(m - ms) * (S8 ? v_up : 1.0f);
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) own.part[wave][d * 4 + e][lane] = o[d][e] * share;
        __syncthreads();
        float* const slot = a.work + (int64_t)blockIdx.x * part_floats(DIM);
        if (!alone && tid < COLS) {
            slot[tid] = top;
            slot[COLS + tid] = all;
            slot[2 * COLS + tid] = listed_end ? 1.0f : 0.0f;
        }
        const float inv = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = wave + WAVES * j;
            float sum = 0.0f;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) sum += own.part[x][i][lane];
            const int row = 16 * (i / 4) + 4 * g + i % 4;
            if (!alone) slot[3 * COLS + i * 64 + lane] = sum;
            else if (there && row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, all == 0.0f ? nothing : sum * inv);
        }
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
    if (sequence_of(a.batch, t) < 0) return;
    const float* const parts = a.work + (int64_t)blockIdx.x * args.parts * part_floats(DIM);
    float top = NONE, all = 0.0f, seen = 0.0f;
    for (int p = 0; p < args.parts; ++p) top = fmaxf(top, parts[p * part_floats(DIM) + col]);
    const float ms = top == NONE ? 0.0f : top;
    float y[SLICE] = {};
    for (int p = 0; p < args.parts; ++p) {
        const float* const in = parts + p * part_floats(DIM);
        const float share = __builtin_amdgcn_exp2f(in[col] - ms);
        all += in[COLS + col] * share;
        seen += in[2 * COLS + col];
#pragma unroll
        for (int i = 0; i < SLICE; ++i) y[i] += in[3 * COLS + (wave * SLICE + i) * 64 + lane] * share;
    }
    const int column = tile * COLS + col;
    if (column >= G) return;
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
    for (int i = 0; i < SLICE; ++i) {
        const int j = wave * SLICE + i, row = 16 * (j / 4) + 4 * g + j % 4;
        if (row < D) store_out(a, (((int64_t)h * G + column) * D + row) * a.ldo + t, all == 0.0f ? (seen > 0.0f ? __builtin_nanf("") : 0.0f) : y[i] * inv);
    }
}

// Lists from which on a wave has one for itself, if its pages fit.  TEAM_FIGURES
constexpr int64_t SINGLE = 1024;
static bool single(const int64_t lists, const int64_t pages) { return lists >= SINGLE && pages <= LISTED / WAVES; }

// Workgroups that share a list: as many as fill the device, but none without a unit of keys.
static int parts_of(const spmm_cache_type_t type, const int page_tokens, const int64_t lists, const int64_t pages)
{
    if (single(lists, pages)) return 1;
    const int unit = type == SPMM_CACHE_S8 ? UNIT<SPMM_CACHE_S8> : UNIT<SPMM_CACHE_BF16>;
    const int64_t units = (pages * page_tokens + unit - 1) / unit, want = CUS * PER_CU / lists, least = (pages + LISTED - 1) / LISTED;
    const int64_t most = units < pages ? units : pages, n = want < 1 ? 1 : want < most ? want : most;
    return (int)(n < least ? least : n);
}

int64_t selected_work_bytes(const spmm_cache_type_t type, const int page_tokens, const int64_t T, const int n_heads, const int group, const int dim, const int64_t pages)
{
    const int64_t lists = T * n_heads * ((group + COLS - 1) / COLS), parts = parts_of(type, page_tokens, lists, pages);
    return parts == 1 ? 16 : 4 * lists * parts * part_floats(dim > 64 ? 128 : 64);
}

template <int DIM, spmm_cache_type_t TYPE, bool EXACT>
static int launch_exact(const SelectedArgs& a, const int64_t lists, void* stream)
{
    return single(lists, a.pages) ? launch(cache_attend_selected<DIM, TYPE, EXACT, 1>, dim3((unsigned)((lists + WAVES - 1) / WAVES + XCDS - 1) / XCDS * XCDS), dim3(THREADS), a, stream)
                                  : launch(cache_attend_selected<DIM, TYPE, EXACT, WAVES>, dim3((unsigned)(lists * a.parts)), dim3(THREADS), a, stream);
}

template <int DIM, spmm_cache_type_t TYPE>
static int launch_dim(const SelectedArgs& a, const int64_t lists, void* stream)
{
    const int rc = a.attend.pool.head_dim == DIM ? launch_exact<DIM, TYPE, true>(a, lists, stream) : launch_exact<DIM, TYPE, false>(a, lists, stream);
    return rc || a.parts == 1 ? rc : launch(cache_join_selected<DIM>, dim3((unsigned)lists), dim3(THREADS), a, stream);
}

int launch_attend_selected(const SelectedArgs& args, const spmm_cache_type_t type, void* stream)
{
    SelectedArgs a = args;
    const int64_t lists = (int64_t)a.attend.T * a.attend.pool.n_heads * ((a.attend.group + COLS - 1) / COLS);
    a.parts = parts_of(type, 1 << a.attend.pool.page_shift, lists, a.pages);
    if (a.attend.pool.head_dim > 64)
        return type == SPMM_CACHE_S8 ? launch_dim<128, SPMM_CACHE_S8>(a, lists, stream) : launch_dim<128, SPMM_CACHE_BF16>(a, lists, stream);
    return type == SPMM_CACHE_S8 ? launch_dim<64, SPMM_CACHE_S8>(a, lists, stream) : launch_dim<64, SPMM_CACHE_BF16>(a, lists, stream);
}

}  // namespace spmm_cache
