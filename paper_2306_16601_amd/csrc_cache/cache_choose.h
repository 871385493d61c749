// The `need` highest of a row of values, the earlier of equal ones first, in the order of the row.
//
// Values are compared as integers of 32 bits in the same order.  The lowest that is chosen is found bit by bit, from the
// highest: a bit stays set if enough values lie at or above what there is of it so far.  Each step counts, and nothing is moved, so a row
// stays in the registers that it was loaded to; the steps end as soon as a count is exact.  What is chosen keeps its order by counting
// too: ranks are sums over the lanes before.  No atomics, and the same result whatever the order of the waves is.
#pragma once

#include "cache_internal.h"

namespace spmm_cache {

// In the order of the values: -0 like 0, NaN above everything.  Never 0, which stands for no value.
__device__ __forceinline__ uint32_t rank_of(const float v)
{
    if (!(v == v)) return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int before_lane(const uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Where the chosen ones begin: all above `least`, and of those equal to it the first `ties`.
struct Border {
    uint32_t least;
    int ties;
};

// A row in the registers of WAVES waves: value i is register i / (64 WAVES) of lane i % 64 of wave i / 64 % WAVES.  counts: LDS of the
// workgroup, [2][WAVES] numbers (one wave needs none).  All threads call it, with the same need >= 1, of at least as many values.
template <int WAVES, int REGS>
__device__ __forceinline__ Border border_of(const uint32_t (&v)[REGS], const int need, int* const counts)
{
    const int wave = threadIdx.x / 64 % WAVES;
    uint32_t least = 0;
    int step = 0;
    // how many values are at or above x
    const auto count = [&](const uint32_t x) {
        int n = 0;
#pragma unroll
        for (int r = 0; r < REGS; ++r) n += __builtin_popcountll(__ballot(v[r] >= x));
        if constexpr (WAVES > 1) {
            int* const at = counts + (step++ & 1) * WAVES;
            if (threadIdx.x % 64 == 0) at[wave] = n;
            __syncthreads();        // (what is written two steps later has been read by then)
            n = 0;
            for (int w = 0; w < WAVES; ++w) n += at[w];
        }
        return n;
    };
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
        const int n = count(least | bit);
        if (n >= need) least |= bit;
        if (n == need) return Border{least - 1, 0};     // (those at or above it, and no more)
    }
    if (least == 0xffffffffu) return Border{least, need};
    return Border{least, need - count(least + 1)};
}

// put(i, place): for every chosen value i, how many are chosen before it.  totals: LDS, [REGS * WAVES][2] (one wave needs none).
template <int WAVES, int REGS, typename F>
__device__ __forceinline__ void put_chosen(const uint32_t (&v)[REGS], const Border border, int (*const totals)[2], const F& put)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int above = __builtin_popcountll(__ballot(v[r] > border.least)), equal = __builtin_popcountll(__ballot(v[r] == border.least));
            if (lane == 0) {
                totals[r * WAVES + wave][0] = above;
                totals[r * WAVES + wave][1] = equal;
            }
        }
        __syncthreads();
        // sums over the groups before, by one wave
        constexpr int GROUPS = REGS * WAVES, EACH = (GROUPS + 63) / 64;
        if (threadIdx.x / 64 == 0) {
            int sum[2] = {0, 0}, mine[EACH][2];
#pragma unroll
            for (int k = 0; k < EACH; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = lane * EACH + k;
                    mine[k][e] = sum[e];
                    sum[e] += at < GROUPS ? totals[at][e] : 0;
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                int s = sum[e];
                for (int i = 1; i < 64; i <<= 1) {
                    const int o = __shfl_up(s, i);
                    if (lane >= i) s += o;
                }
                sum[e] = s - sum[e];
            }
#pragma unroll
            for (int k = 0; k < EACH; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = lane * EACH + k;
                    if (at < GROUPS) totals[at][e] = sum[e] + mine[k][e];
                }
        }
        __syncthreads();
    }
    int above = 0, equal = 0;       // before this register
#pragma unroll
    for (int r = 0; r < REGS; ++r) {
        if constexpr (WAVES > 1) {
            above = totals[r * WAVES + wave][0];
            equal = totals[r * WAVES + wave][1];
        }
        const uint64_t over = __ballot(v[r] > border.least), same = __ballot(v[r] == border.least);
        const int a = above + before_lane(over), e = equal + before_lane(same);
        if (v[r] > border.least || (v[r] == border.least && e < border.ties)) put((r * WAVES + wave) * 64 + lane, a + min(e, border.ties));
        if constexpr (WAVES == 1) {
            above += __builtin_popcountll(over);
            equal += __builtin_popcountll(same);
        }
    }
}

// The same for rows of any length, whose ranks are computed anew at each pass: rank(i) of value i < n.  counts, totals: as above, for REGS = 1.
template <int WAVES, typename R, typename F>
__device__ void choose_long(const int n, const int need, int* const counts, int (*const totals)[2], const R& rank, const F& put)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    int step = 0;
    const auto count = [&](const uint32_t x) {
        int c = 0;
        for (int i0 = 0; i0 < n; i0 += 64 * WAVES) {
            const int i = i0 + wave * 64 + lane;
            c += __builtin_popcountll(__ballot(i < n && rank(i) >= x));
        }
        int* const at = counts + (step++ & 1) * WAVES;
        if (lane == 0) at[wave] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < WAVES; ++w) c += at[w];
        return c;
    };
    Border border = {0, 0};
    bool exact = false;
    for (uint32_t bit = 0x80000000u; bit && !exact; bit >>= 1) {
        const int c = count(border.least | bit);
        if (c >= need) border.least |= bit;
        exact = c == need;
    }
    if (exact) --border.least;
    else border.ties = border.least == 0xffffffffu ? need : need - count(border.least + 1);
    int above = 0, equal = 0;
    for (int i0 = 0; i0 < n; i0 += 64 * WAVES) {
        const int i = i0 + wave * 64 + lane;
        const uint32_t v = i < n ? rank(i) : 0;
        const bool is_over = i < n && v > border.least, is_same = i < n && v == border.least;
        const uint64_t over = __ballot(is_over), same = __ballot(is_same);
        __syncthreads();        // (the last group's sums have been read)
        if (lane == 0) {
            totals[wave][0] = __builtin_popcountll(over);
            totals[wave][1] = __builtin_popcountll(same);
        }
        __syncthreads();
        int a = above, e = equal;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) {
                a += totals[w][0];
                e += totals[w][1];
            }
            above += totals[w][0];
            equal += totals[w][1];
        }
        a += before_lane(over);
        e += before_lane(same);
        if (is_over || (is_same && e < border.ties)) put(i, a + min(e, border.ties));
    }
}

}  // namespace spmm_cache
