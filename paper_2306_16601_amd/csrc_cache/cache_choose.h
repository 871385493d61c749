// The `need` highest of a row of values, the earlier of equal ones first, in the order of the row.
//
// Values are compared as integers of 32 bits in the same order.  Those between the lowest and the highest are counted in bins of equal
// width (LDS), the bin that the border lies in is the next range, and once it holds 64 values or fewer, these are ranked against each
// other: a row of a thousand scores takes one pass of bins, and seldom another.  Counts do not depend on the order of additions, and
// nothing is moved, so a row stays in the registers that it was loaded to.  What is chosen keeps its order by counting too: ranks
// are sums over the lanes before.  (A border that is halved until its count is right takes 10 to 22 passes over the row, 42 us for 16000
// rows of 970 scores; with bins it is 32, and 26 (21 with the row loaded at once) since only those values are counted that can be chosen: where no more are chosen than the row has threads,
// the lowest of the threads' highest values is a bound.)
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

// LDS of the waves that share a row
template <int WAVES>
struct Bins {
    static constexpr int LOG = WAVES > 1 ? 10 : 8, N = 1 << LOG;
    alignas(16) uint32_t count[N];
    uint32_t last[64];          // values of the last range
    int n_last;
    uint32_t ends[WAVES][2];
};

template <int WAVES>
__device__ __forceinline__ void together()
{
    if constexpr (WAVES > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

__device__ __forceinline__ uint32_t of_lane(const uint32_t v, const int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// each(f): f of every value that this thread has of the row (0: none).  1 <= need, less than there are values.  All threads of the row call it.
template <int WAVES, typename E>
__device__ __forceinline__ Border border_of(const E& each, uint32_t need, Bins<WAVES>& bins)
{
    using B = Bins<WAVES>;
    const int tid = threadIdx.x % (64 * WAVES), lane = tid % 64, wave = tid / 64;
    // The highest, and a value that at least `need` reach: the lowest of the threads' highest ones, where there are no more to choose than
    // threads and each has a value, and the lowest of all otherwise.
    uint32_t lo = 0xffffffffu, hi = 0;
    const auto ends = [&] {
        for (int i = 1; i < 64; i <<= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, i));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, i));
        }
        if constexpr (WAVES > 1) {
            __syncthreads();
            if (lane == 0) {
                bins.ends[wave][0] = lo;
                bins.ends[wave][1] = hi;
            }
            __syncthreads();
            for (int w = 0; w < WAVES; ++w) {
                lo = min(lo, bins.ends[w][0]);
                hi = max(hi, bins.ends[w][1]);
            }
        }
        lo = of_lane(lo, 0);
        hi = of_lane(hi, 0);
    };
    each([&](const uint32_t v) { hi = max(hi, v); });
    lo = need <= 64 * WAVES ? hi : 0;
    ends();
    if (lo == 0) {
        lo = 0xffffffffu;
        each([&](const uint32_t v) { lo = min(lo, v - 1); });       // (of no value it is the highest number)
        ends();
        ++lo;
    }

    while (lo < hi) {
        const int shift = max(32 - B::LOG - __builtin_clz(hi - lo), 0);
        for (int i = tid; i < B::N; i += 64 * WAVES) bins.count[i] = 0;
        if (tid == 0) bins.n_last = 0;
        together<WAVES>();
        each([&](const uint32_t v) {
            if (v - lo <= hi - lo) __hip_atomic_fetch_add(&bins.count[(v - lo) >> shift], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        });
        together<WAVES>();
        // the bin in which the count from above reaches need: a lane has the bins EACH * lane .., each wave does the same
        constexpr int EACH = B::N / 64;
        uint32_t c[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; i += 4) {
            const u32x4 x = *(const u32x4*)&bins.count[lane * EACH + i];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += c[i + j] = x[j];
        }
        uint32_t above = sum;
        for (int i = 1; i < 64; i <<= 1) {
            const uint32_t o = (uint32_t)__shfl_down((int)above, i);
            if (lane + i < 64) above += o;
        }
        above -= sum;
        const int at = __builtin_ctzll(__ballot(above < need && need <= above + sum));
        uint32_t bin = 0, over = 0, held = 0;
#pragma unroll
        for (int i = EACH - 1; i >= 0; --i) {
            if (above < need) {
                bin = lane * EACH + i;
                over = above;
                held = c[i];
            }
            above += c[i];
        }
        bin = of_lane(bin, at);
        held = of_lane(held, at);
        need -= of_lane(over, at);
        lo += bin << shift;
        hi = lo + min(hi - lo, (1u << shift) - 1);
        if (held == need) return Border{lo - 1, 0};
        if (held <= 64 && lo < hi) {
            each([&](const uint32_t v) {
                if (v - lo <= hi - lo) bins.last[__hip_atomic_fetch_add(&bins.n_last, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)] = v;
            });
            together<WAVES>();
            const uint32_t x = lane < (int)held ? bins.last[lane] : 0;
            uint32_t higher = 0, equal = 0;
            for (uint32_t i = 0; i < held; ++i) {
                const uint32_t y = of_lane(x, i);
                higher += y > x;
                equal += y == x;
            }
            const int from = __builtin_ctzll(__ballot(x && higher < need && need <= higher + equal));
            const uint32_t least = of_lane(x, from), ties = need - of_lane(higher, from);
            return ties == of_lane(equal, from) ? Border{least - 1, 0} : Border{least, (int)ties};
        }
        together<WAVES>();      // (the counts have been read)
    }
    return Border{lo, (int)need};
}

// put(i, place): for every chosen value i, how many are chosen before it.  Value i is register i / (64 WAVES) of lane i % 64 of wave i / 64 % WAVES.
// totals: LDS, [REGS * WAVES][2] (one wave needs none).
template <int WAVES, int REGS, typename F>
__device__ __forceinline__ void put_chosen(const uint32_t (&v)[REGS], const Border border, int (*const totals)[2], const F& put)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int above = __builtin_popcountll(__ballot(v[r] > border.least)), equal = border.ties ? __builtin_popcountll(__ballot(v[r] == border.least)) : 0;
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
    if (border.ties == 0) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const uint64_t over = __ballot(v[r] > border.least);
            if constexpr (WAVES > 1) above = totals[r * WAVES + wave][0];
            if (v[r] > border.least) put((r * WAVES + wave) * 64 + lane, above + before_lane(over));
            above += __builtin_popcountll(over);
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < REGS; ++r) {
        if constexpr (WAVES > 1) {
            above = totals[r * WAVES + wave][0];
            equal = totals[r * WAVES + wave][1];
        }
        const uint64_t over = __ballot(v[r] > border.least), same = __ballot(v[r] == border.least);
        const int a = above + before_lane(over), e = equal + before_lane(same);
        if (v[r] > border.least || (v[r] == border.least && e < border.ties)) put((r * WAVES + wave) * 64 + lane, a + min(e, border.ties));
        above += __builtin_popcountll(over);
        equal += __builtin_popcountll(same);
    }
}

template <int WAVES, int REGS, typename F>
__device__ __forceinline__ void choose(const uint32_t (&v)[REGS], const int need, Bins<WAVES>& bins, int (*const totals)[2], const F& put)
{
    const Border border = border_of<WAVES>([&](const auto& f) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) f(v[r]);
    }, need, bins);
    put_chosen<WAVES>(v, border, totals, put);
}

// The same for rows of any length, whose ranks are computed anew at each pass: rank(i) of value i < n.  totals: as above, for REGS = 1.
template <int WAVES, typename R, typename F>
__device__ void choose_long(const int n, const int need, Bins<WAVES>& bins, int (*const totals)[2], const R& rank, const F& put)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    const Border border = border_of<WAVES>([&](const auto& f) {
        for (int i = wave * 64 + lane; i < n; i += 64 * WAVES) f(rank(i));
    }, need, bins);
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
