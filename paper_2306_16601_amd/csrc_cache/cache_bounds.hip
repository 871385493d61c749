// Bounds of a page's keys: of each head and dim the largest and the smallest value.
//
// A wave takes a head of a page: lanes side by side hold 16 bytes each of a token's key, as many tokens at a time as a wave's lanes
// are wide, and the groups of lanes are joined at the end.  bfloat16 values are compared as integers of 16 bits, two to an
// instruction: with the other bits of negative ones turned over, their order is that of the values, and what is not finite lies at
// both ends, so that it is found in the results and costs nothing on the way.  Codes of 8 bits are widened and
// multiplied by their scales in binary32, and the results are rounded to bfloat16, which keeps the order.
//
// Reading the keys bounds it: 4 x 16385 tokens of 8 heads of 128 dims in 8 bits (71 MB with scales and results) take 21.2 us, 3.3 TB/s, in bfloat16 (138 MB) 30.0 us, 4.6 TB/s, eight
// loads of a lane under way together; one page and head for each of 64 new tokens takes 5.0 us, of which a launch is 2.4.
#include "cache_internal.h"

namespace spmm_cache {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
constexpr int AHEAD = 8;            // tokens of a lane that are loaded together

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16b __attribute__((ext_vector_type(16)));

// order of bfloat16 values as integers, and back
__device__ __forceinline__ s16x8 ordered(const s16x8 v) { return v ^ ((v >> 15) & (short)0x7fff); }
constexpr short TOP = 0x7f80;       // infinity; -infinity is its other end (-TOP - 1), and NaN lie beyond both

template <spmm_cache_type_t TYPE>
__global__ __launch_bounds__(THREADS) void cache_bounds(const BoundsArgs a)
{
    constexpr bool S8 = TYPE == SPMM_CACHE_S8;
    constexpr int N = S8 ? 16 : 8;      // dims of a lane
    const int b = blockIdx.x, lane = threadIdx.x % 64, shift = a.pool.page_shift, H = a.pool.n_heads, D = a.pool.head_dim;
    const int len = tokens_of(a.batch, b, shift);
    const int64_t new_tokens = (int64_t)a.batch.q_start[b + 1] - a.batch.q_start[b], past = (int64_t)a.batch.kv_len[b] - new_tokens;
    if (new_tokens <= 0 || past >= len) return;
    const int first = past > 0 ? (int)(past >> shift) : 0, pages = ((len - 1) >> shift) + 1 - first;
    const int wide = D / N, deep = 64 / wide, c = lane % wide, r = lane / wide;
    const int64_t all = (int64_t)pages * H;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    for (int64_t w = (int64_t)blockIdx.y * WAVES + wave; w < all; w += (int64_t)gridDim.y * WAVES) {
        const int i = first + (int)(w / H), h = (int)(w % H);
        const int page = a.batch.table[b * a.batch.ld_table + i];
        if ((uint32_t)page >= (uint32_t)a.pool.n_pages) continue;
        const int held = min(len - (i << shift), 1 << shift);
        const int64_t head = (int64_t)page * H + h;
        __bf16* const out = a.pool.bounds + head * 2 * D + c * N;
        if constexpr (!S8) {
            const s16x8* const src = (const s16x8*)((const __bf16*)a.pool.k + (head << shift) * D) + c;
            s16x8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hi[j] = -0x8000;
                lo[j] = 0x7fff;
            }
            if (r < deep)
                for (int t = r; t < held; t += deep * AHEAD) {
                    s16x8 v[AHEAD];
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) v[k] = src[(int64_t)min(t + k * deep, held - 1) * wide];      // (one token twice makes no difference)
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const s16x8 x = ordered(v[k]);
                        hi = __builtin_elementwise_max(hi, x);
                        lo = __builtin_elementwise_min(lo, x);
                    }
                }
            for (int s = 32; s > 0; s >>= 1) {
                if (s >= deep) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // (a lane of the last group may be asked for by one that has no other: its own value then)
                    const int from = r + s < deep ? lane + s * wide : lane;
                    const s16x2 x = __builtin_bit_cast(s16x2, __shfl(__builtin_bit_cast(int, s16x2{hi[2 * j], hi[2 * j + 1]}), from));
                    const s16x2 y = __builtin_bit_cast(s16x2, __shfl(__builtin_bit_cast(int, s16x2{lo[2 * j], lo[2 * j + 1]}), from));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        hi[2 * j + e] = max(hi[2 * j + e], x[e]);
                        lo[2 * j + e] = min(lo[2 * j + e], y[e]);
                    }
                }
            }
            if (r == 0) {
                s16x8 x = ordered(hi), y = ordered(lo);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (hi[j] >= TOP || lo[j] <= -TOP - 1) x[j] = y[j] = 0x7fc0;
                *(s16x8*)out = x;
                *(s16x8*)(out + D) = y;
            }
        } else {
            const u32x4* const src = (const u32x4*)((const int8_t*)a.pool.k + (head << shift) * D) + c;
            const float* const scale = a.pool.k_scale + (head << shift);
            f32x16b hi, lo;
            float odd = 0.0f;       // NaN once a scale is not finite
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                hi[j] = -__builtin_inff();
                lo[j] = __builtin_inff();
            }
            if (r < deep)
                for (int t = r; t < held; t += deep * AHEAD) {
                    u32x4 v[AHEAD];
                    float f[AHEAD];
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const int at = min(t + k * deep, held - 1);
                        v[k] = src[(int64_t)at * wide];
                        f[k] = scale[at];
                    }
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        odd += f[k] * 0.0f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float x = (float)(int8_t)(v[k][j / 4] >> (8 * (j % 4))) * f[k];
                            hi[j] = fmaxf(hi[j], x);
                            lo[j] = fminf(lo[j], x);
                        }
                    }
                }
            for (int s = 32; s > 0; s >>= 1) {
                if (s >= deep) continue;
                const int from = r + s < deep ? lane + s * wide : lane;
                odd += __shfl(odd, from);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    hi[j] = fmaxf(hi[j], __shfl(hi[j], from));
                    lo[j] = fminf(lo[j], __shfl(lo[j], from));
                }
            }
            if (r == 0) {
                bf16x8 x[2], y[2];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const bool fine = odd == 0.0f && fabsf(hi[j]) <= 3.4e38f && fabsf(lo[j]) <= 3.4e38f;
                    x[j / 8][j % 8] = fine ? (__bf16)hi[j] : (__bf16)__builtin_nanf("");
                    y[j / 8][j % 8] = fine ? (__bf16)lo[j] : (__bf16)__builtin_nanf("");
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    *(bf16x8*)(out + 8 * j) = x[j];
                    *(bf16x8*)(out + D + 8 * j) = y[j];
                }
            }
        }
    }
}

int launch_bounds(const BoundsArgs& a, const spmm_cache_type_t type, const int64_t T, void* stream)
{
    // heads of pages that new tokens may lie in, at most; workgroups for them, in equal shares of the sequences, but no fewer than fill the device
    const int64_t n = a.batch.n_seqs, most = ((T >> a.pool.page_shift) + 2) * a.pool.n_heads, all = ((T >> a.pool.page_shift) + 2 * n) * a.pool.n_heads;
    const int64_t share = all / n > 2048 / n * WAVES ? all / n : 2048 / n * WAVES, heads = most < share ? most : share;
    const int64_t groups = (heads + WAVES - 1) / WAVES;
    // (sequences side by side: the device deals workgroups to its XCDs in turn, and the first ones of each sequence are those with work; 64
    // prompts of 100 tokens 4.7 us, 16.4 the other way round.  1024 to 4096 workgroups at least make no difference of 0.7 us.)
    const dim3 grid((unsigned)n, (unsigned)(groups < 65535 ? groups : 65535));
    return type == SPMM_CACHE_S8 ? launch(cache_bounds<SPMM_CACHE_S8>, grid, dim3(THREADS), a, stream) : launch(cache_bounds<SPMM_CACHE_BF16>, grid, dim3(THREADS), a, stream);
}

}  // namespace spmm_cache
