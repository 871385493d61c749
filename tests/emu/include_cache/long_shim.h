// What the kernels for long contexts use beyond include/hip/hip_runtime.h: exchanges between lanes, matrix instructions of 16-bit floating-point
// numbers, atomics in LDS (a workgroup is one OS thread here), and launches by address.
#pragma once
#include <hip/hip_runtime.h>

#include <map>

typedef float emu_f32x4 __attribute__((ext_vector_type(4)));

struct int2 { int x, y; };
struct uint4 { unsigned x, y, z, w; };

namespace emu {
int shuffle(int v, int from);       // what lane `from` of the wave has
emu_f32x4 mfma_16x16x32(const float* a, const float* b, emu_f32x4 c);      // 8 values a lane each
template <typename V>
inline emu_f32x4 mfma(const V a, const V b, const emu_f32x4 c)
{
    float x[8], y[8];
    for (int i = 0; i < 8; ++i) x[i] = (float)a[i], y[i] = (float)b[i];
    return mfma_16x16x32(x, y, c);
}
inline int lane() { return threadIdx.x % 64; }
template <typename T>
inline T shfl(const T v, const int from)
{
    static_assert(sizeof(T) == 4, "");
    return __builtin_bit_cast(T, shuffle(__builtin_bit_cast(int, v), from & 63));
}
inline int before(const unsigned mask, const int at, const unsigned sum)
{
    const int n = lane() - at;
    return sum + __builtin_popcount(n <= 0 ? 0 : n >= 32 ? mask : mask & ((1u << n) - 1));
}

// kernels by their address
typedef std::function<void(dim3, dim3, void**)> Launch;
inline std::map<const void*, Launch>& kernels() { static std::map<const void*, Launch> k; return k; }
template <typename... A, size_t... I>
inline Launch launch_of(void (*kernel)(A...), std::index_sequence<I...>)
{
    return [=](dim3 grid, dim3 block, void** args) {
        const std::tuple<typename std::remove_const<A>::type...> held(*(typename std::remove_const<A>::type*)args[I]...);
        launch(grid, block, [=]() { kernel(std::get<I>(held)...); });
    };
}
template <typename... A>
inline const void* address(void (*kernel)(A...))
{
    kernels()[(const void*)kernel] = launch_of(kernel, std::index_sequence_for<A...>());
    return (const void*)kernel;
}
}  // namespace emu

static inline hipError_t hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void** args, size_t, hipStream_t)
{
    emu::kernels().at(kernel)(grid, block, args);
    return hipSuccess;
}

#define __shfl_xor(v, m) emu::shfl((v), emu::lane() ^ (int)(m))
#define __shfl(v, l) emu::shfl((v), (int)(l))
#define __shfl_up(v, n) emu::shfl((v), emu::lane() >= (int)(n) ? emu::lane() - (int)(n) : emu::lane())
#define __shfl_down(v, n) emu::shfl((v), emu::lane() + (int)(n) < 64 ? emu::lane() + (int)(n) : emu::lane())
#define __ballot(v) emu::ballot((bool)(v))
#define __any(v) (emu::ballot((bool)(v)) != 0)
#define __syncthreads_or(v) emu::together_or((bool)(v))
#define __builtin_amdgcn_mbcnt_lo(m, s) emu::before((m), 0, (s))
#define __builtin_amdgcn_mbcnt_hi(m, s) emu::before((m), 32, (s))
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) emu::mfma((a), (b), (c))
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) emu::mfma((a), (b), (c))
template <typename V>
static inline float emu_fdot2(const V a, const V b, const float c, bool) { return (float)a[0] * (float)b[0] + (float)a[1] * (float)b[1] + c; }
#define __builtin_amdgcn_fdot2_f32_bf16 emu_fdot2
#define __builtin_amdgcn_fdot2 emu_fdot2
#define __HIP_MEMORY_SCOPE_WORKGROUP 3
template <typename T, typename V>
static inline T emu_fetch_max(T* p, V v) { const T old = *p; *p = old < (T)v ? (T)v : old; return old; }
template <typename T, typename V>
static inline T emu_fetch_add(T* p, V v) { const T old = *p; *p = old + (T)v; return old; }
#define __hip_atomic_fetch_max(p, v, order, scope) emu_fetch_max((p), (v))
#define __hip_atomic_fetch_add(p, v, order, scope) emu_fetch_add((p), (v))

namespace emu { bool together_or(bool v); }
