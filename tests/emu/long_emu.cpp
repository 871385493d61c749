// The host emulation (emu.cpp) for the kernels of long contexts: what include_cache/long_shim.h declares, and the calls of the paged cache that
// are not emulated.
#define spmm_measure_peak emu_measure_peak      // (declared with another type in the header that follows)
#include "emu.cpp"
#undef spmm_measure_peak

#include "long_shim.h"

#include "cache_internal.h"

namespace emu {

int shuffle(const int v, const int from)
{
    Wave& w = my_wave();
    w.iv[cur()->linear & 63] = v;
    wave_sync(w, "shuffle (deposit)");
    const int r = w.iv[from];
    wave_sync(w, "shuffle (collect)");
    return r;
}

// D[row][col] += sum over k of A[row][k] B[k][col]: lane l has row, or column, l % 16 and k 8 (l / 16) .. of A and B; column l % 16 and rows 4 (l / 16) .. of D
emu_f32x4 mfma_16x16x32(const float* const a, const float* const b, emu_f32x4 c)
{
    Wave& w = my_wave();
    const int lane = cur()->linear & 63;
    static thread_local float of_a[16][64][8], of_b[16][64][8];
    const int wave = cur()->linear / 64;
    memcpy(of_a[wave][lane], a, 32);
    memcpy(of_b[wave][lane], b, 32);
    wave_sync(w, "mfma (deposit)");
    for (int r = 0; r < 4; ++r) {
        float sum = 0.0f;
        for (int k = 0; k < 32; ++k) sum += of_a[wave][16 * (k / 8) + 4 * (lane / 16) + r][k % 8] * of_b[wave][16 * (k / 8) + lane % 16][k % 8];
        c[r] += sum;
    }
    wave_sync(w, "mfma (collect)");
    return c;
}

bool together_or(const bool v)
{
    static thread_local bool any;
    syncthreads();
    any = false;
    syncthreads();
    any |= v;
    syncthreads();
    return any;
}

}  // namespace emu

// rounding to 16 bits, which the compiler calls for and the host's library need not have
extern "C" __bf16 __truncsfbf2(const float x)
{
    uint32_t u;
    memcpy(&u, &x, 4);
    u = x != x ? u >> 16 | 64 : (u + 0x7fff + (u >> 16 & 1)) >> 16;
    const uint16_t h = (uint16_t)u;
    __bf16 y;
    memcpy(&y, &h, 2);
    return y;
}

namespace spmm_cache {
int launch_append(const AppendArgs&, spmm_out_t, spmm_cache_type_t, void*) { return 1; }
int launch_attend(const AttendArgs&, spmm_cache_type_t, void*) { return 1; }
int64_t attend_work_bytes(spmm_cache_type_t, int64_t, int32_t, int32_t, int32_t, int64_t) { return 16; }
int launch_copy(const CopyArgs&, void*) { return 1; }
int launch_fork(const ForkArgs&, const CopyArgs&, void*) { return 1; }
int launch_compact(const CompactArgs&, const CopyArgs&, void*) { return 1; }
}  // namespace spmm_cache
