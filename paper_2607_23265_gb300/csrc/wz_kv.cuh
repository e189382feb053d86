// What the kernels of the paged 8-bit cache share: e4m3 conversions, page
// scales, the sequence of a unit.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "../../include/wavezip.h"

namespace wz {

constexpr int kScaleLow = -60, kScaleHigh = 60;   // exponents of a page's scale

__device__ __forceinline__ void kv_report(int *status) {
    if (status) atomicOr(status, WZ_STATUS_CACHE);
}

// (lo, hi) to two e4m3 codes, lo in the low byte: nearest, ties to even,
// saturating at +-448.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// The same of two halves.
__device__ __forceinline__ uint32_t e4m3x2(__half2 v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t *>(&v)));
    return r;
}

// Two e4m3 codes as two halves (exact).
__device__ __forceinline__ __half2 half2_of_e4m3(uint16_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(codes));
    return *reinterpret_cast<const __half2 *>(&r);
}

// Four codes, each times a power of two, rounded to e4m3 again.
__device__ __forceinline__ uint32_t e4m3x4_times(uint32_t codes, float f) {
    const float2 a = __half22float2(half2_of_e4m3((uint16_t)(codes & 0xFFFFu)));
    const float2 b = __half22float2(half2_of_e4m3((uint16_t)(codes >> 16)));
    return e4m3x2(a.x * f, a.y * f) | (e4m3x2(b.x * f, b.y * f) << 16);
}

// The smallest power of two s in [2^kScaleLow, 2^kScaleHigh] with x <= 448 s, or
// the largest; x >= 0 finite, as its bits.  448 = 1.75 * 2^8.
__device__ __forceinline__ float fitting_scale(uint32_t bits) {
    int n = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    n = min(max(n, kScaleLow), kScaleHigh);
    return __uint_as_float((uint32_t)(n + 127) << 23);
}

// The sequence b with (cu[b] >> shift) + 2b <= u < (cu[b+1] >> shift) + 2(b+1), by all lanes of
// a warp: 32 places at a time.
__device__ __forceinline__ int kv_find_sequence(const int32_t *cu, int B, int u, int shift) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = B;   // the sequence lies in [lo, hi)
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) >> 5;
        const int at = lo + lane * step;
        const bool before = at < hi && (cu[at] >> shift) + 2 * at <= u;
        const int n = max(__popc(__ballot_sync(0xFFFFFFFFu, before)), 1);
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

}  // namespace wz
