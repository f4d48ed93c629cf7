// One row of a page by one warp, in fp32 (what is looked at again of values that are not finite).
#pragma once

#include "paged.cuh"
#include "per_device.cuh"

#include <cuda_fp16.h>

namespace c2kv {
namespace {

// E4M3 codes of `w`'s low 16 bits as floats.
__device__ __forceinline__ float2 codes2(uint32_t w) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// The lane's D / 32 channels (from D / 32 * lane on) of a row at element offset `at`.
template <typename T, int D, bool kCodes>
__device__ __forceinline__ void lane_row(const void* base, int64_t at, float scale, int lane, float (&x)[D / 32]) {
    constexpr int C = D / 32;
    if constexpr (kCodes) {
        const uint8_t* p = static_cast<const uint8_t*>(base) + at + lane * C;
        if constexpr (C == 4) {
            const uint32_t w = ld_after(reinterpret_cast<const uint32_t*>(p));
            const float2 a = codes2(w), b = codes2(w >> 16);
            x[0] = a.x * scale;
            x[1] = a.y * scale;
            x[2] = b.x * scale;
            x[3] = b.y * scale;
        } else {
            const float2 a = codes2(ld_after(reinterpret_cast<const uint16_t*>(p)));
            x[0] = a.x * scale;
            x[1] = a.y * scale;
        }
    } else {
        const T* p = static_cast<const T*>(base) + at + lane * C;
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = static_cast<float>(p[e]);
    }
}

}  // namespace
}  // namespace c2kv
