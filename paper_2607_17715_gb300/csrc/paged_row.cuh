// One query row of paged attention by one warp on the CUDA cores, in fp32: the keys it sees one
// after the other, so that no key that it does not see takes part in any sum, whatever it holds.
#pragma once

#include "paged.cuh"
#include "per_device.cuh"
#include "rope.cuh"

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

// The lane's channels of query row (token t, head h), turned, in fp32.
template <typename T, int D, int kReq>
__device__ __forceinline__ void lane_query(const PagedAttn<kReq>& P, int64_t t, int h, int lane, float (&x)[D / 32]) {
    constexpr int C = D / 32;
    const T* q = static_cast<const T*>(P.q) + t * P.q_stride + (int64_t)h * D;
    const bool low = lane < 16;
    const int c = (lane & 15) * C;               // first of the lane's channels, within its half
#pragma unroll
    for (int e = 0; e < C; ++e) {
        const float lo = static_cast<float>(q[c + e]), hi = static_cast<float>(q[c + D / 2 + e]);
        float a = lo, b = hi;
        if (P.turn) rotate1(lo, hi, turn_cs(lane_turn(P.rope.turn, c + e), ld_after(P.turn + t)), a, b);
        x[e] = low ? a : b;
    }
}

// Rows lo .. hi - 1 of the request at row `r` of the table: the largest score m (log2 domain),
// the sum l of 2^(score - m), and the lane's channels of the sum of 2^(score - m) v.
template <typename T, int D, bool kCodes, int kReq>
__device__ __forceinline__ void row_attend(const PagedAttn<kReq>& P, const float (&q)[D / 32], int r, int hk, int lo, int hi,
                                           int lane, float& m, float& l, float (&o)[D / 32]) {
    constexpr int C = D / 32;
    const int page_size = 1 << P.pg.page_shift;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < C; ++e) o[e] = 0.f;
    for (int j = lo; j < hi; ++j) {
        const int page = ld_after(P.pg.table + (int64_t)r * P.pg.table_stride + (j >> P.pg.page_shift));
        if (page < 0 || page >= P.pg.n_pages) {
            if (lane == 0) atomicOr(P.err, 1);
            continue;
        }
        const int64_t in_page = (int64_t)hk * page_size + (j & (page_size - 1));
        const int64_t at = (int64_t)page * P.pg.page_stride + in_page * D, sat = (int64_t)page * P.pg.scale_stride + in_page;
        float k[C], v[C];
        lane_row<T, D, kCodes>(P.pg.k, at, kCodes ? ld_after(P.pg.k_scale + sat) : 1.f, lane, k);
        lane_row<T, D, kCodes>(P.pg.v, at, kCodes ? ld_after(P.pg.v_scale + sat) : 1.f, lane, v);
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < C; ++e) s = fmaf(q[e], k[e], s);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= P.scale_log2;
        const float top = fmaxf(m, s);
        // a first score of -inf would make -inf - -inf of the rescale: nothing is summed yet, keep it at 1
        const float f = m == top ? 1.f : exp2f(m - top), w = s == -INFINITY && top == -INFINITY ? 0.f : exp2f(s - top);
        m = top;
        l = l * f + w;
#pragma unroll
        for (int e = 0; e < C; ++e) o[e] = fmaf(w, v[e], o[e] * f);
    }
}

}  // namespace
}  // namespace c2kv
