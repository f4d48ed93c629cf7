// RoPE angles and the 2x2 rotation shared by the streaming kernels.  Channel i pairs with
// i + d/2 and turns by pos * theta^(-2i/d); the angle comes from the phase accumulator in
// RopeTurns (the low 64 bits of pos * turn[i] are the exact fractional turn) and sincospif.
#pragma once

#include <cstdint>

namespace c2kv {
namespace {

__device__ __forceinline__ float2 turn_cs(uint64_t turn, int64_t pos) {
    const uint64_t frac = (uint64_t)pos * turn;                 // turns mod 1, exact
    const float x = (float)(long long)frac * 0x1p-63f;          // 2 * turns in [-1, 1)
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(c, s);
}

// The same from the special-function unit, for rows that are rounded to 11 bits or fewer right after:
// its sine and cosine of an angle in [-pi, pi) are within 2^-20, a thousandth of that rounding, at a
// tenth of the instructions.
__device__ __forceinline__ float2 turn_cs_fast(uint64_t turn, int64_t pos) {
    const int32_t frac = (int32_t)(((uint64_t)pos * turn) >> 32);       // turns mod 1, in 2^-32
    const float a = (float)frac * 1.46291808e-9f;                       // 2 pi / 2^32
    return make_float2(__cosf(a), __sinf(a));
}

// Frequency i of a table in a kernel's parameters, for an index that differs from lane to lane: an
// ordinary load, since the constant cache serves one address of a warp at a time (a prologue that read
// 64 frequencies a token took 9 us that way, 1 so).
__device__ __forceinline__ uint64_t lane_turn(const uint64_t* turns, int i) {
    uint64_t v;
    asm volatile("ld.u64 %0, [%1];" : "=l"(v) : "l"(turns + i));
    return v;
}

// (x, y) turned by the angle whose (cos, sin) is cs, with the rounding spelled out (one
// product rounded, then a fused multiply-add) so that every kernel that turns a pair gets
// the same bits.
__device__ __forceinline__ void rotate1(float x, float y, float2 cs, float& ox, float& oy) {
    ox = __fmaf_rn(x, cs.x, -__fmul_rn(y, cs.y));
    oy = __fmaf_rn(x, cs.y, __fmul_rn(y, cs.x));
}

template <int E>
__device__ __forceinline__ void rotate(const float* x, const float* y, const float2* cs,
                                       float* ox, float* oy) {
#pragma unroll
    for (int e = 0; e < E; ++e) rotate1(x[e], y[e], cs[e], ox[e], oy[e]);
}

}  // namespace
}  // namespace c2kv
