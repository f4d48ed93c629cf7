// Attention of each request's new tokens over its paged cache (c2kv_paged_attend).
#include "paged.cuh"
#include "paged_row.cuh"

#include <algorithm>

namespace c2kv {
namespace {

constexpr int kRowWarps = 4;

// One query row a CTA, its keys dealt to four warps.
template <typename T, int D, bool kCodes, int kReq>
__global__ void __launch_bounds__(kRowWarps * 32) paged_row_kernel(const __grid_constant__ PagedAttn<kReq> P) {
    constexpr int C = D / 32;
    __shared__ float s_m[kRowWarps], s_l[kRowWarps], s_o[kRowWarps][D];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t t = P.req[0].q0 + blockIdx.x / P.hq;
    const int h = blockIdx.x % P.hq, hk = h / (P.hq / P.hkv);
    int r = 0;
    while (t >= P.req[r].q0 + P.req[r].nq) ++r;
    const PagedReq R = P.req[r];
    const int hi = R.n_keys - R.nq + (int)(t - R.q0) + 1;
    const int lo = P.window ? max(0, hi - P.window) : 0;
    float q[C], o[C], m, l;
    lane_query<T, D>(P, t, h, lane, q);
    row_attend<T, D, kCodes>(P, q, r, hk, lo + warp, hi, kRowWarps, lane, m, l, o);
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
#pragma unroll
    for (int e = 0; e < C; ++e) s_o[warp][lane * C + e] = o[e];
    __syncthreads();
    if (warp) return;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) top = fmaxf(top, s_m[w]);
    float acc[C] = {};
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) {
        const float f = s_m[w] == top ? (s_l[w] == 0.f ? 0.f : 1.f) : exp2f(s_m[w] - top);
        sum += s_l[w] * f;
#pragma unroll
        for (int e = 0; e < C; ++e) acc[e] += f == 0.f ? 0.f : s_o[w][lane * C + e] * f;
    }
    T* out = static_cast<T*>(P.out) + (t * P.hq + h) * D + lane * C;
#pragma unroll
    for (int e = 0; e < C; ++e) out[e] = static_cast<T>(sum == 0.f ? 0.f : acc[e] / sum);
    if (P.lse && lane == 0) P.lse[(int64_t)h * P.n_tokens + t] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

template <int kReq>
void fill(PagedAttn<kReq>& P, const PagedAttnCall& c, int d, int b0, int nb) {
    P.pg = c.pg;
    P.q = c.q;
    P.out = c.out;
    P.lse = c.lse;
    P.turn = c.turn;
    P.err = c.err;
    P.q_stride = c.q_stride;
    P.n_tokens = c.ptr[c.batch];
    P.batch = nb;
    P.b0 = b0;
    P.hq = c.hq;
    P.hkv = c.hkv;
    P.window = c.window;
    P.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)d));
    P.rope = *c.rope;
    for (int i = 0; i < nb; ++i)
        P.req[i] = PagedReq{c.ptr[b0 + i], c.ptr[b0 + i + 1] - c.ptr[b0 + i], c.n_keys[b0 + i], 0};
}

template <typename T, int D, bool kCodes, int kReq>
cudaError_t launch_rows(const PagedAttnCall& c, cudaStream_t s) {
    for (int b0 = 0; b0 < c.batch; b0 += kReq) {
        const int nb = std::min(c.batch - b0, kReq);
        PagedAttn<kReq> P;
        fill(P, c, D, b0, nb);
        const int tokens = c.ptr[b0 + nb] - c.ptr[b0];
        if (!tokens) continue;
        paged_row_kernel<T, D, kCodes, kReq><<<tokens * c.hq, kRowWarps * 32, 0, s>>>(P);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, int D>
cudaError_t rows_of(const PagedAttnCall& c, bool codes, cudaStream_t s) {
    const bool few = c.batch <= kPagedFew;
    if (codes) return few ? launch_rows<T, D, true, kPagedFew>(c, s) : launch_rows<T, D, true, kPagedMany>(c, s);
    return few ? launch_rows<T, D, false, kPagedFew>(c, s) : launch_rows<T, D, false, kPagedMany>(c, s);
}

}  // namespace

cudaError_t launch_paged_attn(const PagedAttnCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    if (dtype == kDtypeF32) return d == 128 ? rows_of<float, 128>(c, codes, s) : rows_of<float, 64>(c, codes, s);
    return d == 128 ? rows_of<__nv_bfloat16, 128>(c, codes, s) : rows_of<__nv_bfloat16, 64>(c, codes, s);
}

}  // namespace c2kv
