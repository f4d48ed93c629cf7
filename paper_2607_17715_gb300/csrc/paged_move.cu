// Rows between a dense block and a paged cache: c2kv_paged_append writes new tokens' K (turned to
// their positions) and V, quantised where the pages hold E4M3; c2kv_paged_gather reads rows back.
//
// A row of one KV head is worked on by d / 2 / N threads, N elements to 16 bytes of the dense type:
// a thread holds N channels of the lower half and the N that they turn with, of K and of V, so four
// 16-byte loads are in flight a thread and the turn needs no exchange.  A CTA takes as many tokens as
// fill its threads with rows; their angles are formed once a token, in shared memory, while the rows
// are on their way, and serve every head.
#include "paged.cuh"
#include "rope.cuh"
#include "vec16.cuh"

#include <algorithm>
#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int kMoveThreads = 256;
constexpr int kMaxTokens = 32;          // tokens of a CTA (angles: 32 x 64 x 8 bytes)

// Two fp32 -> two E4M3 codes (round to nearest even, clamped to +-448), lo in the low byte.
__device__ __forceinline__ uint32_t to_codes2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 from_codes2(uint32_t w) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

template <int kReq>
__device__ __forceinline__ int find_request(const PagedMove<kReq>& P, int t) {
    int lo = 0, hi = P.batch;           // the last r with ptr[r] <= t (requests of no token are passed over)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (P.ptr[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The largest magnitude of a row's values as bits, over the threads that share the row: NaN and
// infinity compare above every finite value.
template <int kLanes>
__device__ __forceinline__ uint32_t row_top(uint32_t m) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// A row's scale and its inverse: the largest magnitude becomes 448, the type's largest value.  A row
// whose values are all below 2^-100 is kept as zero (the inverse of its scale could overflow); one
// with an infinity or a NaN gets scale NaN and codes 0, so that whoever sees the row sees NaN and the
// codes stay finite.
__device__ __forceinline__ float2 row_scale(uint32_t top) {
    if (top >= 0x7f800000u) return make_float2(__uint_as_float(0x7fc00000u), 0.f);
    if (top < 0x0d800000u) return make_float2(0.f, 0.f);
    const float s = __fmul_rn(__uint_as_float(top), 1.0f / 448.0f);
    return make_float2(s, __fdiv_rn(1.0f, s));
}

template <int N>
__device__ __forceinline__ void store_codes(void* dst, const float* x, float inv) {
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
        w[i] = to_codes2(x[4 * i] * inv, x[4 * i + 1] * inv) | to_codes2(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16;
    if constexpr (N == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(dst) = w[0];
}

template <int N>
__device__ __forceinline__ void load_codes(const void* src, float* x, float scale) {
    uint32_t w[N / 4];
    if constexpr (N == 8) {
        const uint2 t = __ldg(reinterpret_cast<const uint2*>(src));
        w[0] = t.x;
        w[1] = t.y;
    } else {
        w[0] = __ldg(reinterpret_cast<const uint32_t*>(src));
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const float2 a = from_codes2(w[i]), b = from_codes2(w[i] >> 16);
        x[4 * i] = a.x * scale;
        x[4 * i + 1] = a.y * scale;
        x[4 * i + 2] = b.x * scale;
        x[4 * i + 3] = b.y * scale;
    }
}

template <typename T, int D, bool kCodes, bool kAppend, int kReq>
__global__ void __launch_bounds__(kMoveThreads) paged_move_kernel(const __grid_constant__ PagedMove<kReq> P) {
    constexpr int N = Vec16<T>::N;
    constexpr int kLanes = D / 2 / N;                 // threads a row
    constexpr int kRows = kMoveThreads / kLanes;      // rows a pass
    __shared__ float2 s_cs[kMaxTokens * (D / 2)];
    const int t0 = P.t0 + blockIdx.x * P.tokens_per_cta;
    const int nt = min(P.tokens_per_cta, P.t1 - t0);
    const int lane = threadIdx.x % kLanes, c = lane * N;   // channels c .. and c + D / 2 ..
    const int page_size = 1 << P.pg.page_shift;
    const int n_rows = nt * P.hkv;
    bool angles = P.turn == nullptr;
    // every thread of the CTA makes the same passes (shuffles and the barrier below)
    for (int i0 = 0; i0 < n_rows; i0 += kRows) {
        const int i = i0 + threadIdx.x / kLanes;
        const bool live = i < n_rows;
        const int tl = live ? i / P.hkv : 0, h = live ? i - tl * P.hkv : 0, t = t0 + tl;
        T* const dk = static_cast<T*>(P.k) + (int64_t)t * P.stride + (int64_t)h * D + c;
        T* const dv = static_cast<T*>(P.v) + (int64_t)t * P.stride + (int64_t)h * D + c;
        uint4 rk[2], rv[2];
        if (kAppend && live) {
            rk[0] = ld16(dk);
            rk[1] = ld16(dk + D / 2);
            rv[0] = ld16(dv);
            rv[1] = ld16(dv + D / 2);
        }
        const int r = find_request(P, t);
        const int row = P.start[r] + (t - P.ptr[r]);
        const int page = live ? __ldg(P.pg.table + (int64_t)(P.b0 + r) * P.pg.table_stride + (row >> P.pg.page_shift)) : 0;
        const bool ok = live && page >= 0 && page < P.pg.n_pages;
        if (live && !ok && lane == 0) atomicOr(P.err, 1);
        const int64_t in_page = (int64_t)h * page_size + (row & (page_size - 1));
        const int64_t at = (int64_t)page * P.pg.page_stride + in_page * D + c;
        const int64_t sat = (int64_t)page * P.pg.scale_stride + in_page;
        float xk[2 * N], xv[2 * N];
        if constexpr (kAppend) {
            if (live) {
                Vec16<T>::unpack(rk[0], xk);
                Vec16<T>::unpack(rk[1], xk + N);
                Vec16<T>::unpack(rv[0], xv);
                Vec16<T>::unpack(rv[1], xv + N);
            } else {
#pragma unroll
                for (int e = 0; e < 2 * N; ++e) xk[e] = xv[e] = 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 2 * N; ++e) xk[e] = xv[e] = 0.f;
            if (ok) {
                if constexpr (kCodes) {
                    const uint8_t* pk = static_cast<const uint8_t*>(P.pg.k) + at;
                    const uint8_t* pv = static_cast<const uint8_t*>(P.pg.v) + at;
                    const float sk = __ldg(P.pg.k_scale + sat), sv = __ldg(P.pg.v_scale + sat);
                    load_codes<N>(pk, xk, sk);
                    load_codes<N>(pk + D / 2, xk + N, sk);
                    load_codes<N>(pv, xv, sv);
                    load_codes<N>(pv + D / 2, xv + N, sv);
                } else {
                    const T* pk = static_cast<const T*>(P.pg.k) + at;
                    const T* pv = static_cast<const T*>(P.pg.v) + at;
                    rk[0] = ld16(pk);
                    rk[1] = ld16(pk + D / 2);
                    rv[0] = ld16(pv);
                    rv[1] = ld16(pv + D / 2);
                    Vec16<T>::unpack(rk[0], xk);
                    Vec16<T>::unpack(rk[1], xk + N);
                    Vec16<T>::unpack(rv[0], xv);
                    Vec16<T>::unpack(rv[1], xv + N);
                }
            }
        }
        if (!angles) {
            for (int a = threadIdx.x; a < nt * (D / 2); a += kMoveThreads)
                s_cs[a] = turn_cs(lane_turn(P.rope.turn, a % (D / 2)), __ldg(P.turn + t0 + a / (D / 2)));
            __syncthreads();
            angles = true;
        }
        if (P.turn) {
            float lo[N], hi[N];
            rotate<N>(xk, xk + N, s_cs + tl * (D / 2) + c, lo, hi);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                xk[e] = lo[e];
                xk[N + e] = hi[e];
            }
        }
        if constexpr (kAppend && kCodes) {
            uint32_t mk = 0, mv = 0;
#pragma unroll
            for (int e = 0; e < 2 * N; ++e) {
                mk = max(mk, __float_as_uint(xk[e]) & 0x7fffffffu);
                mv = max(mv, __float_as_uint(xv[e]) & 0x7fffffffu);
            }
            const float2 sk = row_scale(row_top<kLanes>(mk)), sv = row_scale(row_top<kLanes>(mv));
            if (ok) {
                if (sk.y == 0.f)           // kept as zero, or NaN: codes 0
#pragma unroll
                    for (int e = 0; e < 2 * N; ++e) xk[e] = 0.f;
                if (sv.y == 0.f)
#pragma unroll
                    for (int e = 0; e < 2 * N; ++e) xv[e] = 0.f;
                uint8_t* pk = static_cast<uint8_t*>(P.pg.k) + at;
                uint8_t* pv = static_cast<uint8_t*>(P.pg.v) + at;
                store_codes<N>(pk, xk, sk.y);
                store_codes<N>(pk + D / 2, xk + N, sk.y);
                store_codes<N>(pv, xv, sv.y);
                store_codes<N>(pv + D / 2, xv + N, sv.y);
                if (lane == 0) {
                    P.pg.k_scale[sat] = sk.x;
                    P.pg.v_scale[sat] = sv.x;
                }
            }
        } else if (kAppend ? ok : live) {
            T* const ok_ = kAppend ? static_cast<T*>(P.pg.k) + at : dk;
            T* const ov_ = kAppend ? static_cast<T*>(P.pg.v) + at : dv;
            st16(ok_, Vec16<T>::pack(xk));
            st16(ok_ + D / 2, Vec16<T>::pack(xk + N));
            st16(ov_, Vec16<T>::pack(xv));
            st16(ov_ + D / 2, Vec16<T>::pack(xv + N));
        }
    }
}

template <typename T, int D, bool kCodes, bool kAppend, int kReq>
cudaError_t launch_move(const PagedMoveCall& c, cudaStream_t s) {
    constexpr int kRows = kMoveThreads / (D / 2 / Vec16<T>::N);
    for (int b0 = 0; b0 < c.batch; b0 += kReq) {
        const int nb = std::min(c.batch - b0, kReq);
        PagedMove<kReq> P;
        P.pg = c.pg;
        P.k = c.k;
        P.v = c.v;
        P.stride = c.stride;
        P.turn = c.turn;
        P.err = c.err;
        P.batch = nb;
        P.b0 = b0;
        P.hkv = c.hkv;
        P.tokens_per_cta = std::max(1, std::min(kRows / c.hkv, kMaxTokens));
        P.t0 = c.ptr[b0];
        P.t1 = c.ptr[b0 + nb];
        if (P.t1 == P.t0) continue;
        P.rope = *c.rope;
        for (int i = 0; i <= nb; ++i) P.ptr[i] = c.ptr[b0 + i];
        for (int i = 0; i < nb; ++i) P.start[i] = c.start[b0 + i];
        const int ctas = (P.t1 - P.t0 + P.tokens_per_cta - 1) / P.tokens_per_cta;
        paged_move_kernel<T, D, kCodes, kAppend, kReq><<<ctas, kMoveThreads, 0, s>>>(P);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, int D, bool kAppend>
cudaError_t move_of(const PagedMoveCall& c, bool codes, cudaStream_t s) {
    const bool few = c.batch <= kPagedFew;
    if (codes)
        return few ? launch_move<T, D, true, kAppend, kPagedFew>(c, s) : launch_move<T, D, true, kAppend, kPagedMany>(c, s);
    return few ? launch_move<T, D, false, kAppend, kPagedFew>(c, s) : launch_move<T, D, false, kAppend, kPagedMany>(c, s);
}

template <bool kAppend>
cudaError_t move_rows(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    if (dtype == kDtypeF32)
        return d == 128 ? move_of<float, 128, kAppend>(c, codes, s) : move_of<float, 64, kAppend>(c, codes, s);
    return d == 128 ? move_of<__nv_bfloat16, 128, kAppend>(c, codes, s) : move_of<__nv_bfloat16, 64, kAppend>(c, codes, s);
}

// ------------------------------------------------------------------ 8-bit pages as 16-bit ones

constexpr int kExpandThreads = 256;

template <int kReq>
struct PagedExpand {
    PageView from, to;
    int32_t* err;
    int32_t hkv;
    int32_t n;
    int32_t item0[kReq + 1];     // pages of the launch before request i's
    int32_t row[kReq];           // its row of from.table
    int32_t page0[kReq];         // its first page there
    int32_t first[kReq];         // the page of `to` that this becomes
};

// One page of one KV head a CTA: K and V, 16 codes a thread and pass.  A code times its scale is rounded
// to bf16 (2^-9 of it), as the rows of 16-bit pages are: the products that read it are of bf16.  Bytes
// bound it: one read, two written for each code.
template <int D, int kReq>
__global__ void __launch_bounds__(kExpandThreads) paged_expand_kernel(const __grid_constant__ PagedExpand<kReq> P) {
    using T = __nv_bfloat16;
    int r = 0;
    for (int hi = P.n; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.item0[mid] <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    const int i = blockIdx.x - P.item0[r], h = blockIdx.y, size = 1 << P.from.page_shift;
    const int page = __ldg(P.from.table + (int64_t)P.row[r] * P.from.table_stride + P.page0[r] + i);
    const bool ok = page >= 0 && page < P.from.n_pages;
    if (threadIdx.x == 0 && h == 0) {
        const_cast<int32_t*>(P.to.table)[(int64_t)r * P.to.table_stride + P.page0[r] + i] = ok ? P.first[r] + i : -1;
        if (!ok) atomicOr(P.err, 1);
    }
    if (!ok) return;
    constexpr int kChunks = D / 16;
    const int64_t from = (int64_t)page * P.from.page_stride + (int64_t)h * size * D;
    const int64_t sfrom = (int64_t)page * P.from.scale_stride + (int64_t)h * size;
    const int64_t to = (int64_t)(P.first[r] + i) * P.to.page_stride + (int64_t)h * size * D;
    for (int e = threadIdx.x; e < 2 * size * kChunks; e += kExpandThreads) {
        const bool v = e >= size * kChunks;
        const int c = v ? e - size * kChunks : e;
        const uint8_t* src = static_cast<const uint8_t*>(v ? P.from.v : P.from.k) + from + (int64_t)c * 16;
        const float s = __ldg((v ? P.from.v_scale : P.from.k_scale) + sfrom + c / kChunks);
        const uint4 w = ld16(src);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        float f[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 a = from_codes2(x[k]), b = from_codes2(x[k] >> 16);
            f[4 * k] = a.x * s;
            f[4 * k + 1] = a.y * s;
            f[4 * k + 2] = b.x * s;
            f[4 * k + 3] = b.y * s;
        }
        T* dst = static_cast<T*>(v ? P.to.v : P.to.k) + to + (int64_t)c * 16;
        st16(dst, Vec16<T>::pack(f));
        st16(dst + 8, Vec16<T>::pack(f + 8));
    }
}

template <int D, int kReq>
cudaError_t launch_expand(const PagedExpandCall& c, cudaStream_t s) {
    for (int b0 = 0; b0 < c.n; b0 += kReq) {
        const int nb = std::min(c.n - b0, kReq);
        PagedExpand<kReq> P;
        P.from = c.from;
        P.to = c.to;
        P.to.table += (int64_t)b0 * c.to.table_stride;
        P.err = c.err;
        P.hkv = c.hkv;
        P.n = nb;
        int items = 0;
        for (int i = 0; i < nb; ++i) {
            P.item0[i] = items;
            P.row[i] = c.req[b0 + i].row;
            P.page0[i] = c.page0[b0 + i];
            P.first[i] = c.first[b0 + i];
            items += c.pages[b0 + i];
        }
        P.item0[nb] = items;
        if (items == 0) continue;
        paged_expand_kernel<D, kReq><<<dim3(items, c.hkv), kExpandThreads, 0, s>>>(P);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_paged_expand(const PagedExpandCall& c, int d, cudaStream_t s) {
    if (c.n <= kPagedFew) return d == 128 ? launch_expand<128, kPagedFew>(c, s) : launch_expand<64, kPagedFew>(c, s);
    return d == 128 ? launch_expand<128, kPagedMany>(c, s) : launch_expand<64, kPagedMany>(c, s);
}

cudaError_t launch_paged_append(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    return move_rows<true>(c, dtype, d, codes, s);
}
cudaError_t launch_paged_gather(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    return move_rows<false>(c, dtype, d, codes, s);
}

}  // namespace c2kv
