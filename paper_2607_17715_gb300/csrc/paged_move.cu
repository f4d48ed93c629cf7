// Rows between a dense block and a paged cache: c2kv_paged_append writes new tokens' K (turned to
// their positions) and V, quantised where the pages hold E4M3; c2kv_paged_gather reads rows back.
//
// A row of one KV head is worked on by d / 2 / N threads, N elements to 16 bytes of the dense type:
// a thread holds N channels of the lower half and the N that they turn with, of K and of V, and works on
// kU rows at once, so the turn needs no exchange and 64 kU bytes a thread are on their way.  A CTA takes
// several tokens with all their heads: their pages are looked up and their angles formed once a token, in
// shared memory, while the first rows are on their way.
//
// Bytes bound it, and for a token or two the launch.  Measured: 16 requests' contexts read back, 480 MB in
// 73 us (6.6 TB/s); prompts of eight requests appended as codes, 138 MB in 29 us (4.7 TB/s: the CTAs are
// short, and their chain position -> angle -> turn -> largest value is a fifth of it; launched
// with no overlap 32, without a turn 27, with 16-bit pages, a third more bytes, 32).  Angles formed by each thread for itself, with no shared
// memory between, took 38 of the 32; more passes a CTA 34; more CTAs an SM with fewer registers 36.  The
// special-function unit's sine and cosine save half a microsecond and move codes that lie near the middle
// between two: angles are fp32's.
#include "paged.cuh"
#include "per_device.cuh"
#include "rope.cuh"
#include "vec16.cuh"

#include <algorithm>
#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int kMoveThreads = 128;
constexpr int kMaxTokens = 32;          // tokens of a CTA (angles: 32 x 64 x 8 bytes)
// Rows of a thread on their way at once: two of what is read back; one of what is appended, whose maxima
// and turns need the registers (16 requests' contexts read back: 76 us with two, 84 with one; prompts
// appended: 34 and 32).
__host__ __device__ constexpr int rows_at_once(bool append) { return append ? 1 : 2; }
constexpr int kMovePasses = 2;          // passes of a CTA

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
    return make_float2(s, __frcp_rn(s));
}

// N codes of x * inv; inv = 0 (a row kept as zero, or not a number): codes 0.
template <int N>
__device__ __forceinline__ void store_codes(void* dst, const float* x, float inv) {
    uint32_t w[N / 4] = {};
    if (inv != 0.f)
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            w[i] = to_codes2(x[4 * i] * inv, x[4 * i + 1] * inv) | to_codes2(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16;
    if constexpr (N == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(dst) = w[0];
}

template <int N>
__device__ __forceinline__ uint2 ld_codes(const void* src) {
    if constexpr (N == 8) return ld_after(reinterpret_cast<const uint2*>(src));
    else return make_uint2(ld_after(reinterpret_cast<const uint32_t*>(src)), 0u);
}

template <int N>
__device__ __forceinline__ void from_codes(const uint2& w, float* x, float scale) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t v = i ? w.y : w.x;
        const float2 a = from_codes2(v), b = from_codes2(v >> 16);
        x[4 * i] = a.x * scale;
        x[4 * i + 1] = a.y * scale;
        x[4 * i + 2] = b.x * scale;
        x[4 * i + 3] = b.y * scale;
    }
}

// 2 N channels of a row, in two halves: c .. and D / 2 + c ..
template <typename T>
struct Halves {
    uint4 lo, hi;
    __device__ __forceinline__ void load(const T* p, int half) {
        lo = ld_after(reinterpret_cast<const uint4*>(p));
        hi = ld_after(reinterpret_cast<const uint4*>(p + half));
    }
    __device__ __forceinline__ void unpack(float* x) const {
        Vec16<T>::unpack(lo, x);
        Vec16<T>::unpack(hi, x + Vec16<T>::N);
    }
};

// The largest magnitude of a thread's values as bits: NaN if any is (an infinity and a NaN alike make the
// row's scale one).
template <int M>
__device__ __forceinline__ uint32_t top_of(const float* x) {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < M; e += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(x[e]), "f"(x[e + 1]));
    return __float_as_uint(m);
}

template <typename T, int D, bool kCodes, bool kAppend, int kReq>
__global__ void __launch_bounds__(kMoveThreads) paged_move_kernel(const __grid_constant__ PagedMove<kReq> P) {
    constexpr int N = Vec16<T>::N, kU = rows_at_once(kAppend);
    constexpr int kLanes = D / 2 / N;                 // threads a row
    constexpr int kRows = kMoveThreads / kLanes;      // rows a pass of one row a thread
    __shared__ float2 s_cs[kMaxTokens * (D / 2)];
    __shared__ int64_t s_at[kMaxTokens], s_sat[kMaxTokens];   // where a token's row of head 0 is, in elements and scales
    const int t0 = P.t0 + blockIdx.x * P.tokens_per_cta;
    const int nt = min(P.tokens_per_cta, P.t1 - t0);
    const int lane = threadIdx.x % kLanes, c = lane * N;   // channels c .. and c + D / 2 ..
    const int size = 1 << P.pg.page_shift, n_rows = nt * P.hkv;
    T* const dense_k = static_cast<T*>(P.k) + (int64_t)t0 * P.stride + c;
    T* const dense_v = static_cast<T*>(P.v) + (int64_t)t0 * P.stride + c;
    Halves<T> rk[kU], rv[kU];
    int tl[kU], h[kU];                                // token of the CTA and head of each row
    bool live[kU];
    int64_t dense[kU];
    // (threads past the rows take the last one along, and store nothing)
    auto rows_of = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int want = i0 + u * kRows + threadIdx.x / kLanes, i = min(want, n_rows - 1);
            live[u] = want < n_rows;
            tl[u] = (int)(((float)i + 0.5f) * P.per_hkv);      // i / hkv: i is far below 2^20
            h[u] = i - tl[u] * P.hkv;
            dense[u] = (int64_t)tl[u] * P.stride + h[u] * D;
            if (kAppend) {
                rk[u].load(dense_k + dense[u], D / 2);
                rv[u].load(dense_v + dense[u], D / 2);
            }
        }
    };
    after_kernels_before();
    rows_of(0);
    if (threadIdx.x < nt) {                           // one token a thread: its request, row and page
        const int t = t0 + threadIdx.x, r = find_request(P, t), row = P.start[r] + (t - P.ptr[r]);
        const int page = ld_after(P.pg.table + (int64_t)(P.b0 + r) * P.pg.table_stride + (row >> P.pg.page_shift));
        const bool ok = page >= 0 && page < P.pg.n_pages;
        if (!ok) atomicOr(P.err, 1);
        s_at[threadIdx.x] = ok ? page * P.pg.page_stride + (int64_t)(row & (size - 1)) * D : -1;
        s_sat[threadIdx.x] = page * P.pg.scale_stride + (row & (size - 1));
    }
    if (P.turn)
        for (int a = threadIdx.x; a < nt * (D / 2); a += kMoveThreads) {
            const uint64_t turn = lane_turn(P.rope.turn, a % (D / 2));
            s_cs[a] = turn_cs(turn, ld_after(P.turn + t0 + a / (D / 2)));
        }
    __syncthreads();
    // every thread of the CTA makes the same passes (the rows' maxima are exchanged)
    for (int i0 = 0; i0 < n_rows; i0 += kU * kRows) {
        int64_t at[kU], sat[kU];
        bool ok[kU];
        float sk[kU], sv[kU];
        uint2 ck[kU][2], cv[kU][2];                   // codes of both halves (gather)
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int64_t base = s_at[tl[u]];
            ok[u] = base >= 0;
            at[u] = base + (int64_t)(h[u] * size) * D + c;
            sat[u] = s_sat[tl[u]] + h[u] * size;
            if constexpr (!kAppend) {
                if (!ok[u]) continue;
                if constexpr (kCodes) {
                    const uint8_t* pk = static_cast<const uint8_t*>(P.pg.k) + at[u];
                    const uint8_t* pv = static_cast<const uint8_t*>(P.pg.v) + at[u];
                    ck[u][0] = ld_codes<N>(pk);
                    ck[u][1] = ld_codes<N>(pk + D / 2);
                    cv[u][0] = ld_codes<N>(pv);
                    cv[u][1] = ld_codes<N>(pv + D / 2);
                    sk[u] = ld_after(P.pg.k_scale + sat[u]);
                    sv[u] = ld_after(P.pg.v_scale + sat[u]);
                } else {
                    rk[u].load(static_cast<const T*>(P.pg.k) + at[u], D / 2);
                    rv[u].load(static_cast<const T*>(P.pg.v) + at[u], D / 2);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            float x[2 * N];
            auto row = [&](const Halves<T>& r, const uint2 (&codes)[2], float scale) {
                if constexpr (!kAppend && kCodes) {
                    from_codes<N>(codes[0], x, scale);
                    from_codes<N>(codes[1], x + N, scale);
                } else {
                    r.unpack(x);
                }
                if (!kAppend && !ok[u])               // a page that is none reads as zero
#pragma unroll
                    for (int e = 0; e < 2 * N; ++e) x[e] = 0.f;
            };
            auto put = [&](void* pages, float* scales, T* out) {
                if constexpr (kAppend && kCodes) {
                    const float2 s = row_scale(row_top<kLanes>(top_of<2 * N>(x)));
                    if (!live[u] || !ok[u]) return;
                    uint8_t* const p = static_cast<uint8_t*>(pages) + at[u];
                    store_codes<N>(p, x, s.y);
                    store_codes<N>(p + D / 2, x + N, s.y);
                    if (lane == 0) scales[sat[u]] = s.x;
                } else {
                    if (!live[u] || (kAppend && !ok[u])) return;
                    T* const p = kAppend ? static_cast<T*>(pages) + at[u] : out + dense[u];
                    st16(p, Vec16<T>::pack(x));
                    st16(p + D / 2, Vec16<T>::pack(x + N));
                }
            };
            row(rk[u], ck[u], sk[u]);
            if (P.turn) {
                float lo[N], hi[N];
                rotate<N>(x, x + N, s_cs + tl[u] * (D / 2) + c, lo, hi);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    x[e] = lo[e];
                    x[N + e] = hi[e];
                }
            }
            put(P.pg.k, P.pg.k_scale, dense_k);
            row(rv[u], cv[u], sv[u]);
            put(P.pg.v, P.pg.v_scale, dense_v);
        }
        if (i0 + kU * kRows < n_rows) rows_of(i0 + kU * kRows);
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
        P.per_hkv = 1.0f / (float)c.hkv;
        P.t0 = c.ptr[b0];
        P.t1 = c.ptr[b0 + nb];
        const int tokens = P.t1 - P.t0;
        if (tokens == 0) continue;
        // a few passes a CTA where there are rows enough for every SM, one token where there are not
        const int most = std::max(1, std::min(kMovePasses * rows_at_once(kAppend) * kRows / c.hkv, kMaxTokens));
        P.tokens_per_cta = std::max(1, std::min(most, tokens / (4 * device_sms())));
        P.rope = *c.rope;
        for (int i = 0; i <= nb; ++i) P.ptr[i] = c.ptr[b0 + i];
        for (int i = 0; i < nb; ++i) P.start[i] = c.start[b0 + i];
        const int ctas = (tokens + P.tokens_per_cta - 1) / P.tokens_per_cta;
        // (a few tokens: the host takes longer to launch it than the device to run it)
        const cudaError_t e = launch_overlapped(paged_move_kernel<T, D, kCodes, kAppend, kReq>, ctas, kMoveThreads, 0, s, P, P.tokens_per_cta > 1);
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

}  // namespace

cudaError_t launch_paged_append(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    return move_rows<true>(c, dtype, d, codes, s);
}
cudaError_t launch_paged_gather(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    return move_rows<false>(c, dtype, d, codes, s);
}

}  // namespace c2kv
