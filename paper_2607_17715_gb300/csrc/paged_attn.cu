// Attention of each request's new tokens over its paged cache (c2kv_paged_attend).
#include "paged.cuh"
#include "paged_row.cuh"

#include <algorithm>
#include <vector>

namespace c2kv {
namespace {

constexpr int kRowWarps = 4;
constexpr int kMmaRows = 64;             // query rows of a KV head up to which mma.sync takes a request

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
    row_attend<T, D, kCodes>(P, q, R.row, hk, lo + warp, hi, kRowWarps, lane, m, l, o);
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

template <typename T, int D, bool kCodes, int kReq>
cudaError_t launch_rows(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    for (int b0 = 0; b0 < n; b0 += kReq) {
        const int nb = std::min(n - b0, kReq);
        PagedAttn<kReq> P;
        fill_paged(P, c, D, req + b0, nb);
        const int tokens = req[b0 + nb - 1].q0 + req[b0 + nb - 1].nq - req[b0].q0;
        paged_row_kernel<T, D, kCodes, kReq><<<tokens * c.hq, kRowWarps * 32, 0, s>>>(P);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, int D>
cudaError_t rows_of(const PagedAttnCall& c, const PagedReq* req, int n, bool codes, cudaStream_t s) {
    const bool few = n <= kPagedFew;
    if (codes) return few ? launch_rows<T, D, true, kPagedFew>(c, req, n, s) : launch_rows<T, D, true, kPagedMany>(c, req, n, s);
    return few ? launch_rows<T, D, false, kPagedFew>(c, req, n, s) : launch_rows<T, D, false, kPagedMany>(c, req, n, s);
}

// Requests of many rows on tcgen05.  Their 8-bit pages are expanded to 16 bits first, in scratch that the
// stream hands back; requests go in groups so that the scratch stays small beside the cache.
constexpr int64_t kExpandBytes = (int64_t)512 << 20;

cudaError_t launch_many(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (!codes) return launch_paged_tc(c, req, n, d, s);
    const int shift = c.pg.page_shift;
    const int64_t page_bytes = ((int64_t)c.hkv << shift) * d * 2;
    for (int b0 = 0; b0 < n;) {
        std::vector<PagedReq> part;
        std::vector<int32_t> page0, pages, first;
        int64_t total = 0, width = 1;
        for (; b0 < n; ++b0) {
            const PagedReq& q = req[b0];
            const int64_t seen = c.window ? std::max<int64_t>(0, (int64_t)q.n_keys - q.nq + 1 - c.window) : 0;   // the first row that a query sees
            const int32_t lo = (int32_t)(seen >> shift), hi = (int32_t)(((int64_t)q.n_keys + (1 << shift) - 1) >> shift);
            if (!part.empty() && (total + hi - lo) * page_bytes * 2 > kExpandBytes) break;
            page0.push_back(lo);
            pages.push_back(std::max(0, hi - lo));
            first.push_back((int32_t)total);
            total += pages.back();
            width = std::max<int64_t>(width, hi);
            part.push_back(q);
        }
        const int m = (int)part.size();
        const size_t half = (size_t)std::max<int64_t>(1, total) * page_bytes;
        void* p = nullptr;
        cudaError_t e = context_alloc(c.ctx, &p, 2 * half + (size_t)m * width * 4);
        if (e == cudaErrorMemoryAllocation) {           // no room: code by code, slower
            (void)cudaGetLastError();
            e = launch_paged_mma(c, part.data(), m, d, true, s);
            if (e != cudaSuccess) return e;
            continue;
        }
        if (e != cudaSuccess) return e;
        PagedExpandCall x{};
        x.from = c.pg;
        x.to = PageView{p, static_cast<char*>(p) + half, nullptr, nullptr,
                        reinterpret_cast<const int32_t*>(static_cast<char*>(p) + 2 * half), page_bytes / 2, 0, width,
                        (int32_t)std::max<int64_t>(1, total), shift};
        x.err = c.err;
        x.hkv = c.hkv;
        x.n = m;
        x.req = part.data();
        x.page0 = page0.data();
        x.pages = pages.data();
        x.first = first.data();
        e = launch_paged_expand(x, d, s);
        PagedAttnCall a = c;
        a.pg = x.to;
        for (int i = 0; i < m; ++i) part[i].row = i;
        if (e == cudaSuccess) e = launch_paged_tc(a, part.data(), m, d, s);
        context_free(c.ctx, p);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_paged_attn(const PagedAttnCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    std::vector<PagedReq> req;
    req.reserve(c.batch);
    for (int r = 0; r < c.batch; ++r)
        if (c.ptr[r + 1] > c.ptr[r]) req.push_back(PagedReq{c.ptr[r], c.ptr[r + 1] - c.ptr[r], c.n_keys[r], r, 0, 1, 0, 0, 0});
    const int n = (int)req.size();
    if (dtype == kDtypeF32)
        return d == 128 ? rows_of<float, 128>(c, req.data(), n, codes, s) : rows_of<float, 64>(c, req.data(), n, codes, s);
    // requests of many rows on tcgen05, those of few on mma.sync
    std::vector<PagedReq> few, many;
    for (const PagedReq& q : req) ((int64_t)q.nq * (c.hq / c.hkv) > kMmaRows ? many : few).push_back(q);
    cudaError_t e = cudaSuccess;
    if (!many.empty()) e = launch_many(c, many.data(), (int)many.size(), d, codes, s);
    if (e == cudaSuccess && !few.empty()) e = launch_paged_mma(c, few.data(), (int)few.size(), d, codes, s);
    return e;
}

}  // namespace c2kv
