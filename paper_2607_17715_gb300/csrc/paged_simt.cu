// Paged attention of fp32 contexts (c2kv_paged_attend): CUDA cores and fp32 throughout, by the loop that
// the library's other fp32 attentions use (attention_core).  Here is what a row and a key are: packed row
// r = t * G + g is the request's query t, head h_kv * G + g; key j lies in its page, in fp32 or as E4M3
// codes that become fp32 on their way into shared memory.  The queries turn there too.
//
// FP32 multiply-adds bound long calls (140 tokens over 9495 rows, 16 / 4 heads of 128: 366 us, 30 TFLOP/s),
// the few key tiles of a CTA's chain short ones (3 requests of up to 61 tokens over 700 rows, heads of 64:
// 39 us).
#include <algorithm>

#include "attn_core.cuh"
#include "paged.cuh"
#include "rope.cuh"

#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int kSimtReq = 64;             // requests of a launch

// What a row sees (sees(row, key) of attention_core): up to its last key, or through its tree.
struct TreeRow {
    int start;               // the last key before the tree that it does not see
    const uint32_t* bits;    // [kTreeWords]
};

template <int D, bool kCodes, bool kTree>
struct PagedJob {
    const PagedAttn<kSimtReq>& P;
    const PagedReq& R;
    const int32_t* table;
    uint32_t* gap;                       // shared: some page was none, so its keys are hidden
    int hk, g_heads, row0, nrows, nkeys;
    int first, last;                     // last keys that the CTA's first and last rows see
    const uint32_t* bits;                // shared (trees): [query from that of row0 on][kTreeWords] ...
    const int* start;                    // ... and [query]
    float scale_log2;
    __device__ int64_t token(int r) const { return R.q0 + r / g_heads; }
    __device__ int head(int r) const { return hk * g_heads + r % g_heads; }
    __device__ const float* q_row(int r) const { return static_cast<const float*>(P.q) + token(r) * P.q_stride + (int64_t)head(r) * D; }
    __device__ float* out_row(int r) const { return static_cast<float*>(P.out) + (token(r) * P.hq + head(r)) * D; }
    __device__ float* lse_at(int r) const { return P.lse ? P.lse + (int64_t)head(r) * P.n_tokens + token(r) : nullptr; }
    __device__ int before() const { return R.n_keys - R.nq; }
    __device__ int lowest() const { return (kTree ? before() : first) - P.window; }  // the last key that a window hides from all (a tree's root has the least depth)
    __device__ bool needed(int, int k1) const { return !P.window || k1 > lowest() + 1; }
    __device__ bool whole(int k0, int k1) const {
        return k1 - 1 <= (kTree ? before() - 1 : first) && (!P.window || k0 > last - P.window) && *reinterpret_cast<volatile uint32_t*>(gap) == 0u;
    }
    __device__ auto row(int r) const {
        if constexpr (kTree) {
            const int i = (r < nrows ? r : nrows - 1) / g_heads - row0 / g_heads;
            return TreeRow{start[i], bits + i * kTreeWords};
        } else {
            return before() + r / g_heads;                         // its last key
        }
    }
    __device__ int page_of(int key) const {
        const int page = __ldg(table + (key >> P.pg.page_shift));
        return page >= 0 && page < P.pg.n_pages ? page : -1;
    }
    __device__ bool sees_nothing(int r) const { return of_no_weight<kTree>(P, R, r / g_heads) == 0.f; }
    __device__ bool sees(int end, int key) const { return key <= end && (!P.window || key > end - P.window) && in_page(key); }
    __device__ bool sees(TreeRow w, int key) const { return tree_sees(key, before(), w.start, w.bits) && in_page(key); }
    __device__ bool in_page(int key) const { return *reinterpret_cast<volatile uint32_t*>(gap) == 0u || page_of(key) >= 0; }
    // page of a key that some row may see; -1 for one that none does, and for a page that is none
    __device__ int page_at(int key) const {
        if (key >= nkeys || (P.window && key <= lowest())) return -1;
        const int page = page_of(key);
        if (page < 0) {
            atomicOr(P.err, 1);
            *gap = 1u;
        }
        return page;
    }
    __device__ void load_rows(bool keys, uint8_t* dst, int pitch, int rows, int k0) const {
        constexpr int kChunks = kCodes ? D / 16 : D / 4;           // 16-byte chunks a row
        const int size = 1 << P.pg.page_shift;
        if constexpr (!kCodes) {
            const float* const base = static_cast<const float*>(keys ? P.pg.k : P.pg.v);
            for (int i = threadIdx.x; i < rows * kChunks; i += kCoreThreads) {
                const int r = i / kChunks, c = i - r * kChunks, key = k0 + r, page = page_at(key);
                const float* p = base + (int64_t)max(page, 0) * P.pg.page_stride + ((int64_t)hk * size + (key & (size - 1))) * D + 4 * c;
                const uint32_t n = page >= 0 ? 16u : 0u;           // 0: zeros, nothing read
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst + (size_t)r * pitch + c * 16)), "l"(p), "r"(n)
                             : "memory");
            }
        } else {
            const uint8_t* const base = static_cast<const uint8_t*>(keys ? P.pg.k : P.pg.v);
            const float* const scales = keys ? P.pg.k_scale : P.pg.v_scale;
            constexpr int U = 4;                                   // loads in flight a thread
            for (int i0 = threadIdx.x; i0 < rows * kChunks; i0 += U * kCoreThreads) {
                uint4 w[U];
                float s[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * kCoreThreads, r = i / kChunks, c = i - r * kChunks, key = k0 + r;
                    const int page = i < rows * kChunks ? page_at(key) : -1;
                    const int64_t in_page = (int64_t)hk * size + (key & (size - 1));
                    w[u] = page >= 0 ? ld16(base + (int64_t)page * P.pg.page_stride + in_page * D + 16 * c) : make_uint4(0u, 0u, 0u, 0u);
                    s[u] = page >= 0 ? __ldg(scales + (int64_t)page * P.pg.scale_stride + in_page) : 0.f;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * kCoreThreads, r = i / kChunks, c = i - r * kChunks;
                    if (i >= rows * kChunks) break;
                    const uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
                    float4* o = reinterpret_cast<float4*>(dst + (size_t)r * pitch + c * 64);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t a, b;
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((uint16_t)x[e]));
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((uint16_t)(x[e] >> 16)));
                        const float2 f = __half22float2(*reinterpret_cast<__half2*>(&a)), g = __half22float2(*reinterpret_cast<__half2*>(&b));
                        o[e] = make_float4(f.x * s[u], f.y * s[u], g.x * s[u], g.y * s[u]);
                    }
                }
            }
        }
    }
    __device__ void turn_queries(uint8_t* q, int pitch, int rows) const {
        if (!P.turn) return;
        for (int i = threadIdx.x; i < rows * (D / 2); i += kCoreThreads) {
            const int r = i / (D / 2), c = i % (D / 2);
            if (row0 + r >= nrows) break;
            float* const x = reinterpret_cast<float*>(q + (size_t)r * pitch);
            float a, b;
            rotate1(x[c], x[c + D / 2], turn_cs(lane_turn(P.rope.turn, c), __ldg(P.turn + token(row0 + r))), a, b);
            x[c] = a;
            x[c + D / 2] = b;
        }
        __syncthreads();
    }
};

template <int D, bool kCodes, bool kTree>
struct CoreOwnRows<PagedJob<D, kCodes, kTree>> {
    static constexpr bool value = true;
};

// Item: a row tile of a request (over `ns` CTAs of a cluster), times KV heads along y.
template <int D, bool kCodes, int RT, bool kTree>
__global__ void __launch_bounds__(kCoreThreads, core_ctas(D, RT)) paged_simt_kernel(const __grid_constant__ PagedAttn<kSimtReq> P, int ns) {
    extern __shared__ __align__(16) uint8_t core_smem[];
    __shared__ uint32_t s_gap;
    __shared__ uint32_t s_bits[kTree ? Core<D, RT>::kRows * kTreeWords : 1];
    __shared__ int s_start[kTree ? Core<D, RT>::kRows : 1];
    if (threadIdx.x == 0) s_gap = 0u;
    __syncthreads();
    const int item = (int)(blockIdx.x / (unsigned)ns), rank = (int)(blockIdx.x % (unsigned)ns);
    int r = 0;
    while (r + 1 < P.batch && P.req[r + 1].item0 <= item) ++r;
    PagedJob<D, kCodes, kTree> j{P, P.req[r]};
    j.table = P.pg.table + (int64_t)j.R.row * P.pg.table_stride;
    j.gap = &s_gap;
    j.hk = blockIdx.y;
    j.g_heads = P.hq / P.hkv;
    j.row0 = (item - j.R.item0) * Core<D, RT>::kRows;
    j.nrows = j.R.nq * j.g_heads;
    const int rows = min(Core<D, RT>::kRows, j.nrows - j.row0), before = j.R.n_keys - j.R.nq;
    j.first = before + j.row0 / j.g_heads;
    j.last = before + (j.row0 + rows - 1) / j.g_heads;
    j.nkeys = max(0, j.last + 1);
    j.scale_log2 = P.scale_log2;
    if constexpr (kTree) {               // the queries' ways through the tree
        j.bits = s_bits;
        j.start = s_start;
        const int q0 = j.row0 / j.g_heads, n = (j.row0 + rows - 1) / j.g_heads - q0 + 1;
        if ((int)threadIdx.x < n) {
#pragma unroll
            for (int i = 0; i < kTreeWords; ++i) s_bits[threadIdx.x * kTreeWords + i] = 0u;
            s_start[threadIdx.x] = tree_bits(P.parent + j.R.q0, q0 + (int)threadIdx.x, before, P.window, P.err, s_bits + threadIdx.x * kTreeWords);
        }
        __syncthreads();
    }
    attention_core<float, D, RT>(j, j.row0, ns, rank, core_smem);
}

template <int D, bool kCodes, int RT, bool kTree>
CoreKernel<D, RT> ready() {
    static PerDevice<CoreKernel<D, RT>> kept;
    return kept.get([] { return CoreKernel<D, RT>(reinterpret_cast<const void*>(&paged_simt_kernel<D, kCodes, RT, kTree>), device_sms()); });
}

template <int D, bool kCodes, int RT, bool kTree>
cudaError_t launch_form(PagedAttn<kSimtReq>& P, CorePlan plan, cudaStream_t s) {
    constexpr int kRows = Core<D, RT>::kRows;
    int64_t items = 0;
    for (int i = 0; i < P.batch; ++i) {
        P.req[i].item0 = (int32_t)items;
        items += ((int64_t)P.req[i].nq * (P.hq / P.hkv) + kRows - 1) / kRows;
    }
    if (items * plan.ns > 0x7fffffffLL || P.hkv > 65535) return cudaErrorInvalidValue;
    void* args[2] = {&P, &plan.ns};
    return core_launch(reinterpret_cast<const void*>(&paged_simt_kernel<D, kCodes, RT, kTree>), dim3((unsigned)(items * plan.ns), P.hkv),
                       Core<D, RT>::kSmem, plan, false, args, s);
}

template <int D, bool kCodes, bool kTree>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    const CoreKernel<D, 4> large = ready<D, kCodes, 4, kTree>();
    const CoreKernel<D, 1> small = ready<D, kCodes, 1, kTree>();
    const CoreKernel<D, 0> four = ready<D, kCodes, 0, kTree>();
    if (large.err != cudaSuccess) return large.err;
    if (small.err != cudaSuccess || four.err != cudaSuccess) return small.err != cudaSuccess ? small.err : four.err;
    for (int b0 = 0; b0 < n; b0 += kSimtReq) {
        const int nb = std::min(n - b0, kSimtReq);
        PagedAttn<kSimtReq> P;
        fill_paged(P, c, D, req + b0, nb);
        // the cut is planned for requests as large as the largest, as many as make up all rows
        int64_t rows = 0, most = 1, keys = 1;
        for (int i = 0; i < nb; ++i) {
            const int64_t r = (int64_t)P.req[i].nq * (c.hq / c.hkv);
            rows += r;
            most = std::max(most, r);
            keys = std::max<int64_t>(keys, c.window ? std::min<int64_t>(P.req[i].n_keys, (int64_t)c.window + P.req[i].nq) : P.req[i].n_keys);
        }
        const CorePlan plan = core_plan(most, c.hkv * std::max<int64_t>(1, (rows + most / 2) / most), keys, D, false,
                                        [&](int form, int ns, bool alone) {
                                            return form == 4 ? large.slots[alone][ns] : form == 1 ? small.slots[alone][ns] : four.slots[alone][ns];
                                        });
        const cudaError_t e = plan.form == 4   ? launch_form<D, kCodes, 4, kTree>(P, plan, s)
                              : plan.form == 1 ? launch_form<D, kCodes, 1, kTree>(P, plan, s)
                                               : launch_form<D, kCodes, 0, kTree>(P, plan, s);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <bool kTree>
cudaError_t by_kind(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? launch<128, true, kTree>(c, req, n, s) : launch<128, false, kTree>(c, req, n, s);
    return codes ? launch<64, true, kTree>(c, req, n, s) : launch<64, false, kTree>(c, req, n, s);
}

}  // namespace

// This file is compiled twice: trees of tokens are paged_simt_tree.cu's.
#ifndef C2KV_TREES

cudaError_t launch_paged_simt(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return c.parent ? launch_paged_simt_tree(c, req, n, d, codes, s) : by_kind<false>(c, req, n, d, codes, s);
}

#else

cudaError_t launch_paged_simt_tree(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return by_kind<true>(c, req, n, d, codes, s);
}

#endif

}  // namespace c2kv
