// Paged attention of few query rows in fp32 contexts (c2kv_paged_attend): a generated token or two of each
// request, on the CUDA cores in fp32 throughout.
//
// The rows of a (request, KV head), four at a time, meet every key once.  Eight lanes take a key, D / 8
// channels each, and four keys are under way in a warp; every eight lanes keep a running maximum, sum and
// output of their own, so that nothing but a score's sum crosses lanes until the end.  Weights are relative
// to the maximum so far, never above 1: fp32 values may be as large as the type holds.  Two such groups of
// keys are worked on together, their chains being what takes the time.  A CTA's four warps share a stretch
// of keys in blocks of 32; they join in shared memory, the stretches in the CTA that ends last.
//
// Issue bounds it (a key takes 2 D / 8 multiply-adds a row and lane, and half as much around them), at half
// of its rate with the two warps a scheduler that registers leave.  Measured, 32 / 8 heads of 128 channels,
// E4M3 pages: one token over 30000 rows 49 us, 16 requests' over 9000 rows 191 (the bytes alone: 45), 27
// requests' over 1381 66.  With one group of keys at a time, rows one after the other, the 191 were 223.
#include "paged.cuh"
#include "per_device.cuh"
#include "ptx.cuh"
#include "rope.cuh"

#include <algorithm>
#include <cuda_fp16.h>
#include <optional>

namespace c2kv {
namespace {

constexpr int kLaneWarps = 4, kLaneThreads = 32 * kLaneWarps;
constexpr int kLaneBlk = 32;             // keys of a warp's block: one page lookup a lane
constexpr int kLaneReq = 64;             // requests of a launch
constexpr int kPair = 2;                 // groups of four keys worked on together
// CTAs an SM, by registers and the rings' bytes.
__host__ __device__ constexpr int lane_ctas(int d) { return d == 64 ? 3 : 2; }

struct LaneLaunch {
    PagedAttn<kLaneReq> a;
    float* part_o;                       // [item][row][D], of cut keys
    float* part_lse;                     // [item][row], log2
    uint32_t* tickets;                   // [unit], zero between launches
};

// What a lane takes of four keys, K and V: D / 8 channels of one of them.  Lane i's are i C .. of codes, and
// four of every 32 of fp32 values.  Copies go to a ring of the lane's own in shared memory, so only the lane
// itself waits for them.
template <int D, bool kCodes>
struct LaneRing {
    static constexpr int C = D / 8;
    static constexpr int kLine = kCodes && C == 8 ? 8 : 16;         // bytes of a copy
    static constexpr int kLines = C * (kCodes ? 1 : 4) / kLine;     // copies of a row
    static constexpr int kDepth = kCodes ? 8 : D == 64 ? 8 : 6;     // groups of four keys on their way
    static constexpr int kGroup = 2 * (kLines * kLine + (kCodes ? 4 : 0)) * 32;
    static constexpr int kBytes = kLaneWarps * kDepth * kGroup;
    __device__ static __forceinline__ int channel(int i, int e) { return kCodes ? i * C + e : (e >> 2) * 32 + i * 4 + (e & 3); }
    // line `k` of side v (0: K, 1: V), and the scale of it
    __device__ static __forceinline__ uint32_t line(int v, int k, int lane) { return ((v * kLines + k) * 32 + lane) * kLine; }
    __device__ static __forceinline__ uint32_t scale(int v, int lane) { return 2 * kLines * kLine * 32 + (v * 32 + lane) * 4; }
    template <int N>
    __device__ static __forceinline__ void copy(uint32_t to, const void* from, bool there) {      // zeros where not
        if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(N), "r"(there ? N : 0) : "memory");
    }
    __device__ static __forceinline__ void unpack(const uint8_t* group, int v, int lane, float (&x)[C]) {
        if constexpr (kCodes) {
            uint32_t w[C / 4];
            if constexpr (C == 16) {
                const uint4 y = *reinterpret_cast<const uint4*>(group + line(v, 0, lane));
                w[0] = y.x;
                w[1] = y.y;
                w[2] = y.z;
                w[3] = y.w;
            } else {
                const uint2 y = *reinterpret_cast<const uint2*>(group + line(v, 0, lane));
                w[0] = y.x;
                w[1] = y.y;
            }
#pragma unroll
            for (int k = 0; k < C / 4; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t y;
                    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"((uint16_t)(w[k] >> (16 * h))));
                    const float2 f = __half22float2(*reinterpret_cast<__half2*>(&y));
                    x[4 * k + 2 * h] = f.x;
                    x[4 * k + 2 * h + 1] = f.y;
                }
        } else {
#pragma unroll
            for (int k = 0; k < kLines; ++k) {
                const float4 y = *reinterpret_cast<const float4*>(group + line(v, k, lane));
                x[4 * k] = y.x;
                x[4 * k + 1] = y.y;
                x[4 * k + 2] = y.z;
                x[4 * k + 3] = y.w;
            }
        }
    }
};

template <int D, bool kCodes, int NR>
__global__ void __launch_bounds__(kLaneThreads, lane_ctas(D)) paged_lane_kernel(const __grid_constant__ LaneLaunch X) {
    using Ring = LaneRing<D, kCodes>;
    constexpr int C = Ring::C, kDepth = Ring::kDepth, kGroups = kLaneBlk / 4;
    extern __shared__ __align__(16) uint8_t ring_bytes[];
    const PagedAttn<kLaneReq>& P = X.a;
    __shared__ float s_q[NR][D];
    __shared__ __align__(16) float s_o[kLaneWarps][NR][D];
    __shared__ float s_m[kLaneWarps][NR], s_l[kLaneWarps][NR];
    __shared__ bool s_last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, sub = lane / 8, i8 = lane % 8;
    int r = 0;
    for (int hi = P.batch; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.req[mid].item0 <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    const PagedReq R = P.req[r];
    const int G = P.group, n_rows = R.nq * G, n_tiles = R.tiles;
    int at = blockIdx.x - R.item0;
    const int rt = at % n_tiles;
    at /= n_tiles;
    const int hk = at % P.hkv, split = at / P.hkv;
    const int row0 = rt * NR, live = min(NR, n_rows - row0);
    // the last key that each row sees, and the keys that any of them does
    int end[NR];
#pragma unroll
    for (int k = 0; k < NR; ++k) end[k] = R.n_keys - R.nq + (row0 + min(k, live - 1)) / G;
    const int k_hi = max(0, end[NR - 1] + 1), k_lo = P.window ? max(0, end[0] - P.window + 1) : 0;
    const int blk_lo = k_lo / kLaneBlk, blocks = max(0, (k_hi + kLaneBlk - 1) / kLaneBlk - blk_lo);
    const int b0 = blk_lo + (int)((int64_t)blocks * split / R.splits), b1 = blk_lo + (int)((int64_t)blocks * (split + 1) / R.splits);
    const int size = 1 << P.pg.page_shift;
    const int32_t* const table = P.pg.table + (int64_t)R.row * P.pg.table_stride;

    // block b's pages: lane i knows that of key i, -1 where no row sees it or it lies in none
    auto pages_of = [&](int b) {
        const int key = b * kLaneBlk + lane;
        int page = -1;
        if (b < b1 && key >= k_lo && key < k_hi) {
            page = ld_after(table + (key >> P.pg.page_shift));
            if (page < 0 || page >= P.pg.n_pages) {
                atomicOr(P.err, 1);
                page = -1;
            }
        }
        return page;
    };
    after_kernels_before();
    uint8_t* const ring = ring_bytes + warp * kDepth * Ring::kGroup;
    const int mine = b0 + warp < b1 ? (b1 - b0 - warp + kLaneWarps - 1) / kLaneWarps * kGroups : 0;   // the warp's groups of four keys
    int pages = pages_of(b0 + warp), pages_next = pages_of(b0 + warp + kLaneWarps);
    uint32_t there = 0;                                              // bit k: the lane's key k groups before the last one asked for
    auto key_of = [&](int n) { return (b0 + warp + n / kGroups * kLaneWarps) * kLaneBlk + n % kGroups * 4 + sub; };
    auto ask = [&](int n) {                                          // group n of the warp's
        if (n < mine) {
            if (n > 0 && n % kGroups == 0) {
                pages = pages_next;
                pages_next = pages_of(b0 + warp + (n / kGroups + 1) * kLaneWarps);
            }
            const int key = key_of(n), page = __shfl_sync(0xffffffffu, pages, n % kGroups * 4 + sub);
            const bool ok = page >= 0;
            there = there << 1 | (ok ? 1u : 0u);
            const int64_t in_page = (int64_t)hk * size + (key & (size - 1)), row = ok ? page : 0;
            const int64_t from = row * P.pg.page_stride + in_page * D;
            const uint32_t to = smem_u32(ring + n % kDepth * Ring::kGroup);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const uint8_t* const p = static_cast<const uint8_t*>(v ? P.pg.v : P.pg.k) + from * (kCodes ? 1 : 4);
#pragma unroll
                for (int k = 0; k < Ring::kLines; ++k) Ring::template copy<Ring::kLine>(to + Ring::line(v, k, lane), p + (k * 8 + i8) * Ring::kLine, ok);
                if constexpr (kCodes) Ring::template copy<4>(to + Ring::scale(v, lane), (v ? P.pg.v_scale : P.pg.k_scale) + row * P.pg.scale_stride + in_page, ok);
            }
        } else {
            there <<= 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int n = 0; n < kDepth - kPair; ++n) ask(n);

    // the queries, turned, while the first keys are on their way
    for (int k = threadIdx.x; k < NR * (D / 2); k += kLaneThreads) {
        const int row = min(k / (D / 2), live - 1), c = k % (D / 2);
        const int64_t tok = R.q0 + (row0 + row) / G;
        const float* q = static_cast<const float*>(P.q) + tok * P.q_stride + (int64_t)(hk * G + (row0 + row) % G) * D + c;
        float lo = q[0], hi = q[D / 2];
        if (P.turn) {
            const float x = lo, y = hi;
            rotate1(x, y, turn_cs(lane_turn(P.rope.turn, c), ld_after(P.turn + tok)), lo, hi);
        }
        s_q[k / (D / 2)][c] = lo;
        s_q[k / (D / 2)][c + D / 2] = hi;
    }
    __syncthreads();
    float q[NR][C], o[NR][C], m[NR], l[NR];
#pragma unroll
    for (int k = 0; k < NR; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.f;
#pragma unroll
        for (int e = 0; e < C; ++e) {
            q[k][e] = s_q[k][Ring::channel(i8, e)];
            o[k][e] = 0.f;
        }
    }

#pragma unroll 1
    for (int n = 0; n < mine; n += kPair) {
#pragma unroll
        for (int u = 0; u < kPair; ++u) ask(n + kDepth - kPair + u); // (into the groups before these)
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - kPair) : "memory");
        const uint8_t* group[kPair];
        float s[kPair][NR];
        uint32_t sees = 0;                                           // bit u NR + k: row k sees the lane's key of group u
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            group[u] = ring + (n + u) % kDepth * Ring::kGroup;
            const int key = key_of(n + u);
            float x[C];
            Ring::unpack(group[u], 0, lane, x);
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                s[u][k] = 0.f;
#pragma unroll
                for (int e = 0; e < C; ++e) s[u][k] = fmaf(q[k][e], x[e], s[u][k]);
                if ((there >> (kDepth - 1 - u) & 1u) && key <= end[k] && (!P.window || key > end[k] - P.window)) sees |= 1u << (u * NR + k);
            }
        }
#pragma unroll
        for (int h = 1; h < 8; h <<= 1)
#pragma unroll
            for (int u = 0; u < kPair; ++u)
#pragma unroll
                for (int k = 0; k < NR; ++k) s[u][k] += __shfl_xor_sync(0xffffffffu, s[u][k], h);
        bool moves = false;
        float top[NR];
#pragma unroll
        for (int k = 0; k < NR; ++k) top[k] = m[k];
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            float f = P.scale_log2;
            if constexpr (kCodes) f *= *reinterpret_cast<const float*>(group[u] + Ring::scale(0, lane));
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                s[u][k] = sees >> (u * NR + k) & 1u ? s[u][k] * f : -INFINITY;
                top[k] = fmaxf(top[k], s[u][k]);
                moves = moves || top[k] > m[k];
            }
        }
        if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                const float f = top[k] > m[k] ? exp2f(m[k] - top[k]) : 1.f;
                m[k] = top[k];
                l[k] *= f;
#pragma unroll
                for (int e = 0; e < C; ++e) o[k][e] *= f;
            }
        }
#pragma unroll
        for (int u = 0; u < kPair; ++u)
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                s[u][k] = s[u][k] == -INFINITY ? 0.f : exp2f(s[u][k] - m[k]);      // (one that is not seen: 0)
                l[k] += s[u][k];
            }
        const bool all = __all_sync(0xffffffffu, sees == (1u << (kPair * NR)) - 1);
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            float x[C];
            Ring::unpack(group[u], 1, lane, x);
            if constexpr (kCodes) {
                const float f = *reinterpret_cast<const float*>(group[u] + Ring::scale(1, lane));
#pragma unroll
                for (int k = 0; k < NR; ++k) s[u][k] *= f;
            }
            if (all) {
#pragma unroll
                for (int e = 0; e < C; ++e)
#pragma unroll
                    for (int k = 0; k < NR; ++k) o[k][e] = fmaf(s[u][k], x[e], o[k][e]);
            } else {
#pragma unroll
                for (int k = 0; k < NR; ++k)
                    if (sees >> (u * NR + k) & 1u)                   // a value that a row does not see takes no part
#pragma unroll
                        for (int e = 0; e < C; ++e) o[k][e] = fmaf(s[u][k], x[e], o[k][e]);
            }
        }
    }

    // four keys' lanes join, then the warps
#pragma unroll
    for (int k = 0; k < NR; ++k) {
        float top = m[k];
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float a = exp2f(m[k] - (top == -INFINITY ? 0.f : top));
        l[k] *= a;
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 8);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 16);
#pragma unroll
        for (int e = 0; e < C; ++e) {
            o[k][e] *= a;
            o[k][e] += __shfl_xor_sync(0xffffffffu, o[k][e], 8);
            o[k][e] += __shfl_xor_sync(0xffffffffu, o[k][e], 16);
        }
        if (sub == k % 4) {
#pragma unroll
            for (int e = 0; e < C; ++e) s_o[warp][k][Ring::channel(i8, e)] = o[k][e];
            if (i8 == 0) {
                s_m[warp][k] = top;
                s_l[warp][k] = l[k];
            }
        }
    }
    __syncthreads();
    const bool whole = R.splits == 1;
    auto put = [&](int row, int f, float4 x, float lse2) {
        const int64_t tok = R.q0 + (row0 + row) / G;
        const int h = hk * G + (row0 + row) % G;
        *reinterpret_cast<float4*>(static_cast<float*>(P.out) + (tok * P.hq + h) * D + 4 * f) = x;
        if (f == 0 && P.lse) P.lse[(int64_t)h * P.n_tokens + tok] = lse2 * 0.69314718055994531f;
    };
    // n results of a row joined: their log2 weights (or references) and sums, and four channels
    struct Joined {
        float top = -INFINITY, sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        __device__ void add(float m, float l, float4 y) {
            const float now = fmaxf(top, m), base = now == -INFINITY ? 0.f : now, a = exp2f(top - base), w = exp2f(m - base);
            top = now;
            sum = fmaf(l, w, sum * a);
            x = make_float4(fmaf(y.x, w, x.x * a), fmaf(y.y, w, x.y * a), fmaf(y.z, w, x.z * a), fmaf(y.w, w, x.w * a));
        }
        __device__ float4 value(float none) const {                  // (none: of no weight)
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            return sum == 0.f ? make_float4(none, none, none, none) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        }
        __device__ float lse2() const { return sum == 0.f ? -INFINITY : top + log2f(sum); }
    };
    auto none = [&](const Joined& j, int row) {
        return j.sum == 0.f ? of_no_weight(P, R.row, R.n_keys - R.nq + (row0 + row) / G) : 0.f;
    };
    for (int k = threadIdx.x; k < live * (D / 4); k += kLaneThreads) {
        const int row = k / (D / 4), f = k % (D / 4);
        Joined j;
#pragma unroll
        for (int w = 0; w < kLaneWarps; ++w) j.add(s_m[w][row], s_l[w][row], *reinterpret_cast<const float4*>(&s_o[w][row][4 * f]));
        if (whole) {
            put(row, f, j.value(none(j, row)), j.lse2());
        } else {
            *reinterpret_cast<float4*>(X.part_o + ((int64_t)blockIdx.x * NR + row) * D + 4 * f) = j.value(0.f);
            if (f == 0) X.part_lse[(int64_t)blockIdx.x * NR + row] = j.lse2();
        }
    }
    if (whole) return;
    // the stretch that ends last joins them all: every partial is visible before its ticket is taken
    const int unit = R.unit0 + hk * n_tiles + rt;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();                 // (cumulative: of what the CTA's threads wrote before the barrier)
        s_last = atomicAdd(X.tickets + unit, 1u) == (uint32_t)(R.splits - 1);
        if (s_last) X.tickets[unit] = 0;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    const int64_t step = (int64_t)P.hkv * n_tiles, item0 = R.item0 + (int64_t)hk * n_tiles + rt;
    for (int k = threadIdx.x; k < live * (D / 4); k += kLaneThreads) {
        const int row = k / (D / 4), f = k % (D / 4);
        Joined j;
#pragma unroll 8
        for (int s = 0; s < R.splits; ++s) {
            const int64_t item = item0 + s * step;
            const float e = __ldcg(X.part_lse + item * NR + row);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(X.part_o + (item * NR + row) * D + 4 * f));
            j.add(e, e == -INFINITY ? 0.f : 1.f, y);
        }
        put(row, f, j.value(none(j, row)), j.lse2());
    }
}

template <int D, bool kCodes, int NR>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_lane_kernel<D, kCodes, NR>;
    constexpr int kSmem = LaneRing<D, kCodes>::kBytes;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, kSmem);
    if (e != cudaSuccess) return e;
    for (int b0 = 0; b0 < n; b0 += kLaneReq) {
        const int nb = std::min(n - b0, kLaneReq);
        LaneLaunch X;
        fill_paged(X.a, c, D, req + b0, nb);
        // stretches: as many blocks each as make one wave of CTAs of all, but one a warp at least
        const int slots = device_sms() * lane_ctas(D), G = c.hq / c.hkv;
        auto blocks_of = [&](const PagedReq& q) {
            const int64_t keys = c.window ? std::min<int64_t>(q.n_keys, (int64_t)c.window + q.nq + kLaneBlk) : q.n_keys;
            return std::max<int64_t>(1, (keys + kLaneBlk - 1) / kLaneBlk);
        };
        auto units_of = [&](const PagedReq& q) { return (((int64_t)q.nq * G + NR - 1) / NR) * c.hkv; };
        int64_t total = 0;
        for (int i = 0; i < nb; ++i) total += blocks_of(X.a.req[i]) * units_of(X.a.req[i]);
        int64_t per = std::max<int64_t>(kLaneWarps, (total + slots - 1) / slots);
        auto splits_of = [&](const PagedReq& q) { return (blocks_of(q) + per - 1) / per; };
        for (int tries = 0; tries < 64; ++tries) {
            int64_t items = 0;
            bool any = false;
            for (int i = 0; i < nb; ++i) {
                items += units_of(X.a.req[i]) * splits_of(X.a.req[i]);
                any = any || splits_of(X.a.req[i]) > 1;
            }
            if (items <= slots || !any) break;
            per = std::max(per + 1, per * 33 / 32);
        }
        int64_t items = 0, units = 0;
        bool split = false;
        auto lay_out = [&](bool cut) {
            items = units = 0;
            split = false;
            for (int i = 0; i < nb; ++i) {
                PagedReq& q = X.a.req[i];
                q.splits = cut ? (int32_t)splits_of(q) : 1;
                split = split || q.splits > 1;
                q.item0 = (int32_t)items;
                q.unit0 = (int32_t)units;
                q.tiles = (int32_t)(units_of(q) / c.hkv);
                units += units_of(q);
                items += units_of(q) * q.splits;
            }
        };
        lay_out(true);
        X.part_o = X.part_lse = nullptr;
        X.tickets = nullptr;
        std::optional<Workspace> work;
        if (split) {
            const size_t o_bytes = (size_t)items * NR * D * 4;
            work.emplace(c.ctx, o_bytes + (size_t)items * NR * 4, (size_t)units);
            if (work->err == cudaErrorMemoryAllocation) {        // no room for partials: keys are not cut, slower
                (void)cudaGetLastError();
                lay_out(false);
            } else if (work->err != cudaSuccess) {
                return work->err;
            } else {
                X.part_o = static_cast<float*>(work->p);
                X.part_lse = reinterpret_cast<float*>(static_cast<char*>(work->p) + o_bytes);
                X.tickets = work->counters;
            }
        }
        e = launch_overlapped(kernel, (unsigned)items, kLaneThreads, kSmem, s, X);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool kCodes>
cudaError_t by_rows(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    bool one = true;
    for (int i = 0; i < n; ++i) one = one && (int64_t)req[i].nq * (c.hq / c.hkv) == 1;
    return one ? launch<D, kCodes, 1>(c, req, n, s) : launch<D, kCodes, 4>(c, req, n, s);
}

}  // namespace

cudaError_t launch_paged_lane(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? by_rows<128, true>(c, req, n, s) : by_rows<128, false>(c, req, n, s);
    return codes ? by_rows<64, true>(c, req, n, s) : by_rows<64, false>(c, req, n, s);
}

}  // namespace c2kv
