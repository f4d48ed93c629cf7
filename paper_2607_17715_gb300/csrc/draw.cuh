// A token drawn from a row of probabilities by a cluster of CTAs (verify.cu, verify_tree.cu): weights that are
// whole multiples of 2^-44, each warp's stretch of the row summed, and the stretch that holds the goal searched.
#pragma once

#include "paged.cuh"
#include "per_device.cuh"

namespace c2kv {
namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A weight in [0, 1] as a multiple of 2^-44, cut off, in two parts of 22 bits; NaN counts as 0 (fmaxf
// gives its other operand).  Adding 2^23 rounded down leaves a whole number's bits in the fraction, and
// every difference here is exact: five FP32 operations, where the conversion to 64 bits is slow.
struct Parts {
    uint32_t hi, lo;
};
__device__ __forceinline__ Parts parts(float w) {
    const float x = fminf(fmaxf(w, 0.f), 1.f) * 0x1p22f;
    const float a = __fadd_rd(x, 0x1p23f);
    const float b = __fadd_rd((x - (a - 0x1p23f)) * 0x1p22f, 0x1p23f);
    return {__float_as_uint(a) - 0x4b000000u, __float_as_uint(b) - 0x4b000000u};
}
__device__ __forceinline__ uint64_t whole(float w) {
    const Parts p = parts(w);
    return ((uint64_t)p.hi << 22) + p.lo;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// Every CTA of the cluster has started: only then does its shared memory take stores.  Said when the kernel
// starts, and waited for ahead of the first store.
__device__ __forceinline__ void cluster_started() {
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_started_wait() {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// 8 bytes to this CTA's shared address `local`, in the cluster's CTA `rank`.
__device__ __forceinline__ void st_peer(const uint64_t* local, uint32_t rank, uint64_t v) {
    const uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(local));
    uint32_t peer;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(a), "r"(rank));
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer), "l"(v) : "memory");
}

// The row that a token is drawn from: what p leaves over q (q may be null), or p without the refused
// token `drop`.
struct Row {
    const float* p;
    const float* q;
    int drop;
};

constexpr int kChunk = 512;              // elements a warp has on their way at once, 16 a lane

// Weights of elements i + 128 u + 4 lane + e (v[4 u + e]) below b, 0 past it: by four 16-byte loads of
// each row where both allow it (128 KB in flight an SM; at half of it the rows came at 2.4 TB/s).  Rows
// that do not (an odd vocabulary) are read in the same order for a search; for a sum, whose order is
// free, lanes take neighbours.
template <bool kInOrder>
__device__ __forceinline__ void load_chunk(const Row& w, int i, int b, int lane, float (&v)[16]) {
    // (i is a multiple of 32 elements, so the rows' addresses decide)
    const bool wide = ((reinterpret_cast<uintptr_t>(w.p) | reinterpret_cast<uintptr_t>(w.q)) & 15u) == 0 && i + kChunk <= b;
    if (wide) {
        float4 x[4], y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = ld_after(reinterpret_cast<const float4*>(w.p + i + 128 * u) + lane);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            y[u] = w.q ? ld_after(reinterpret_cast<const float4*>(w.q + i + 128 * u) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            v[4 * u] = x[u].x - y[u].x;
            v[4 * u + 1] = x[u].y - y[u].y;
            v[4 * u + 2] = x[u].z - y[u].z;
            v[4 * u + 3] = x[u].w - y[u].w;
        }
    } else {
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int e = kInOrder ? i + 128 * (u / 4) + 4 * lane + u % 4 : i + 32 * u + lane;
            v[u] = e < b && e != w.drop ? ld_after(w.p + e) - (w.q ? ld_after(w.q + e) : 0.f) : 0.f;
        }
        return;
    }
    const int drop = w.drop - i - 4 * lane;              // from the lane's first element
#pragma unroll
    for (int u = 0; u < 16; ++u)
        if (drop == 128 * (u / 4) + u % 4) v[u] = 0.f;
}

// The sum of a warp's stretch [a, b).
__device__ __forceinline__ uint64_t stretch_sum(const Row& w, int a, int b, int lane) {
    uint64_t sum = 0;
    for (int i = a; i < b; i += kChunk) {
        float v[16];
        load_chunk<false>(w, i, b, lane, v);
        uint32_t hi = 0, lo = 0;         // (parts of at most 2^22, 16 of them)
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const Parts x = parts(v[u]);
            hi += x.hi;
            lo += x.lo;
        }
        sum += ((uint64_t)hi << 22) + lo;
    }
    return warp_sum(sum);
}

// The first element of [a, b) whose running sum, from `before` on, passes goal (there is one).
__device__ __forceinline__ int find(const Row& w, int a, int b, int lane, uint64_t before, uint64_t goal) {
    for (int i = a; i < b; i += kChunk) {
        float v[16];
        load_chunk<true>(w, i, b, lane, v);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            uint64_t x[4], upto = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) upto += x[e] = whole(v[4 * u + e]);
            const uint64_t mine = upto;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, before + upto > goal);
            if (past) {
                const int from = __ffs(past) - 1;
                uint64_t run = before + upto - mine;
                int e = 0;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    run += x[k];
                    e += run <= goal;
                }
                return i + 128 * u + 4 * from + __shfl_sync(0xffffffffu, e, from);
            }
            before += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
    return b - 1;
}

// What the running sum of weights has to pass: floor(total k / 2^24), u cut to a whole multiple k of 2^-24.
__device__ __forceinline__ uint64_t goal_of(uint64_t total, float u) {
    const uint64_t k = min((uint64_t)__float2ull_rz(fmaxf(u * 0x1p24f, 0.f)), (uint64_t)0xffffff);
    return (total >> 24) * k + (((total & 0xffffff) * k) >> 24);
}

}  // namespace
}  // namespace c2kv
