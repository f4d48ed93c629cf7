// Verification of drafted tokens (c2kv_verify_drafts): how many of a request's drafts the target's
// probabilities accept, and the token that follows them, from given random numbers.
//
// Draft i (token x) is accepted while u_i q_i(x) < p_i(x).  At the first refusal the next token comes
// from max(p - q, 0), after the last draft from p, by inverse CDF: weights are whole multiples of
// 2^-44, so their sums are the same in any order and the drawn token does not depend on how the
// vocabulary is split.
//
// Two rows of the vocabulary are read once a request, which bounds the call at HBM's rate for a batch
// and at the chain draft -> probabilities -> sum -> search for one request.  A cluster of CTAs shares a
// request: each warp sums one contiguous stretch, the CTAs exchange their totals through distributed
// shared memory, and the warp whose stretch holds the goal reads that stretch again (from L2).  Clusters
// are as large as keeps them all on the GPU at once: 64 requests in clusters of 8 took two rounds.
//
// Measured: 64 requests over 131072 tokens, 67 MB in 15 us (4.5 TB/s); one over 32000, 7.5 us, nearly all of it
// the chain, and the host's checks and launch.
#include "paged.cuh"
#include "per_device.cuh"

#include <algorithm>

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

template <int kReq>
__global__ void __launch_bounds__(kVerThreads, 2) verify_kernel(const __grid_constant__ VerifyParams<kReq> P) {
    __shared__ uint64_t s_warp[kVerWarps];
    __shared__ uint64_t s_total[2][kMaxCluster];          // of the cluster's CTAs, a pass
    __shared__ int s_accepted;
    const uint32_t rank = cluster_rank(), n_cta = cluster_size();
    const int r = blockIdx.x / n_cta, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int lo = P.ptr[r], n = P.ptr[r + 1] - lo, V = P.vocab;
    const int64_t p_row = (int64_t)lo + P.b0 + r;         // the request's first row of p
    cluster_started();
    after_kernels_before();
    if (warp == 0) {
        int a = 0;
        for (; a < n; a += 32) {
            bool yes = true;
            if (a + lane < n) {
                const int x = ld_after(P.tokens + lo + a + lane);
                yes = x >= 0 && x < V;
                if (!yes) {
                    if (rank == 0) atomicOr(P.err, 1);
                } else {
                    const float px = ld_after(P.p + (p_row + a + lane) * P.p_stride + x);
                    const float qx = P.q ? ld_after(P.q + (int64_t)(lo + a + lane) * P.q_stride + x) : 1.f;
                    yes = __fmul_rn(ld_after(P.u_accept + lo + a + lane), qx) < px;
                }
            }
            const uint32_t no = __ballot_sync(0xffffffffu, !yes);
            if (no) {
                a += __ffs(no) - 1;
                break;
            }
        }
        if (lane == 0) s_accepted = min(a, n);
    }
    __syncthreads();
    const int acc = s_accepted;
    Row w{P.p + (p_row + acc) * P.p_stride, nullptr, -1};
    if (acc < n) {
        if (P.q) w.q = P.q + (int64_t)(lo + acc) * P.q_stride;
        else w.drop = ld_after(P.tokens + lo + acc);
    }
    // warps of the cluster take stretches of whole 32-element lines, in order
    const int warps = kVerWarps * (int)n_cta;
    const int per = ((V + warps - 1) / warps + 31) / 32 * 32;
    const int64_t first = (int64_t)((int)rank * kVerWarps + warp) * per;
    const int a = (int)min((int64_t)V, first), b = (int)min((int64_t)V, first + per);
    uint64_t before = 0, total = 0;
    for (int pass = 0; pass < 2; ++pass) {
        const uint64_t mine = stretch_sum(w, a, b, lane);
        if (pass) __syncthreads();         // (s_warp is summed above by others than its warps)
        if (lane == 0) s_warp[warp] = mine;
        __syncthreads();
        if (pass == 0) cluster_started_wait();
        if (warp == 0) {
            const uint64_t t = warp_sum(lane < kVerWarps ? s_warp[lane] : 0);
            if (lane < n_cta) st_peer(&s_total[pass][rank], lane, t);
            __syncwarp();
        }
        cluster_sync();                    // (also of the warps' sums)
        before = total = 0;
        for (uint32_t c = 0; c < n_cta; ++c) {
            const uint64_t t = s_total[pass][c];
            total += t;
            if (c < rank) before += t;
        }
        if (total != 0 || pass == 1) break;
        // nothing is left of p over q (a refusal that rounding made): p itself
        w.q = nullptr;
        w.drop = -1;
    }
    if (rank == 0 && threadIdx.x == 0) {
        P.n_accepted[P.b0 + r] = acc;
        if (total == 0) P.next_token[P.b0 + r] = -1;
    }
    if (total == 0) return;
    const float uf = ld_after(P.u_next + P.b0 + r) * 0x1p24f;
    const uint64_t u = min((uint64_t)__float2ull_rz(fmaxf(uf, 0.f)), (uint64_t)0xffffff);
    const uint64_t goal = (total >> 24) * u + (((total & 0xffffff) * u) >> 24);
    for (int i = 0; i < warp; ++i) before += s_warp[i];
    if (goal < before || goal >= before + s_warp[warp]) return;
    const int token = find(w, a, b, lane, before, goal);
    if (lane == 0) P.next_token[P.b0 + r] = token;
}

template <int kReq>
cudaError_t launch(const VerifyCall& c, cudaStream_t s) {
    int size = kMaxCluster;
    while (size > 1 && (int64_t)size * c.batch > 2 * (int64_t)device_sms()) size /= 2;
    for (int b0 = 0; b0 < c.batch; b0 += kReq) {
        const int nb = std::min(c.batch - b0, kReq);
        VerifyParams<kReq> P;
        P.tokens = c.tokens;
        P.p = c.p;
        P.q = c.q;
        P.u_accept = c.u_accept;
        P.u_next = c.u_next;
        P.n_accepted = c.n_accepted;
        P.next_token = c.next_token;
        P.err = c.err;
        P.p_stride = c.p_stride;
        P.q_stride = c.q_stride;
        P.vocab = c.vocab;
        P.b0 = b0;
        for (int i = 0; i <= nb; ++i) P.ptr[i] = c.ptr[b0 + i];
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute at[2] = {};
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {(unsigned)size, 1, 1};
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(nb * size);
        cfg.blockDim = dim3(kVerThreads);
        cfg.stream = s;
        cfg.attrs = at;
        cfg.numAttrs = 2;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, verify_kernel<kReq>, P);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_verify(const VerifyCall& c, cudaStream_t s) {
    return c.batch <= kPagedFew ? launch<kPagedFew>(c, s) : launch<kPagedMany>(c, s);
}

}  // namespace c2kv
