// The walk down a tree of drafted tokens (c2kv_verify_tree): at each node a token is drawn from the target's
// probabilities, by inverse CDF with a given random number, and where a child of the node holds it the walk goes
// on there.  So the tokens kept, and the one after them, are the target's own draws, whatever was drafted.
//
// Each level is a chain of its own: the row's sum, the search for the goal, the child.  A cluster of CTAs shares
// a request (as in verify.cu): each warp sums a stretch, the CTAs exchange their totals through distributed shared
// memory, the warp that holds the goal finds the token and tells every CTA, and each looks the child up in its own
// copy of the tree.
//
// The levels bound it, 2 to 3 us each (a cold row, two exchanges, the search): 16 trees of up to 32 nodes over 131072 tokens
// take 22.7 us, one of 16 nodes over 32000 tokens 12.4.  Holding a warp's stretch in registers for the search, and asking for
// a likely child's row ahead, were slower (26.9 and 15.6: 64 registers do not hold both).
#include "draw.cuh"

#include <algorithm>

namespace c2kv {
namespace {

template <int kReq>
__global__ void __launch_bounds__(kVerThreads, 2) verify_tree_kernel(const __grid_constant__ VerifyTreeParams<kReq> P) {
    __shared__ uint64_t s_warp[kVerWarps];
    __shared__ uint64_t s_total[2][kMaxCluster];          // of the cluster's CTAs, every other level
    __shared__ uint64_t s_token;
    __shared__ int32_t s_parent[kTreeMost], s_drafted[kTreeMost];
    __shared__ int s_child;
    const uint32_t rank = cluster_rank(), n_cta = cluster_size();
    const int r = blockIdx.x / n_cta, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int lo = P.ptr[r], n = P.ptr[r + 1] - lo, V = P.vocab;
    cluster_started();
    after_kernels_before();
    static_assert(kTreeMost <= kVerThreads, "a node a thread");
    if ((int)threadIdx.x < n) {
        const int p = ld_after(P.parent + lo + threadIdx.x);
        s_parent[threadIdx.x] = p;
        s_drafted[threadIdx.x] = ld_after(P.tokens + lo + threadIdx.x);
        if (rank == 0 && (p < -1 || p >= (int)threadIdx.x)) atomicOr(P.err, 1);
        if (rank == 0) P.path[lo + threadIdx.x] = threadIdx.x == 0 ? 0 : -1;
    }
    __syncthreads();                       // (the path is written again below)
    cluster_started_wait();
    // warps of the cluster take stretches of whole 32-element lines, in order
    const int warps = kVerWarps * (int)n_cta;
    const int per = ((V + warps - 1) / warps + 31) / 32 * 32;
    const int64_t first = (int64_t)((int)rank * kVerWarps + warp) * per;
    const int a = (int)min((int64_t)V, first), b = (int)min((int64_t)V, first + per);
    int node = 0, accepted = 0, token = -1;
    for (int level = 0; level < n; ++level) {
        const Row w{P.p + (int64_t)(lo + node) * P.p_stride, nullptr, -1};
        const float u = ld_after(P.u + lo + node);
        const uint64_t mine = stretch_sum(w, a, b, lane);
        if (lane == 0) s_warp[warp] = mine;
        if (threadIdx.x == 0) s_child = n;
        __syncthreads();
        if (warp == 0) {
            const uint64_t t = warp_sum(lane < kVerWarps ? s_warp[lane] : 0);
            if (lane < n_cta) st_peer(&s_total[level & 1][rank], lane, t);
            __syncwarp();
        }
        cluster_sync();
        uint64_t before = 0, total = 0;
        for (uint32_t c = 0; c < n_cta; ++c) {
            const uint64_t t = s_total[level & 1][c];
            total += t;
            if (c < rank) before += t;
        }
        token = -1;
        if (total == 0) break;             // (the same in every CTA)
        const uint64_t goal = goal_of(total, u);
        for (int i = 0; i < warp; ++i) before += s_warp[i];
        if (goal >= before && goal < before + mine) {
            const int x = find(w, a, b, lane, before, goal);
            if (lane < n_cta) st_peer(&s_token, lane, (uint64_t)x);
        }
        cluster_sync();                    // (nor is s_warp or s_token read below the next one)
        token = (int)s_token;
        // the first child that holds it (a parent is before its child: another is never reached)
        if ((int)threadIdx.x < n && (int)threadIdx.x > node && s_parent[threadIdx.x] == node && s_drafted[threadIdx.x] == token)
            atomicMin(&s_child, (int)threadIdx.x);
        __syncthreads();
        const int child = s_child;
        __syncthreads();
        if (child == n) break;
        node = child;
        ++accepted;
        if (rank == 0 && threadIdx.x == 0) P.path[lo + accepted] = child;
    }
    if (rank == 0 && threadIdx.x == 0) {
        P.n_accepted[P.b0 + r] = accepted;
        P.next_token[P.b0 + r] = token;
    }
}

template <int kReq>
cudaError_t launch(const VerifyTreeCall& c, cudaStream_t s) {
    int size = kMaxCluster;
    while (size > 1 && (int64_t)size * c.batch > 2 * (int64_t)device_sms()) size /= 2;
    for (int b0 = 0; b0 < c.batch; b0 += kReq) {
        const int nb = std::min(c.batch - b0, kReq);
        VerifyTreeParams<kReq> P;
        P.tokens = c.tokens;
        P.parent = c.parent;
        P.p = c.p;
        P.u = c.u;
        P.n_accepted = c.n_accepted;
        P.path = c.path;
        P.next_token = c.next_token;
        P.err = c.err;
        P.p_stride = c.p_stride;
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
        const cudaError_t e = cudaLaunchKernelEx(&cfg, verify_tree_kernel<kReq>, P);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_verify_tree(const VerifyTreeCall& c, cudaStream_t s) {
    return c.batch <= kPagedFew ? launch<kPagedFew>(c, s) : launch<kPagedMany>(c, s);
}

}  // namespace c2kv
