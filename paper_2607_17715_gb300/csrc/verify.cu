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
#include "draw.cuh"

#include <algorithm>

namespace c2kv {
namespace {

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
    const uint64_t goal = goal_of(total, ld_after(P.u_next + P.b0 + r));
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
