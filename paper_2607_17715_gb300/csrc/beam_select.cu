// The best continuations of beams over the vocabulary (c2kv_beam_select).
//
// A candidate is a place w V + v of a request with the score s_w + (x[w][v] - norm_w), each operation rounded to
// fp32; the `best` of largest score are kept, of equal ones those of the lowest places.  So the choice does not
// depend on how the vocabulary is cut.
//
// Every value is read once, which bounds a batch.  A CTA takes a stretch of one beam, 4096 values at a time in
// registers, and keeps the best so far in shared memory: of later values only those above the last of them matter,
// hardly any.  Of the first 4096 a bound is found cheaply: of the lanes' largest values, every warp's r-th largest,
// the least of them over the warps (8 r >= best values are no smaller).  What passes is ranked by counting.  The CTA
// that ends last joins those of its request the same way.
#include "paged.cuh"
#include "per_device.cuh"

#include <algorithm>
#include <optional>

namespace c2kv {
namespace {

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kSelEach = 16;                              // values a thread
constexpr int kSelChunk = kSelThreads * kSelEach;
constexpr int kSelList = 1024;                            // candidates that are ranked at once
static_assert(kSelList >= 2 * kSelThreads + kBeamsMost, "joining takes two a thread");

// A score as a whole number of the same order, 0 for what is no candidate (-inf and NaN); -0 is 0.
__device__ __forceinline__ uint32_t key_of(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);
    return s > -INFINITY ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float score_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Whether (key a, place i) comes before (key b, place j).
__device__ __forceinline__ bool before(uint32_t a, uint32_t i, uint32_t b, uint32_t j) { return a > b || (a == b && i < j); }

// The best so far, in order, and what is to be ranked with them.
struct Best {
    uint2 list[kSelList];                                 // (key, place): [0, kept) the best, [kept, n) new ones
    uint2 next[kBeamsMost];
    int n;
    uint32_t bound;
    uint32_t sum;
};

// Ranks list[0, n) and keeps the `best` first of it; every thread of the CTA.  Returns how many are kept.
__device__ __forceinline__ int rank_list(Best& s, int best) {
    __syncthreads();
    const int n = s.n;
    for (int i = threadIdx.x; i < n; i += kSelThreads) {
        const uint2 x = s.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) {
            const uint2 y = s.list[j];
            rank += before(y.x, y.y, x.x, x.y);
        }
        if (rank < best) s.next[rank] = x;
    }
    __syncthreads();
    const int kept = min(n, best);
    if ((int)threadIdx.x < kept) s.list[threadIdx.x] = s.next[threadIdx.x];
    if (threadIdx.x == 0) s.n = kept;
    __syncthreads();
    return kept;
}

// The thread's values that pass, to the end of the list: those of `take` (bits).
template <class Entry>
__device__ __forceinline__ void append(Best& s, uint32_t take, int lane, const Entry& entry) {
    if (!__any_sync(0xffffffffu, take != 0u)) return;
    const int mine = __popc(take);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    int at = 0;
    if (lane == 31) at = atomicAdd(&s.n, upto);
    at = __shfl_sync(0xffffffffu, at, 31) + upto - mine;
    for (; take; take &= take - 1, ++at)
        if (at < kSelList) s.list[at] = entry(__ffs(take) - 1);
}

template <bool kBf16>
struct Values;
template <>
struct Values<false> {
    // place of value u of the thread's in a chunk
    __device__ static __forceinline__ int place(int u) { return (u >> 2) * (4 * kSelThreads) + threadIdx.x * 4 + (u & 3); }
    __device__ static __forceinline__ float one(const void* x, int64_t i) { return ld_after(static_cast<const float*>(x) + i); }
    __device__ static __forceinline__ void whole(const void* x, int64_t i, float (&v)[kSelEach]) {
        float4 y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = ld_after(reinterpret_cast<const float4*>(static_cast<const float*>(x) + i + place(4 * k)));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[4 * k] = y[k].x;
            v[4 * k + 1] = y[k].y;
            v[4 * k + 2] = y[k].z;
            v[4 * k + 3] = y[k].w;
        }
    }
};
template <>
struct Values<true> {
    __device__ static __forceinline__ int place(int u) { return (u >> 3) * (8 * kSelThreads) + threadIdx.x * 8 + (u & 7); }
    __device__ static __forceinline__ float one(const void* x, int64_t i) {
        return __uint_as_float((uint32_t)ld_after(static_cast<const uint16_t*>(x) + i) << 16);
    }
    __device__ static __forceinline__ void whole(const void* x, int64_t i, float (&v)[kSelEach]) {
        uint4 y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) y[k] = ld_after(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + i + place(8 * k)));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t w[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[8 * k + 2 * e] = __uint_as_float(w[e] << 16);
                v[8 * k + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
            }
        }
    }
};

template <bool kBf16>
__global__ void __launch_bounds__(kSelThreads) beam_select_kernel(const __grid_constant__ BeamParams P) {
    using X = Values<kBf16>;
    __shared__ Best s;
    __shared__ bool s_last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, K = P.best, V = P.vocab;
    const int r = blockIdx.x / P.parts, part = blockIdx.x - r * P.parts, of_beam = P.parts / P.width;
    const int w = part / of_beam, a = (part - w * of_beam) * P.per, b = min(V, a + P.per);
    const int64_t row = (int64_t)r * P.width + w;
    if (threadIdx.x == 0) s.n = 0;
    after_kernels_before();
    const float score = ld_after(P.score + row), norm = P.norm ? ld_after(P.norm + row) : 0.f;
    const bool done = P.done && ld_after(P.done + row) != 0;
    __syncthreads();
    if (done) {                                           // goes on as it is
        if (threadIdx.x == 0 && a == 0 && key_of(score)) {
            s.list[0] = make_uint2(key_of(score), (uint32_t)(w * V + P.end_token));
            s.n = 1;
        }
        __syncthreads();
    } else if (score > -INFINITY) {
        const int64_t base = row * P.x_stride;
        const bool wide = ((reinterpret_cast<uintptr_t>(P.x) + (uintptr_t)(base + a) * (kBf16 ? 2 : 4)) & 15u) == 0;
        uint32_t last = 0u;                               // the last of the best so far: later values have to be above it
        for (int c = a; c < b; c += kSelChunk) {
            uint32_t key[kSelEach], top = 0u;
            float v[kSelEach];
            if (wide && c + kSelChunk <= b) {
                X::whole(P.x, base + c, v);
            } else {
#pragma unroll
                for (int u = 0; u < kSelEach; ++u) v[u] = c + X::place(u) < b ? X::one(P.x, base + c + X::place(u)) : -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < kSelEach; ++u) {
                key[u] = key_of(__fadd_rn(score, P.norm ? __fsub_rn(v[u], norm) : v[u]));
                top = max(top, key[u]);
            }
            if (threadIdx.x == 0) {
                s.bound = 0xffffffffu;
                s.sum = 0u;
            }
            if (!__syncthreads_or(top > last)) continue;
            // a bound: `best` values at least are no smaller
            uint32_t bound = 0u, rest = top;
            for (int i = (K + kSelWarps - 1) / kSelWarps; i > 0; --i) {
                bound = __reduce_max_sync(0xffffffffu, rest);
                const uint32_t at = __ballot_sync(0xffffffffu, rest == bound);
                if (lane == __ffs(at) - 1) rest = 0u;
            }
            if (lane == 0) atomicMin(&s.bound, bound);
            __syncthreads();
            // what passes, by key and then by place: 32 and 12 bits, no two alike
            uint64_t least = (uint64_t)max(s.bound, last + 1u) << 12;
            auto passes = [&](int u) { return ((uint64_t)key[u] << 12 | (uint32_t)(kSelChunk - 1 - X::place(u))) >= least; };
            auto add = [&] {
                int n = 0;
#pragma unroll
                for (int u = 0; u < kSelEach; ++u) n += passes(u);
                n = __reduce_add_sync(0xffffffffu, n);
                if (lane == 0) atomicAdd(&s.sum, (uint32_t)n);
                __syncthreads();
            };
            add();
            if (s.n + s.sum > kSelList) {                 // more than fit (many equal values): the `best` of them, bit by bit
                uint64_t found = 0ull;
                for (int bit = 43; bit >= 0; --bit) {
                    __syncthreads();
                    if (threadIdx.x == 0) s.sum = 0u;
                    __syncthreads();
                    least = found | 1ull << bit;
                    add();
                    if (s.sum >= (uint32_t)K) found = least;
                }
                least = max(found, (uint64_t)(last + 1u) << 12);
            }
            uint32_t take = 0u;
#pragma unroll
            for (int u = 0; u < kSelEach; ++u) take |= (passes(u) ? 1u : 0u) << u;
            append(s, take, lane, [&](int u) {
                uint2 e = make_uint2(0u, 0u);
#pragma unroll
                for (int k = 0; k < kSelEach; ++k)
                    if (k == u) e = make_uint2(key[k], (uint32_t)(w * V + c + X::place(k)));
                return e;
            });
            const int now = rank_list(s, K);
            last = now == K ? s.list[K - 1].x : 0u;
        }
    }
    __syncthreads();
    // this part's best, and the join of the request's parts by the CTA that ends last
    uint2* const mine = P.part + (int64_t)blockIdx.x * K;
    if ((int)threadIdx.x < K) mine[threadIdx.x] = (int)threadIdx.x < s.n ? s.list[threadIdx.x] : make_uint2(0u, 0u);
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();                                  // (cumulative: of what the CTA's threads wrote before the barrier)
        s_last = atomicAdd(P.tickets + r, 1u) == (uint32_t)(P.parts - 1);
        if (s_last) P.tickets[r] = 0;
        __threadfence();
        s.n = 0;
    }
    __syncthreads();
    if (!s_last) return;
    const uint2* const all = P.part + (int64_t)r * P.parts * K;
    const int n = P.parts * K;
    uint2 last = make_uint2(0u, 0u);
    for (int i0 = 0; i0 < n; i0 += 2 * kSelThreads) {
        uint2 e[2];
        uint32_t take = 0u;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = i0 + k * kSelThreads + threadIdx.x;
            e[k] = i < n ? __ldcg(all + i) : make_uint2(0u, 0u);
            if (e[k].x != 0u && before(e[k].x, e[k].y, last.x, last.y)) take |= 1u << k;
        }
        if (!__syncthreads_or(take != 0u)) continue;
        append(s, take, lane, [&](int k) { return k ? e[1] : e[0]; });
        const int now = rank_list(s, K);
        if (now == K) last = s.list[K - 1];
    }
    __syncthreads();
    if ((int)threadIdx.x < K) {
        const bool there = (int)threadIdx.x < s.n;
        const uint2 e = there ? s.list[threadIdx.x] : make_uint2(0u, 0u);
        const int parent = there ? (int)(e.y / (uint32_t)V) : -1, token = there ? (int)(e.y % (uint32_t)V) : -1;
        const int64_t at = (int64_t)r * K + threadIdx.x;
        P.parent[at] = parent;
        P.token[at] = token;
        P.score_out[at] = there ? score_of(e.x) : -INFINITY;
        if (P.done_out) P.done_out[at] = there && (token == P.end_token || (P.done && ld_after(P.done + (int64_t)r * P.width + parent) != 0));
    }
}

}  // namespace

cudaError_t launch_beam_select(const BeamCall& c, cudaStream_t s) {
    BeamParams P = c.p;
    // stretches of whole chunks, as many as fill the GPU a few CTAs deep
    const int64_t beams = (int64_t)P.batch * P.width;
    const int chunks = (P.vocab + kSelChunk - 1) / kSelChunk;
    const int cuts = (int)std::min<int64_t>(chunks, (4ll * device_sms() + beams - 1) / beams), each = (chunks + cuts - 1) / cuts;
    P.per = each * kSelChunk;
    const int of_beam = (P.vocab + P.per - 1) / P.per;
    P.parts = of_beam * P.width;
    const int64_t items = (int64_t)P.batch * P.parts;
    Workspace work(c.ctx, (size_t)items * P.best * sizeof(uint2), (size_t)P.batch);
    if (work.err != cudaSuccess) return work.err;
    P.part = static_cast<uint2*>(work.p);
    P.tickets = work.counters;
    return launch_overlapped(c.bf16 ? beam_select_kernel<true> : beam_select_kernel<false>, dim3((unsigned)items), kSelThreads, 0, s, P);
}

}  // namespace c2kv
