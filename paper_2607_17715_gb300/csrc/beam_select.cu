// The best continuations of beams over the vocabulary (c2kv_beam_select).
//
// A candidate is a place w V + v of a request with the score s_w + (x[w][v] - norm_w), each operation rounded to
// fp32; the `best` of largest score are kept, of equal ones those of the lowest places.  So the choice does not
// depend on how the vocabulary is cut.
//
// Every value is read once, the least that a batch takes.  A CTA takes a stretch of one beam, 4096 or 16384 values, all on
// their way at once and kept as they come: in registers, but for 60 bytes a thread of 64 16-bit values, where 64 registers let four CTAs
// share an SM.  Few of them need be looked at: of the lanes' largest values
// every warp's r-th largest, and the least of those over the warps, is a bound that `best` values reach (r times the warps).
// The score rises with the value, so the bound holds for values, less what the score's rounding can hide.  What passes
// is ranked by counting.  The CTA that ends last joins its request's stretches the same way, the bound from their first ones.
// 16 x 8 beams over 131072 16-bit logits take 19 us, where a list of every value above the first ones took 47; one request
// of 16 beams 15, four beams over 32000 7.4.
#include "paged.cuh"
#include "per_device.cuh"

#include <algorithm>

namespace c2kv {
namespace {

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kSelList = 1024;                            // candidates that are ranked at once

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

struct Best {
    uint2 list[kSelList];                                 // (key, place)
    uint2 best[kBeamsMost];                               // the first of them, in order
    int n;
    int bound;
    uint32_t sum;
};

// Floats as whole numbers of the same order, and back (-0 below 0; no NaN).
__device__ __forceinline__ int ordered(float x) {
    const int i = __float_as_int(x);
    return i < 0 ? i ^ 0x7fffffff : i;
}
__device__ __forceinline__ float of_ordered(int i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }

// Appends to the list; past its end nothing is written, and s.n says how many there were.
__device__ __forceinline__ void append(Best& s, uint32_t key, uint32_t place) {
    const int at = atomicAdd(&s.n, 1);
    if (at < kSelList) s.list[at] = make_uint2(key, place);
}

// Leaves of list[0, n) what a bound does not: of the threads' largest keys every warp's r-th largest, and the least of those
// over the warps, is a key that `best` reach (8 r >= best).  Returns how many there are.
__device__ __forceinline__ int shorten(Best& s, int n, int best) {
    constexpr int kMine = kSelList / kSelThreads;
    uint2 mine[kMine];
    uint32_t rest = 0u, bound = 0u;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int i = threadIdx.x + k * kSelThreads;
        mine[k] = i < n ? s.list[i] : make_uint2(0u, 0u);
        rest = max(rest, mine[k].x);
    }
    for (int i = (best + kSelWarps - 1) / kSelWarps; i > 0; --i) {
        bound = __reduce_max_sync(0xffffffffu, rest);
        const uint32_t at = __ballot_sync(0xffffffffu, rest == bound);
        if ((int)(threadIdx.x % 32) == __ffs(at) - 1) rest = 0u;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s.sum = 0xffffffffu;
        s.n = 0;
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) atomicMin(&s.sum, bound);
    __syncthreads();
    bound = s.sum;
#pragma unroll
    for (int k = 0; k < kMine; ++k)
        if (mine[k].x != 0u && mine[k].x >= bound) append(s, mine[k].x, mine[k].y);
    __syncthreads();
    return s.n;
}

// The first `best` of list[0, n), in order; every thread of the CTA.  Returns how many there are.
// (Every entry meets every other: a long list is shortened first.  Four beams over 50000 values took 42 us without, 512
// beams over 32000 124.)
__device__ __forceinline__ int rank_list(Best& s, int n, int best) {
    if (n > 128) n = shorten(s, n, best);
    for (int i = threadIdx.x; i < n; i += kSelThreads) {
        const uint2 x = s.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) {
            const uint2 y = s.list[j];
            rank += before(y.x, y.y, x.x, x.y);
        }
        if (rank < best) s.best[rank] = x;
    }
    __syncthreads();
    return min(n, best);
}

// A thread's values of a stretch as they lie in memory: kEach of them, 16 bytes' worth next to one another.
template <bool kBf16, int kEach>
struct Values {
    static constexpr int kVec = kBf16 ? 8 : 4;
    static constexpr int kStretch = kEach * kSelThreads;
    uint4 raw[kEach / kVec];
    __device__ static __forceinline__ int place(int u) { return (u / kVec) * (kVec * kSelThreads) + threadIdx.x * kVec + u % kVec; }
    // the values that lie before place t, a bit each
    __device__ static __forceinline__ uint64_t before_place(int t) {
        const int g = t / (kVec * kSelThreads), e = max(0, min(kVec, t - g * kVec * kSelThreads - (int)threadIdx.x * kVec)), n = g * kVec + e;
        return n >= 64 ? ~0ull : (1ull << n) - 1;
    }
    __device__ static __forceinline__ float one(const void* x, int at) {
        if constexpr (kBf16) return __uint_as_float((uint32_t)ld_after(static_cast<const uint16_t*>(x) + at) << 16);
        else return ld_after(static_cast<const float*>(x) + at);
    }
    __device__ __forceinline__ float operator[](int u) const {
        const uint4& y = raw[u / kVec];
        const int e = u % kVec;
        if constexpr (kBf16) {
            const uint32_t w = e < 2 ? y.x : e < 4 ? y.y : e < 6 ? y.z : y.w;
            return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
        } else {
            return __uint_as_float(e == 0 ? y.x : e == 1 ? y.y : e == 2 ? y.z : y.w);
        }
    }
    // values [0, n) from x on; NaN (no candidate) past them.  wide: x lies on 16 bytes.
    __device__ __forceinline__ void load(const void* x, int n, bool wide) {
#pragma unroll
        for (int k = 0; k < kEach / kVec; ++k) {
            const int at = place(k * kVec);
            if (wide && at + kVec <= n) {
                raw[k] = ld_after(reinterpret_cast<const uint4*>(static_cast<const char*>(x) + (int64_t)at * (kBf16 ? 2 : 4)));
            } else {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (kBf16) {
                        const uint16_t* const p = static_cast<const uint16_t*>(x) + at + 2 * e;
                        w[e] = (at + 2 * e < n ? ld_after(p) : 0x7fffu) | (uint32_t)(at + 2 * e + 1 < n ? ld_after(p + 1) : 0x7fffu) << 16;
                    } else {
                        w[e] = at + e < n ? ld_after(static_cast<const uint32_t*>(x) + at + e) : 0x7fffffffu;
                    }
                }
                raw[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};

// Where more values pass a bound than are ranked at once (many equal ones: a mask's lowest value, say), exactly the
// `best` of the stretch go to the list.  `bound`: a value that so many reach.
template <class X, class Append>
__device__ __noinline__ int take_exactly(Best& s, const void* x, int n, bool wide, float score, float norm, bool has_norm, float bound, int best,
                                         int lane, const Append& append_all) {
    constexpr int kEach = X::kStretch / kSelThreads;
    X v;                                                  // (read again: an argument would lie in local memory all along)
    v.load(x, n, wide);
    auto key_at = [&](int u) { return key_of(__fadd_rn(score, has_norm ? __fsub_rn(v[u], norm) : v[u])); };
    auto total = [&](int mine) {                          // over the CTA
        __syncthreads();
        if (threadIdx.x == 0) s.sum = 0u;
        __syncthreads();
        const int n = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) atomicAdd(&s.sum, (uint32_t)n);
        __syncthreads();
        return (int)s.sum;
    };
    auto above = [&](uint32_t key) {                      // values whose keys are larger, a bit each
        asm volatile("" : "+f"(score));                   // (the keys are formed again each time: they would not fit registers)
        uint64_t m = 0ull;
#pragma unroll
        for (int u = 0; u < kEach; ++u) m |= (uint64_t)(key_at(u) > key) << u;
        return m;
    };
    // the key of the last one taken: the bound's, if fewer are above it; else found bit by bit
    uint32_t key = key_of(__fadd_rn(score, has_norm ? __fsub_rn(bound, norm) : bound));
    if (key == 0u || total(__popcll(above(key))) >= best) {
        key = 0u;
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t tried = key | 1u << bit;
            if (total(__popcll(above(tried - 1u))) >= best) key = tried;
        }
    }
    const uint64_t larger = above(key), equal = key ? above(key - 1u) & ~larger : 0ull;
    const int missing = best - total(__popcll(larger));
    // of the equal ones the first: the place before which so many lie
    int place = 0;
#pragma unroll 1
    for (int step = X::kStretch; step > 0; step >>= 1)
        if (total(__popcll(equal & X::before_place(min(place + step, X::kStretch)))) <= missing) place = min(place + step, X::kStretch);
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    append_all(larger | (equal & X::before_place(place)));
    __syncthreads();
    return s.n;
}

template <bool kBf16, int kEach>
__global__ void __launch_bounds__(kSelThreads, kEach > 16 && !kBf16 ? 2 : 4) beam_select_kernel(const __grid_constant__ BeamParams P) {
    using X = Values<kBf16, kEach>;
    static_assert(kEach <= 64, "a bit a value");
    __shared__ Best s;
    __shared__ bool s_last;
    const int lane = threadIdx.x % 32, K = P.best, V = P.vocab;
    const int r = blockIdx.x / P.parts, part = blockIdx.x - r * P.parts, of_beam = P.parts / P.width;
    const int w = part / of_beam, length = ((V + of_beam - 1) / of_beam + 7) & ~7;     // (whole 16-byte lines: equal stretches but for that)
    const int a = (part - w * of_beam) * length, n = min(length, V - a);
    const int64_t row = (int64_t)(P.b0 + r) * P.width + w;
    if (threadIdx.x == 0) {
        s.n = 0;
        s.bound = 0x7fffffff;
    }
    after_kernels_before();
    const float score = ld_after(P.score + row), norm = P.norm ? ld_after(P.norm + row) : 0.f;
    const bool done = P.done && ld_after(P.done + row) != 0;
    auto score_at = [&](float v) { return __fadd_rn(score, P.norm ? __fsub_rn(v, norm) : v); };
    int kept = 0;
    if (done) {                                           // goes on as it is
        if (a == 0 && key_of(score) != 0u) {
            kept = 1;
            if (threadIdx.x == 0) s.best[0] = make_uint2(key_of(score), (uint32_t)(w * V + P.end_token));
        }
    } else if (score > -INFINITY) {
        const char* const x = static_cast<const char*>(P.x) + (row * P.x_stride + a) * (kBf16 ? 2 : 4);
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15u) == 0;
        X v;
        v.load(x, n, wide);
        float top = -INFINITY;                            // (fmaxf leaves NaN out)
#pragma unroll
        for (int u = 0; u < kEach; ++u) top = fmaxf(top, v[u]);
        {
            // (of warps all of whose lanes have values: a short vocabulary leaves some without)
            const int full = min(kSelWarps, n / (32 * X::kVec)), rounds = full > 0 ? (K + full - 1) / full : 33;
            int rest = ordered(top), bound = ordered(-INFINITY);
            for (int i = rounds <= 32 ? rounds : 0; i > 0; --i) {
                bound = __reduce_max_sync(0xffffffffu, rest);
                const uint32_t at = __ballot_sync(0xffffffffu, rest == bound);
                if (lane == __ffs(at) - 1) rest = ordered(-INFINITY);
            }
            __syncthreads();
            if (lane == 0 && ((int)threadIdx.x / 32 < full || rounds > 32)) atomicMin(&s.bound, bound);
            __syncthreads();
        }
        // Scores of values below the bound may round to the bound's: by 2^-23 of what is added, less than this
        const float bound = of_ordered(s.bound);
        float least = bound - 0x1p-20f * (fabsf(bound) + fabsf(norm) + fabsf(score));
        if (!(least == least)) least = -INFINITY;
        uint64_t take = 0ull;                             // a bit a value
        if (top >= least) {
#pragma unroll
            for (int u = 0; u < kEach; ++u) take |= (uint64_t)(v[u] >= least) << u;
        }
        auto append_all = [&](uint64_t which) {           // (values from memory again: few)
            for (; which; which &= which - 1) {
                const int at = X::place(__ffsll((long long)which) - 1);
                const uint32_t key = key_of(score_at(X::one(x, at)));
                if (key != 0u) append(s, key, (uint32_t)(w * V + a + at));
            }
        };
        append_all(take);
        __syncthreads();
        int found = s.n;
        if (found > kSelList) found = take_exactly<X>(s, x, n, wide, score, norm, P.norm != nullptr, bound, K, lane, append_all);
        kept = rank_list(s, found, K);
    }
    // this stretch's best, and the join of the request's by the CTA that ends last
    __syncthreads();
    uint2* const mine = P.part + (int64_t)blockIdx.x * K;
    if ((int)threadIdx.x < K) mine[threadIdx.x] = (int)threadIdx.x < kept ? s.best[threadIdx.x] : make_uint2(0u, 0u);
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
    const int entries = P.parts * K;
    // a bound: the K-th of the first entries of up to 256 stretches
    uint2 bound = make_uint2(1u, 0xffffffffu);            // (any candidate)
    const int heads = min(P.parts, kSelThreads);
    if (heads >= K && K > 1) {
        const uint2 head = (int)threadIdx.x < heads ? __ldcg(all + (int64_t)threadIdx.x * K) : make_uint2(0u, 0u);
        if ((int)threadIdx.x < heads) s.list[threadIdx.x] = head;
        if (threadIdx.x == 0) s.best[0] = bound;
        __syncthreads();
        int rank = 0;
        for (int j = 0; j < heads; ++j) {
            const uint2 y = s.list[j];
            rank += before(y.x, y.y, head.x, head.y);
        }
        if (rank == K - 1 && head.x != 0u) s.best[0] = head;      // (of stretches without a candidate none has a rank)
        __syncthreads();
        bound = s.best[0];
        __syncthreads();
    }
    int total = 0;                                        // the best so far, s.best
    constexpr int kAhead = 8;                             // entries of a thread on their way at once
    for (int i0 = 0; i0 < entries; i0 += kAhead * kSelThreads) {
        uint2 e[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * kSelThreads + threadIdx.x;
            e[k] = i < entries ? __ldcg(all + i) : make_uint2(0u, 0u);
        }
        // (what is left of the list: no more than was there, and two a thread)
#pragma unroll
        for (int k = 0; k < kAhead; k += 2) {
            const int past = i0 + (k + 2) * kSelThreads;
            if (past - 2 * kSelThreads >= entries) break;
#pragma unroll
            for (int j = k; j < k + 2; ++j)
                if (e[j].x != 0u && !before(bound.x, bound.y, e[j].x, e[j].y)) append(s, e[j].x, e[j].y);
            __syncthreads();
            if (s.n > kSelList - 2 * kSelThreads || past >= entries) {
                total = rank_list(s, s.n, K);
                if ((int)threadIdx.x < total) s.list[threadIdx.x] = s.best[threadIdx.x];
                if (total == K) bound = s.best[K - 1];
                __syncthreads();
                if (threadIdx.x == 0) s.n = total;
            }
            __syncthreads();
        }
    }
    if ((int)threadIdx.x < K) {
        const bool there = (int)threadIdx.x < total;
        const uint2 e = there ? s.best[threadIdx.x] : make_uint2(0u, 0u);
        const int parent = there ? (int)(e.y / (uint32_t)V) : -1, token = there ? (int)(e.y % (uint32_t)V) : -1;
        const int64_t at = (int64_t)(P.b0 + r) * K + threadIdx.x;
        P.parent[at] = parent;
        P.token[at] = token;
        P.score_out[at] = there ? score_of(e.x) : -INFINITY;
        if (P.done_out)
            P.done_out[at] = there && (token == P.end_token || (P.done && ld_after(P.done + (int64_t)(P.b0 + r) * P.width + parent) != 0));
    }
}

template <bool kBf16, int kEach>
cudaError_t launch(const BeamCall& c, cudaStream_t s) {
    BeamParams P = c.p;
    constexpr int kStretch = kEach * kSelThreads;
    P.parts = (P.vocab + kStretch - 1) / kStretch * P.width;
    const int most = std::max(1, (1 << 16) / P.parts), per = std::min(P.batch, most);      // requests a launch
    Workspace work(c.ctx, (size_t)per * P.parts * P.best * sizeof(uint2), (size_t)per);
    if (work.err != cudaSuccess) return work.err;
    P.part = static_cast<uint2*>(work.p);
    P.tickets = work.counters;
    for (P.b0 = 0; P.b0 < P.batch; P.b0 += per) {
        const unsigned items = (unsigned)(std::min(per, P.batch - P.b0) * P.parts);
        const cudaError_t e = launch_overlapped(beam_select_kernel<kBf16, kEach>, dim3(items), kSelThreads, 0, s, P);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_beam_select(const BeamCall& c, cudaStream_t s) {
    // Long stretches where they fill the GPU.
    const bool large = (int64_t)c.p.batch * c.p.width * ((c.p.vocab + 16383) / 16384) >= 2 * device_sms();
    if (c.bf16) return large ? launch<true, 64>(c, s) : launch<true, 16>(c, s);
    return large ? launch<false, 64>(c, s) : launch<false, 16>(c, s);
}

}  // namespace c2kv
