// Paged attention of trees of tokens whose rows fill a tile or two (c2kv_paged_attend_tree): tcgen05 straight from
// the pages.
//
// Key tiles made ahead (paged_expand.cu) pay where many row tiles meet them.  Here a (request, KV head) has one or
// two, of 128 rows each, and reading the pages bounds the call: TMA brings them into shared memory, and nothing but
// partials goes back.  8-bit codes become f16 there, relative to a power of two for every
// 32 keys (a V scale that is NaN makes NaN of the rows that see it, and zero of the row itself).  16-bit pages are operands as they lie,
// the queries and the weights two bf16 terms each.
//
// Roundings: a code times its scale has eleven bits, as the queries and the weights over codes have; over 16-bit pages both have
// 16.  A scale has two terms, or fp32's bits in a tile with one below 2^-20 of what its 32 keys' power of two is for (rows that a
// query does not see among them), so the product alone is rounded, down to 2^-29 of that.  Weights take V's powers of two, one
// for most keys as in paged_expand.cu, and lose bits where 32 keys' own is more than 2^24 above another's which count as much.
// Outputs over normal keys and values are off by 1.7e-3 of their norm from 64 bits, which is their own rounding to bf16 (16-bit
// pages: 2.4e-3 with one term of the weights, in 0.89 of the time).
//
// A CTA has an SM to itself, in two groups that take the tiles of 128 keys in turn, each with its own scores and output in
// tensor memory, and its own warps: four for the softmax (a row a thread), four that convert (8-bit codes) or look after
// tiles that are not whole, one that issues products and copies.  So a tile's conversions run beside the softmax of the
// one before, one group's products beside the other's softmax, and the products of a tile's first 64 weights beside the
// forming of its others.  The groups' results join in shared memory, the
// stretches' in a kernel of their own.  Stretches go out longest first, as long as lets the last SM end first.
//
// A tile of 128 keys takes a CTA 1.6 us: tensor cores are busy for 1.1 us of it (16-bit pages, two terms of queries and weights) or 0.6,
// shared memory for 0.9 (products of 128 x 128 read both operands from it at its full rate), the exponentials 0.5.  A stretch
// takes 5 us before its first scores and after its last.  Eight trees of up to 64 nodes over up to 6000 rows of 16-bit pages
// take 58 us (1.8 TB/s of pages, which two row tiles read), 32 nodes over 120000 rows of 8-bit pages 98 us (2.6).
// Tried and slower, with fewer terms: scores 64 keys at a time in two pieces of tensor memory (62 -> 68 us), the next piece of scores
// asked for while one is worked on (61 -> 63), all 128 scores of a row held (spills); the largest of a tile first, then its weights
// (52 -> 54, 103 -> 107).  Nothing is full: the chain scores, weights, products takes most of a group's time for a tile.
//
// Values of V that are not finite (16-bit pages): 0 times one is NaN for rows that do not see it, and a query's second
// term makes NaN of an infinity of K.  A CTA whose results show either begins again with care: such values become zero in
// the tile and are noted, and the rows that see them take them in at the end; keys of a tile with an infinity meet the
// first terms alone.
#include "paged_tile.cuh"

#include <algorithm>
#include <array>
#include <cuda_fp16.h>
#include <optional>
#include <vector>

namespace c2kv {
namespace {

constexpr int kDirGroup = 128;           // threads of a group's softmax, and of its conversions
constexpr int kDirThreads = 4 * kDirGroup + 64;
constexpr int kTurned = 16;              // rows of queries that a warp of the softmax turns (32 by half the warps took 4 us)
constexpr uint32_t kDirTmem = 512;       // a group: S (P over it), O
// What a reference lies below a row's largest score when it is set, and what scores may pass it by before it moves (powers of
// two).  f16 weights: up to 2^15; further up at first (2^12, 2^14) references move oftener (32 nodes over 120000 rows 6 and 11 us more),
// lower (2^8) a tail of small weights has fewer bits.  bf16 ones have fp32's range and meet V as it is: from 2^-8 up to
// one, so that sums of values near the type's largest are numbers where the values' mean is.
__host__ __device__ constexpr float below_top(bool codes) { return codes ? 10.f : -7.f; }
__host__ __device__ constexpr float room_above(bool codes) { return codes ? 15.f : 0.f; }
constexpr int kLeastTiles = 2;           // of a stretch: one a group
constexpr int kItemTiles = 6, kJoinTiles = 3;   // what a stretch takes beside its tiles, and the kernel that joins them, in tiles
constexpr int kMostCuts = 256;           // stretches of one unit's keys: their weights join in shared memory

template <int kReq>
struct DirectLaunch {
    CUtensorMap tm_k, tm_v;              // [n_pages][Hkv][page_size][d], boxes of a page's rows (at most 128)
    uint4* odd;                          // [key tile][Hkv]: rows of V with values that are not finite (16-bit pages)
    float* part_o;                       // [item][128][D] normalised
    float* part_lse;                     // [item][128] log2 domain
    PagedAttn<kReq> a;
};

// Shared memory: queries, then each group's tiles and what is small.
template <int D, bool kCodes>
struct Dir : TileOf<D> {
    using TileOf<D>::kTile;
    static constexpr int kRaw = kCodes ? BN * D : 0;       // bytes of a tile of codes
    static constexpr int kQ = (kCodes ? 1 : 2) * kTile;
    static constexpr int kGroupBytes = 2 * kTile + 2 * kRaw;                  // K, V, and as they come
    static constexpr int kSmall = kQ + 2 * kGroupBytes;    // [group] (codes) scales of K and V; the join's sums
    static constexpr int kBack = kSmall + 2 * 1024;        // powers of two of the queries' rows: a byte each
    static constexpr int kBars = kBack + BM;               // [group] scores, output, K, V, K's and V's tiles ready, last 64 weights, scales, first 64 weights, their products
    static constexpr int kWords = kBars + 2 * 10 * 8;       // tensor memory, abort, [group] K not finite, rows touched (four), [group][2] pages, [group][12] units, [group][4] notes, [group] far
    static constexpr int kSmem = kWords + 192;
};
static_assert(Dir<128, true>::kSmem <= 232448 && Dir<128, false>::kSmem <= 232448, "shared memory of a CTA");

// A barrier of a group's conversions, and whether x holds in any thread of them.
__device__ __forceinline__ void convert_sync(int g) { asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory"); }
__device__ __forceinline__ bool convert_or(int g, bool x) {
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any)
                 : "r"((uint32_t)x), "r"(1 + g)
                 : "memory");
    return any != 0u;
}

// The queries' rows of a warp (kTurned), turned, as two bf16 terms: the first in place, what it lacks a tile behind.
template <int D, int kReq>
__device__ __forceinline__ void turn_queries_twice(const PagedAttn<kReq>& P, const QueryRows<D>& k, int warp, int lane, uint32_t sQ) {
    using C = TileOf<D>;
    constexpr int E = QueryRows<D>::E;
    const int r0 = warp * kTurned, c = lane * E, q0 = c >> 3, q1 = (D / 2 + c) >> 3;
    cp_async_wait<0>();
    __syncwarp();
    float2 cs[E];
    int pos_cs = __shfl_sync(0xffffffffu, k.pos, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) cs[e] = turn_cs_fast(k.turn[e], pos_cs);
#pragma unroll 8
    for (int i = 0; i < kTurned; ++i) {
        const uint32_t at = sQ + (r0 + i) * 128 + (c & 7) * 2;
        const uint32_t a0 = at + (q0 >> 3) * C::kHalf + (((q0 & 7) ^ (i & 7)) << 4), a1 = at + (q1 >> 3) * C::kHalf + (((q1 & 7) ^ (i & 7)) << 4);
        uint32_t x0, x1;
        if constexpr (E == 2) {
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x0) : "r"(a0));
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x1) : "r"(a1));
        } else {
            uint16_t y0, y1;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y0) : "r"(a0));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y1) : "r"(a1));
            x0 = y0;
            x1 = y1;
        }
        float x[E], y[E], lo[E], hi[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            lo[e] = x[e] = __uint_as_float(e == 0 ? x0 << 16 : x0 & 0xffff0000u);
            hi[e] = y[e] = __uint_as_float(e == 0 ? x1 << 16 : x1 & 0xffff0000u);
        }
        if (P.turn) {
            const int pos = __shfl_sync(0xffffffffu, k.pos, i);
            if (pos != pos_cs) {                             // the heads of a token share its angles
#pragma unroll
                for (int e = 0; e < E; ++e) cs[e] = turn_cs_fast(k.turn[e], pos);
                pos_cs = pos;
            }
            rotate<E>(x, y, cs, lo, hi);
        }
        // (what is left of an infinity is nothing)
        auto left = [](float v, uint32_t first) {
            const float d = v - __uint_as_float(first << 16);
            return fabsf(d) < 3.0e38f ? d : 0.f;
        };
        const uint32_t f0 = pack_bf16(lo[0], E == 2 ? lo[E - 1] : 0.f), f1 = pack_bf16(hi[0], E == 2 ? hi[E - 1] : 0.f);
        const uint32_t s0 = pack_bf16(left(lo[0], f0 & 0xffffu), E == 2 ? left(lo[E - 1], f0 >> 16) : 0.f);
        const uint32_t s1 = pack_bf16(left(hi[0], f1 & 0xffffu), E == 2 ? left(hi[E - 1], f1 >> 16) : 0.f);
        if constexpr (E == 2) {
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(a0), "r"(f0));
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(a1), "r"(f1));
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(a0 + C::kTile), "r"(s0));
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(a1 + C::kTile), "r"(s1));
        } else {
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(a0), "h"((uint16_t)f0));
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(a1), "h"((uint16_t)f1));
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(a0 + C::kTile), "h"((uint16_t)s0));
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(a1 + C::kTile), "h"((uint16_t)s1));
        }
    }
}

// The power of two that brings the largest scale, of these bits, to [2^6, 2^7).
__device__ __forceinline__ int unit_of(uint32_t top) { return min(119, (int)(top >> 23) - 126 - 7); }
// V's common power leaves room for rows 2^kCommonRoom above a sample's largest.  (Scales are normal numbers of f16 down to 2^-20 of what a
// power is for: 32 keys with one further down keep their own.)
constexpr int kCommonRoom = 12, kNoUnit = -1000;

// Which rows of a key tile are there: of 16-key groups that lie in pages (bits), from lo to below hi.
struct Rows {
    uint32_t groups;
    int lo, hi;
    __device__ __forceinline__ bool all() const { return groups == 0xffu && lo <= 0 && hi >= BN; }
    __device__ __forceinline__ bool has(int row) const { return (groups >> (row >> 4) & 1u) != 0u && row >= lo && row < hi; }
    // of 32 rows from 32 k on, a bit each
    __device__ __forceinline__ uint32_t of32(int k) const {
        return within((groups >> (2 * k) & 1u ? 0xffffu : 0u) | (groups >> (2 * k + 1) & 1u ? 0xffff0000u : 0u), 32 * k, lo - 1, hi - 1);
    }
};

// A tile of codes [128][D] times their rows' scales (two f16 terms in a word) as f16 in 64-channel blocks under the 128-byte
// swizzle, by a group's threads; (not `all`) rows that are not there become zero.  The product is rounded once, by 2^-11 of a value at
// most, as in key tiles (with one term of the scale, twice: scores over channels eight times the others' were off by 1.6 times as
// much, and 32 nodes over 120000 rows took 3 % less time).  A second term is itself short of bits where the scale is far below the
// largest of its 32 keys; where the first would be, below 2^-20 of it, wide_codes_to_f16 has the tile.  (Scales in fp32 on the
// scores and the weights instead, whose rows every thread reads from shared memory, took the softmax twice the time: 3400 clocks a
// tile for 1600.)
template <int D>
__device__ __forceinline__ void codes_to_f16(uint32_t raw, uint32_t tile, const uint32_t* scale, int t, bool all, const Rows& rows) {
    constexpr int kChunks = D / 16, kStep = kDirGroup / kChunks, kPasses = BN / kStep;
    const int chunk = t % kChunks, block = chunk / 4, q = chunk % 4 * 2, first = block & 1;
    uint4 w[kPasses];
    uint32_t f[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        w[i] = lds128(raw + (t / kChunks + kStep * i) * D + chunk * 16);
        f[i] = scale[t / kChunks + kStep * i];
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int row = t / kChunks + kStep * i;
        if (!all && !rows.has(row)) w[i] = make_uint4(0u, 0u, 0u, 0u);
        const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(x[e / 2] >> (16 * (e & 1)))));
            const __half2 c = *reinterpret_cast<const __half2*>(&h), s = *reinterpret_cast<const __half2*>(&f[i]);
            const __half2 z = __hfma2(c, __low2half2(s), __hmul2(c, __high2half2(s)));
            y[e] = *reinterpret_cast<const uint32_t*>(&z);
        }
        const uint32_t at = tile + block * TileOf<D>::kHalf + row * 128;
        // (the blocks' threads begin with different halves, so that a row's eight meet all banks)
        const uint4 a = make_uint4(y[0], y[1], y[2], y[3]), b = make_uint4(y[4], y[5], y[6], y[7]);
        sts128_(at + (((q + first) ^ (row & 7)) << 4), first ? b : a);
        sts128_(at + (((q + 1 - first) ^ (row & 7)) << 4), first ? a : b);
    }
}

// The same by scales in fp32, for tiles with some that f16 has not as normal numbers: one rounding, of the product, to eleven
// bits down to 2^-29 of what the largest scale makes of a code of 448.
template <int D>
__device__ __noinline__ void wide_codes_to_f16(uint32_t raw, uint32_t tile, const uint32_t* scale, int t, bool all, Rows rows) {
    constexpr int kChunks = D / 16, kStep = kDirGroup / kChunks;
    const int chunk = t % kChunks, q = chunk % 4 * 2;
#pragma unroll 1
    for (int row = t / kChunks; row < BN; row += kStep) {
        uint4 w = lds128(raw + row * D + chunk * 16);
        if (!all && !rows.has(row)) w = make_uint4(0u, 0u, 0u, 0u);
        const float f = __uint_as_float(scale[row]);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 z = codes2(x[e / 2] >> (16 * (e & 1)));
            y[e] = pack_f16(z.x * f, z.y * f);
        }
        const uint32_t at = tile + chunk / 4 * TileOf<D>::kHalf + row * 128;
        sts128_(at + ((q ^ (row & 7)) << 4), make_uint4(y[0], y[1], y[2], y[3]));
        sts128_(at + (((q + 1) ^ (row & 7)) << 4), make_uint4(y[4], y[5], y[6], y[7]));
    }
}

// (16-bit pages) whether a tile has values that are not finite in the thread's row; and V's tile put right: rows that are
// not there become zero, with care values that are not finite too, and whether there were any.  A thread a row.
template <int D>
__device__ __forceinline__ bool tile_odd(uint32_t tile, int t, const Rows& rows) {
    const int row = t;
    bool odd = false;
    if (!rows.has(row)) return false;
#pragma unroll 4
    for (int line = 0; line < D / 8; ++line) {
        const uint4 w = lds128(tile + line / 8 * TileOf<D>::kHalf + row * 128 + line % 8 * 16);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) odd = odd || (((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0u;
    }
    return odd;
}
template <int D>
__device__ __forceinline__ bool put_right(uint32_t tile, int t, const Rows& rows, bool care) {
    const int row = t;
    const bool there = rows.has(row);
    bool odd = false;
    if (there && !care) return false;
#pragma unroll 1
    for (int line = 0; line < D / 8; ++line) {
        const uint32_t at = tile + line / 8 * TileOf<D>::kHalf + row * 128 + line % 8 * 16;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (there) {
            w = lds128(at);
            uint32_t* const x = reinterpret_cast<uint32_t*>(&w);
            uint32_t any = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {                    // (an exponent of ones carries into the bit above it)
                const uint32_t out = ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                any |= out;
                x[e] &= ~((out >> 15) * 0xffffu);
            }
            if (any == 0u) continue;
            odd = true;
        }
        sts128_(at, w);
    }
    return odd;
}

template <int D, bool kCodes, int kReq>
__global__ void __launch_bounds__(kDirThreads, 1) paged_direct_kernel(const __grid_constant__ DirectLaunch<kReq> X) {
    using T = __nv_bfloat16;
    using C = Dir<D, kCodes>;
    constexpr uint32_t idS = kCodes ? idesc_f16(BM, BN, false) : idesc_bf16(BM, BN, false);
    constexpr uint32_t idO = kCodes ? idesc_f16(BM, D, true) : idesc_bf16(BM, D, true);
    constexpr int EB = kCodes ? 1 : 2, kBox = kCodes ? D : 64;       // channels of a TMA box
    const PagedAttn<kReq>& P = X.a;
    extern __shared__ __align__(1024) uint8_t smem[];
    enum { kSoftmax, kConvert, kIssue };
    const int role = threadIdx.x / (2 * kDirGroup), t = threadIdx.x % kDirGroup, lane = threadIdx.x % 32;
    const int g = role == kIssue ? threadIdx.x / 32 & 1 : threadIdx.x / kDirGroup & 1;
    const uint32_t sQ = smem_u32(smem), sK = sQ + C::kQ + g * C::kGroupBytes, sV = sK + C::kTile;
    const uint32_t inK = kCodes ? sV + C::kTile : sK, inV = kCodes ? inK + C::kRaw : sV;      // where the pages go
    uint32_t* const scales = reinterpret_cast<uint32_t*>(smem + C::kSmall) + g * BN * 2;      // (codes) [K, V][key], two f16 terms
    int8_t* const s_back = reinterpret_cast<int8_t*>(smem + C::kBack);
    const uint32_t bars = sQ + C::kBars + g * 80, barS = bars, barO = bars + 8, barK = bars + 16, barV = bars + 24;
    const uint32_t readyK = bars + 32, readyV = bars + 40, readyP = bars + 48, readyC = bars + 56, readyW = bars + 64, barW = bars + 72;     // (an arrival a warp)
    uint32_t* const words = reinterpret_cast<uint32_t*>(smem + C::kWords);
    volatile uint32_t* const abort = words + 1;
    volatile uint32_t* const s_alone = words + 2 + g;         // the queries' first terms alone: K's tile has values that are not finite
    uint32_t* const s_touched = words + 4;                    // [4]: a bit a row
    volatile uint32_t* const s_groups = words + 8 + 2 * g;    // [2]: which 16-key groups of a tile lie in pages, every other tile's
    // (codes) exponents that 32 keys lack: K's of every other tile, V's; and rows of V's tile that are not finite, a bit each
    volatile int32_t* const s_units = reinterpret_cast<int32_t*>(words) + 12 + 12 * g;
    volatile uint32_t* const s_note = words + 36 + 4 * g;
    uint8_t* const s_far = reinterpret_cast<uint8_t*>(words + 44 + g);       // (codes) 32 keys of a tile with scales far apart, a byte each
    if ((sQ & 1023u) != 0u) {                                 // (tiles lie on their swizzle's pattern: it always does)
        if (threadIdx.x == 0) atomicOr(P.err, 2);
        return;
    }
    const Item w = find_item<true, BM>(P, (int)blockIdx.x);
    const int hi = w.R.n_keys;
    const int n = (w.n + 1 - g) / 2;                          // the group's tiles: g, g + 2, ..
    if (threadIdx.x == 0) {
        for (int i = 0; i < 20; ++i) mbar_init(sQ + C::kBars + 8 * i, i % 10 < 4 || i % 10 == 9 ? 1 : 4);
        *abort = 0u;
        for (int i = 0; i < 4; ++i) s_touched[i] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&X.tm_k)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&X.tm_v)) : "memory");
    }
    if (threadIdx.x / 32 == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(words)), "r"(kDirTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    after_kernels_before();
    QueryRows<D> rows;
    if (role == kSoftmax) rows = fetch_queries<D, kTurned>(P, w, (int)threadIdx.x / 32, lane, sQ);
    tc_fence_before();
    __syncthreads();                                          // (barriers, tensor memory)
    tc_fence_after();
    const uint32_t tmem = words[0] + (uint32_t)(g * 256), tmemO = tmem + BN;
    // the kernel that joins cut keys may be set up from here on: it waits for this grid to end
    if (threadIdx.x == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto key_of = [&](int i) { return (w.j0 + 2 * i + g) * BN; };
    auto rows_of = [&](int i) { return Rows{s_groups[i & 1], w.k_lo - key_of(i), hi - key_of(i)}; };
    auto arrive = [&](uint32_t bar) {                         // the warp has written what the products read
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    uint32_t uses = 0;                                        // of the barriers, parity of their next phase: a tile each

    // the page of 16-key group lane % 8 of the group's tile i, -1 for none or without a key that any query sees
    auto pages_of = [&](int i) {
        const int key = key_of(i) + (lane & 7) * 16;
        // (pages that a window has left behind may be gone from the table)
        if (i >= n || key >= hi || ((key >> P.pg.page_shift) + 1) << P.pg.page_shift <= w.k_lo) return -1;
        const int page = ld_after(P.pg.table + (int64_t)w.R.row * P.pg.table_stride + (key >> P.pg.page_shift));
        if (page >= 0 && page < P.pg.n_pages) return page;
        atomicOr(P.err, 1);
        return -1;
    };

    if (role == kIssue) {
        const int box_rows = min(BN, 1 << P.pg.page_shift), boxes = BN / box_rows;
        // a tile of `pages` into shared memory
        auto bring = [&](const CUtensorMap* tm, uint32_t to, uint32_t bar, int pages) {
            const int p = __shfl_sync(0xffffffffu, pages, lane * (box_rows / 16) & 7);
            const bool mine = lane < boxes && p >= 0;
            const uint32_t count = __popc(__ballot_sync(0xffffffffu, mine));
            if (lane == 0) mbar_expect_tx(bar, count * (uint32_t)(box_rows * D * EB));
            __syncwarp();
            if (mine) {
#pragma unroll
                for (int b = 0; b < D / kBox; ++b)
                    tma_load_4d(to + b * TileOf<D>::kHalf + lane * box_rows * (kBox * EB), tm, b * kBox, 0, w.hk, p, bar);
            }
        };
        auto bring_k = [&](int i, int pages) {                // K of tile i, and which rows the others find there
            const uint32_t there = __ballot_sync(0xffffffffu, pages >= 0) & 0xffu;
            if (lane == 0) s_groups[i & 1] = there;
            bring(&X.tm_k, inK, barK, pages);
        };
        const uint64_t dq = sw128_desc(sQ, 16, 1024), dk = sw128_desc(sK, 16, 1024), dv = sw128_desc(sV, C::kHalf, 1024);
        auto scores = [&](int i, uint32_t phase, bool care) {
            if constexpr (kCodes) {
                mbar_wait(readyK, phase, P.err, abort);
            } else {
                mbar_wait(barK, phase, P.err, abort);
                if (care) mbar_wait(readyK, (uint32_t)i & 1u, P.err, abort);          // (this way round alone)
            }
            if (lane == 0) {
                tc_fence_after();
                const bool alone = !kCodes && care && *s_alone != 0u;
#pragma unroll
                for (int y = kCodes ? 0 : 1; y >= 0; --y) {
                    if (y == 1 && alone) continue;
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t off = (uint64_t)(((kk >> 2) * C::kHalf + (kk & 3) * 32) >> 4);
                        mma_bf16(tmem, dq + (uint64_t)(y * C::kTile >> 4) + off, dk + off, idS, kk > 0 || (!kCodes && y == 0 && !alone) ? 1u : 0u);
                    }
                }
                mma_commit(barS);
            }
            __syncwarp();
        };
        auto all = [&](bool care) {
            int pages = pages_of(0), pages1 = pages_of(1);    // of this tile and the next
            if (n > 0) {
                bring_k(0, pages);
                bring(&X.tm_v, inV, barV, pages);
            }
            if (!care) __syncthreads();                       // (the queries)
            if (n > 0) scores(0, uses, care);
            for (int i = 0; i < n; ++i, uses ^= 1u) {
                const int pages2 = pages_of(i + 2);
                const bool more = i + 1 < n;
                // a next tile where this one's has been read: by the conversion, or by the products
                if constexpr (!kCodes) mbar_wait(barS, uses, P.err, abort);
                if (more) bring_k(i + 1, pages1);
                mbar_wait(readyV, uses, P.err, abort);
                if (kCodes && more) bring(&X.tm_v, inV, barV, pages1);
                for (int half = 0; half < 2; ++half) {
                    mbar_wait(half ? readyP : readyW, uses, P.err, abort);
                    if (lane == 0) {
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < BN / 32; ++kk) {
                            const int k = half * (BN / 32) + kk;
                            const uint64_t v = dv + (uint64_t)((k * 16 * 128) >> 4);
                            if constexpr (kCodes) {
                                mma_bf16_ts(tmemO, tmem + (uint32_t)k * 8u, v, idO, k > 0 || i > 0 ? 1u : 0u);
                            } else {                          // what the first terms lack, and those
                                mma_bf16_ts(tmemO, tmem + (uint32_t)(k / 2 * 32 + k % 2 * 8 + 16), v, idO, k > 0 || i > 0 ? 1u : 0u);
                                mma_bf16_ts(tmemO, tmem + (uint32_t)(k / 2 * 32 + k % 2 * 8), v, idO, 1u);
                            }
                        }
                        mma_commit(half ? barO : barW);
                    }
                    __syncwarp();
                }
                if (more) scores(i + 1, uses ^ 1u, care);
                if constexpr (!kCodes) {
                    mbar_wait(barO, uses, P.err, abort);
                    if (more) bring(&X.tm_v, inV, barV, pages1);
                }
                pages = pages1;
                pages1 = pages2;
            }
        };
        all(false);
        if constexpr (!kCodes)
            if (__syncthreads_or(0)) all(true);
        for (int i = 0; i < 4; ++i) __syncthreads();          // (of the join below)
        return;
    }
    if (role == kConvert) {
        // (codes) K's and V's scale of key t of tile i
        [[maybe_unused]] int pages1 = -1;                     // of the next tile
        [[maybe_unused]] float k_scale = 0.f, v_scale = 0.f;
        auto ask_scales = [&](int i, int pages) {
            const int p = __shfl_sync(0xffffffffu, pages, t >> 4), at = key_of(i) + t;
            const bool ok = p >= 0 && at >= w.k_lo && at < hi;
            const int64_t from = (int64_t)p * P.pg.scale_stride + (w.hk << P.pg.page_shift) + (t & ((1 << P.pg.page_shift) - 1));
            k_scale = v_scale = 0.f;
            if (ok) {
                k_scale = ld_after(P.pg.k_scale + from);
                v_scale = ld_after(P.pg.v_scale + from);
            }
        };
        // ... relative to a power of two for 32 keys, the largest to [2^6, 2^7): a code's product is below 2^16.  `none`: the
        // power of keys that are all zero; `far`: a scale that is no normal number of f16 then.  V's is `shared` where all of theirs are
        // normal numbers by it: references of weights take it, and where one 32 keys' is above the others' these have fewer bits
        int common = kNoUnit;
        auto put_scale = [&](float x, uint32_t* to, int least, int none, int shared, bool& far) {
            const uint32_t y = __float_as_uint(x) & 0x7fffffffu, top = __reduce_max_sync(0xffffffffu, y < 0x7f800000u ? y : 0u);
            int unit = top == 0u ? none : max(least, unit_of(top));
            auto below = [&](int unit) { return y - 1u < ((uint32_t)max(unit + 113, 1) << 23) - 1u; };      // 2^(unit - 14), and not zero
            if (shared != kNoUnit && unit <= shared && !__any_sync(0xffffffffu, below(shared))) unit = shared;
            const __half first = __float2half_rn(x * pow2i(-unit));
            const __half2 h = __halves2half2(first, __float2half_rn(x * pow2i(-unit) - __half2float(first)));
            far = far || below(unit);
            to[t] = *reinterpret_cast<const uint32_t*>(&h);
            return unit;
        };
        // K's (V's) tile i, some of whose scales f16 has not, by scales in fp32: over what its threads made of it.  (As another
        // way instead of a second one it cost tiles that do not take it 1 %.)
        [[maybe_unused]] auto again = [&](int i, bool v, const Rows& there) {
            uint32_t* const to = scales + (v ? BN : 0);
            const int p = __shfl_sync(0xffffffffu, pages_of(i), t >> 4), at = key_of(i) + t, unit = s_units[v ? 8 + t / 32 : (i & 1) * 4 + t / 32];
            float x = 0.f;
            if (p >= 0 && at >= w.k_lo && at < hi)
                x = ld_after((v ? P.pg.v_scale : P.pg.k_scale) + (int64_t)p * P.pg.scale_stride + (w.hk << P.pg.page_shift) +
                             (t & ((1 << P.pg.page_shift) - 1)));
            if (v && !(fabsf(x) < CUDART_INF_F)) x = 0.f;
            convert_sync(g);                                  // (the f16 ones have been read)
            to[t] = __float_as_uint(x * pow2i(-unit));
            convert_sync(g);
            wide_codes_to_f16<D>(v ? inV : inK, v ? sV : sK, to, t, there.all(), there);
        };
        auto all = [&](bool care) {
            if constexpr (kCodes) {
                // V's common power: room for rows 2^kCommonRoom above the largest of 32 spread over what is seen
                const int key = w.k_lo + (int)((int64_t)(hi - w.k_lo) * lane / 32);
                const int page = ld_after(P.pg.table + (int64_t)w.R.row * P.pg.table_stride + (key >> P.pg.page_shift)), pages0 = pages_of(0);
                pages1 = pages_of(1);
                uint32_t y = 0u;
                if (page >= 0 && page < P.pg.n_pages)
                    y = __float_as_uint(ld_after(P.pg.v_scale + (int64_t)page * P.pg.scale_stride + (w.hk << P.pg.page_shift) +
                                                 (key & ((1 << P.pg.page_shift) - 1)))) & 0x7fffffffu;
                ask_scales(0, pages0);
                const uint32_t top = __reduce_max_sync(0xffffffffu, y < 0x7f800000u ? y : 0u);
                if (top != 0u) common = max(-90, min(119, unit_of(top) + kCommonRoom));
            }
            if (!care) __syncthreads();
            for (int i = 0; i < n; ++i, uses ^= 1u) {
                if constexpr (kCodes) {
                    mbar_wait(barK, uses, P.err, abort);
                    if (i > 0) mbar_wait(barS, uses ^ 1u, P.err, abort);             // the products before have read K's tile, and V's
                    const bool odd = !(fabsf(v_scale) < CUDART_INF_F);       // (V's row becomes zero, and NaN of the rows that see it)
                    // (V's from -90 on: the sum of weights takes 2^-unit.  And -90 where all are zero, at 0 it would raise references)
                    bool far = false;
                    const int k_unit = put_scale(k_scale, scales, -120, 0, kNoUnit, far);
                    const int v_unit = put_scale(odd ? 0.f : v_scale, scales + BN, -90, -90, common, far);
                    if (lane == 0) s_units[(i & 1) * 4 + t / 32] = k_unit;
                    far = __any_sync(0xffffffffu, far);
                    if (lane == 0) s_far[t / 32] = far;
                    convert_sync(g);
                    far = *reinterpret_cast<volatile uint32_t*>(s_far) != 0u;
                    ask_scales(i + 1, pages1);
                    pages1 = pages_of(i + 2);
                    codes_to_f16<D>(inK, sK, scales, t, true, Rows{});               // (hidden keys' scores are replaced)
                    if (far) again(i, false, Rows{0xffu, 0, BN});
                    fence_proxy_async();
                    arrive(readyK);
                    mbar_wait(barV, uses, P.err, abort);
                    const Rows there = rows_of(i);
                    if (i > 0) mbar_wait(barO, uses ^ 1u, P.err, abort);
                    const uint32_t note = __ballot_sync(0xffffffffu, odd);
                    if (lane == 0) {                          // (the tile before has been taken)
                        s_units[8 + t / 32] = v_unit;
                        s_note[t / 32] = note;
                    }
                    arrive(readyC);
                    codes_to_f16<D>(inV, sV, scales + BN, t, there.all(), there);
                    if (far) again(i, true, there);
                    fence_proxy_async();
                    convert_sync(g);                          // (the scales have been read)
                } else {
                    if (care) {
                        mbar_wait(barK, uses, P.err, abort);
                        const bool odd = convert_or(g, tile_odd<D>(sK, t, rows_of(i)));
                        if (t == 0) *s_alone = odd;
                        arrive(readyK);
                    }
                    mbar_wait(barV, uses, P.err, abort);
                    const Rows there = rows_of(i);
                    if (care || !there.all()) {
                        const uint32_t odd = __ballot_sync(0xffffffffu, put_right<D>(sV, t, there, care));
                        fence_proxy_async();
                        if (care && lane == 0) {
                            s_note[t / 32] = odd;
                            reinterpret_cast<uint32_t*>(X.odd + (int64_t)(w.R.scratch + w.j0 + 2 * i + g) * P.hkv + w.hk)[t / 32] = odd;
                        }
                    }
                }
                arrive(readyV);
            }
        };
        all(false);
        if constexpr (!kCodes)
            if (__syncthreads_or(0)) all(true);
        for (int i = 0; i < 4; ++i) __syncthreads();
        return;
    }

    const int G = P.hq / P.hkv, row = t;
    const uint32_t lane_addr = (uint32_t)(t & ~31) << 16;
    const uint32_t colS = tmem + lane_addr, colO = tmemO + lane_addr;
    const Climb<PagedAttn<kReq>> sight(P, w, (w.row0 + min(row, w.live - 1)) / G);
    float ref = -CUDART_INF_F, l = 0.f;
    bool touched = false;                                     // by values that are not finite
    // (an output of products that came before these scores, and are done)
    auto scale_output = [&](float alpha) {
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
            uint32_t ov[16];
            tmem_ld16(colO + c * 16, ov);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
            tmem_st16(colO + c * 16, ov);
        }
    };
    // a sum of weights by 2^e, e <= 0: further down than one factor of fp32 reaches (V's units differ by up to 2^209)
    auto lowered = [](float sum, float e) {
        if constexpr (kCodes) sum *= ex2(fminf(e + 120.f, 0.f));
        return sum * ex2(kCodes ? fmaxf(e, -120.f) : e);
    };
    // weights of 32 keys, by a power of two
    auto scale_weights = [&](int c, float alpha) {
        tmem_st_wait();
#pragma unroll 1
        for (int x = 0; x < (kCodes ? 1 : 2); ++x) {
            const uint32_t at = colS + (kCodes ? c * 16 : c * 32 + x * 16);
            uint32_t pv[16];
            tmem_ld16(at, pv);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float2 w = kCodes ? __half22float2(*reinterpret_cast<const __half2*>(&pv[e]))
                                        : make_float2(__uint_as_float(pv[e] << 16), __uint_as_float(pv[e] & 0xffff0000u));
                pv[e] = kCodes ? pack_f16(w.x * alpha, w.y * alpha) : pack_bf16(w.x * alpha, w.y * alpha);
            }
            tmem_st16(at, pv);
        }
    };
    auto softmax = [&](bool care) {
        ref = -CUDART_INF_F;
        l = 0.f;
        if (!care) {                                          // the first tiles are on their way meanwhile
            if constexpr (kCodes) turn_queries<D, kTurned>(P, rows, (int)threadIdx.x / 32, lane, sQ, s_back);
            else turn_queries_twice<D>(P, rows, (int)threadIdx.x / 32, lane, sQ);
            fence_proxy_async();
            __syncthreads();
        }
        const float row_f = kCodes ? P.scale_log2 * pow2i(s_back[row]) : P.scale_log2;
        for (int i = 0; i < n; ++i, uses ^= 1u) {
            const int key0 = key_of(i);
            // (codes: what follows is known while the scores are formed)
            mbar_wait(kCodes ? readyC : barS, uses, P.err, abort);
            const Rows there = rows_of(i);                    // (written ahead of the copies that the scores are behind)
            // of 32 keys (codes): scores in units of 2^[K's exponent], weights of V's
            // (within fp32's normal range: hidden scores of -inf times zero would be no number)
            auto factor = [&](int c) { return kCodes ? fminf(fmaxf(row_f * pow2i(s_units[(i & 1) * 4 + c]), 0x1p-126f), 0x1.fffffep127f) : row_f; };
            auto exponent = [&](int c) { return kCodes ? (float)s_units[8 + c] : 0.f; };
            const bool edge = !there.all() || !sight.sees_tile(key0);
            uint32_t seen[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (edge) {
                sight.of64(key0, seen[0], seen[1]);
                sight.of64(key0 + 64, seen[2], seen[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c) seen[c] &= there.of32(c);
            }
            if (kCodes ? (s_note[0] | s_note[1] | s_note[2] | s_note[3]) != 0u : care) {       // rows of V that are not finite
                if (!kCodes) mbar_wait(readyV, uses, P.err, abort);
                uint32_t of[4];
                sight.of64(key0, of[0], of[1]);
                sight.of64(key0 + 64, of[2], of[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c) touched = touched || (s_note[c] & of[c]) != 0u;
            }
            if constexpr (kCodes) mbar_wait(barS, uses, P.err, abort);
            tc_fence_after();
            // 32 keys at a time: 128 scores do not fit the registers, and what does not goes through an L1 that shared memory
            // leaves next to nothing of.  The reference is a whole number: where a later piece moves it, weights that are written
            // already take the difference in their exponents.
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t sv[32];
                tmem_ld32(colS + c * 32, sv);
                tmem_ld_wait();
                if (edge) {
                    const uint32_t bits = c < 2 ? c == 0 ? seen[0] : seen[1] : c == 2 ? seen[2] : seen[3];
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!(bits >> e & 1u)) sv[e] = __float_as_uint(-CUDART_INF_F);
                }
                const float f = factor(c);
                float ve = exponent(c);
                float m = -CUDART_INF_F, m2 = -CUDART_INF_F;
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    m = fmax3(m, __uint_as_float(sv[e]), __uint_as_float(sv[e + 1]));
                    m2 = fmax3(m2, __uint_as_float(sv[e + 2]), __uint_as_float(sv[e + 3]));
                }
                const float most = fmaf(fmaxf(m, m2), f, ve);
                const bool moves = most > ref + room_above(kCodes);      // (from -inf: any number)
                if (__any_sync(0xffffffffu, moves)) {
                    float alpha = 1.f;
                    if (moves) {
                        const float to = ceilf(most - below_top(kCodes));
                        alpha = ex2(ref - to);
                        l = lowered(l, ref - to);
                        ref = to;
                    }
                    if (c >= 2) {                             // (the products of the first half are under way)
                        mbar_wait(barW, uses, P.err, abort);
                        tc_fence_after();
                    }
                    if (i > 0 || c >= 2) scale_output(alpha);
                    if (c & 1) scale_weights(c - 1, alpha);
                }
                // weights of 2^-40 and less are nothing in f16: the sum takes them where fp32 still holds them
                if constexpr (kCodes) ve = fmaxf(ve, fminf(fmaf(-fmaxf(m, m2), f, ref - 40.f), 200.f));
                const float off = ve - (ref == -CUDART_INF_F ? 0.f : ref);
                float ps[4] = {0.f, 0.f, 0.f, 0.f};
                uint32_t pk[16];
                [[maybe_unused]] uint32_t pl[16];             // (16-bit pages) what the first terms, cut off, lack
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    float a[4];
                    ffma2(a[0], a[1], __uint_as_float(sv[e]), __uint_as_float(sv[e + 1]), f, off);
                    ffma2(a[2], a[3], __uint_as_float(sv[e + 2]), __uint_as_float(sv[e + 3]), f, off);
#pragma unroll
                    for (int k = 0; k < 4; ++k) a[k] = ex2(a[k]);
                    fadd2(ps[0], ps[1], a[0], a[1]);
                    fadd2(ps[2], ps[3], a[2], a[3]);
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        if constexpr (kCodes) {
                            pk[e / 2 + k / 2] = pack_f16(a[k], a[k + 1]);
                        } else {
                            const uint32_t x = __float_as_uint(a[k]), y = __float_as_uint(a[k + 1]);
                            pk[e / 2 + k / 2] = __byte_perm(x, y, 0x7632);
                            pl[e / 2 + k / 2] = pack_bf16(a[k] - __uint_as_float(x & 0xffff0000u), a[k + 1] - __uint_as_float(y & 0xffff0000u));
                        }
                    }
                }
                if constexpr (kCodes) {
                    tmem_st16(colS + c * 16, pk);             // (over scores that are taken: the thread's own)
                } else {
                    tmem_st16(colS + c * 32, pk);
                    tmem_st16(colS + c * 32 + 16, pl);
                }
                l = fmaf((ps[0] + ps[1]) + (ps[2] + ps[3]), ex2(-ve), l);
                if (c == 1) {
                    tmem_st_wait();
                    tc_fence_before();
                    arrive(readyW);
                }
            }
            tmem_st_wait();
            tc_fence_before();
            arrive(readyP);
        }
        if (n > 0) {
            mbar_wait(barO, uses ^ 1u, P.err, abort);
            tc_fence_after();
        }
    };
    softmax(false);
    if constexpr (!kCodes) {
        // values that are not finite: of a sum, or (where weights of zero met them) of the output
        float z = l * 0.f;
        if (n > 0) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
                uint32_t ov[16];
                tmem_ld16(colO + c * 16, ov);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) z = fmaf(__uint_as_float(ov[e]), 0.f, z);
            }
        }
        tc_fence_before();
        if (__syncthreads_or(z != 0.f)) {
            tc_fence_after();
            softmax(true);
        }
    }

    // (found again: kept over the tiles it would take registers of theirs)
    int item;
    asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(item));
    const Item v = find_item<true, BM>(P, item);
    const bool there = row < v.live;
    const int my = min(row, v.live - 1), tok = (v.row0 + my) / G;

    // the groups join: the second's output, in units of the common reference, through its tiles, a column a row of them
    float* const joined = reinterpret_cast<float*>(smem + C::kQ + C::kGroupBytes);            // [D][128]
    float* const of_group = reinterpret_cast<float*>(smem + C::kSmall);                       // [reference, sum, of the first][128]
    tc_fence_before();
    __syncthreads();                                          // (what lay there has been read)
    tc_fence_after();
    of_group[2 * BM * g + row] = ref;
    of_group[2 * BM * g + BM + row] = l;
    if (touched) atomicOr(s_touched + row / 32, 1u << (row & 31));
    __syncthreads();
    const float ref0 = of_group[row], l0 = of_group[BM + row], ref1 = of_group[2 * BM + row], l1 = of_group[3 * BM + row];
    const float top = fmaxf(ref0, ref1), base = top == -CUDART_INF_F ? 0.f : top;
    const float a0 = ex2(ref0 - base), a1 = ex2(ref1 - base);
    if (g == 1) {
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
            uint32_t ov[16];
            if (n > 0) {
                tmem_ld16(colO + c * 16, ov);
                tmem_ld_wait();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) joined[(c * 16 + e) * BM + row] = n > 0 ? __uint_as_float(ov[e]) * a1 : 0.f;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    l = lowered(l0, ref0 - base) + lowered(l1, ref1 - base);
    const bool poisoned = s_touched[row / 32] >> (row & 31) & 1u;            // (codes) by a row of V whose scale is no number
    const float inv = l == 0.f ? 0.f : kCodes && poisoned ? CUDART_NAN_F : 1.0f / l;
    const float lse2 = l == 0.f ? -CUDART_INF_F : top + log2f(l);
    const bool whole = v.R.splits == 1;
    if (g == 0) {
        const int64_t out_tok = v.R.q0 + tok;
        const int h = v.hk * G + (v.row0 + my) % G;
        T* const orow = static_cast<T*>(P.out) + (out_tok * P.hq + h) * D;
        float* const prow = X.part_o + ((int64_t)item * BM + row) * D;
        const bool wide = (reinterpret_cast<uintptr_t>(P.out) & 31u) == 0;
        const float none = there && whole && l == 0.f ? of_no_weight<true>(P, v.R, tok) : 0.f;
#pragma unroll 2
        for (int c = 0; c < D / 16; ++c) {
            uint32_t ov[16];
            if (n > 0) {
                tmem_ld16(colO + c * 16, ov);
                tmem_ld_wait();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float y = fmaf(n > 0 ? __uint_as_float(ov[e]) : 0.f, a0, joined[(c * 16 + e) * BM + row]);
                ov[e] = __float_as_uint(l == 0.f ? none : y * inv);
            }
            if (!there) continue;
            if (whole) {
                uint32_t o8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o8[e] = pack_bf16(__uint_as_float(ov[2 * e]), __uint_as_float(ov[2 * e + 1]));
                if (wide) {
                    stg256(orow + c * 16, o8);
                } else {
                    *reinterpret_cast<uint4*>(orow + c * 16) = make_uint4(o8[0], o8[1], o8[2], o8[3]);
                    *reinterpret_cast<uint4*>(orow + c * 16 + 8) = make_uint4(o8[4], o8[5], o8[6], o8[7]);
                }
            } else {
                stg256(prow + c * 16, ov);
                stg256(prow + c * 16 + 8, ov + 8);
            }
        }
        if (there) {
            if (!whole) X.part_lse[(int64_t)item * BM + row] = lse2;
            else if (P.lse) P.lse[(int64_t)h * P.n_tokens + out_tok] = lse2 * 0.69314718055994531f;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (!kCodes && g == 0) {
        const uint32_t bad = __ballot_sync(0xffffffffu, there && poisoned && l < CUDART_INF_F);
        if (bad) take_in<D, kCodes, BM>(X, v, bad, sight, row & ~31, lane, smem);
    }
    if (threadIdx.x / 32 == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(words[0]), "r"(kDirTmem) : "memory");
    }
}

// ------------------------------------------------------------------ host side

template <int D, bool kCodes, int kReq>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_direct_kernel<D, kCodes, kReq>;
    constexpr int kSmem = Dir<D, kCodes>::kSmem;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, kSmem);
    if (e != cudaSuccess) return e;
    const int G = c.hq / c.hkv;
    for (int b0 = 0; b0 < n; b0 += kReq) {
        const int nb = std::min(n - b0, kReq);
        DirectLaunch<kReq> X;
        fill_paged(X.a, c, D, req + b0, nb);
        // key tiles of each request, and the stretches of them that are done first
        std::array<int, kReq> tiles{};
        int64_t notes = 0, work = 0;
        int longest = 0;
        for (int i = 0; i < nb; ++i) {
            PagedReq& q = X.a.req[i];
            const int64_t first = c.window ? std::max<int64_t>(0, (int64_t)q.n_keys - q.nq + 1 - c.window) : 0;
            const int lo = (int)(first / BN), hi = (int)(((int64_t)q.n_keys + BN - 1) / BN);
            tiles[i] = std::max(1, hi - lo);
            q.tile0 = 0;
            q.tiles = (int32_t)(((int64_t)q.nq * G + BM - 1) / BM);
            q.scratch = (int32_t)(notes - lo);
            notes += tiles[i];
            work += (int64_t)tiles[i] * q.tiles * c.hkv;
            longest = std::max(longest, tiles[i]);
        }
        const int slots = device_sms();
        auto splits_at = [&](int i, int per) { return std::min((tiles[i] + per - 1) / per, kMostCuts); };
        auto length_at = [&](int i, int per) { return (tiles[i] + splits_at(i, per) - 1) / splits_at(i, per); };
        std::array<int, kReq> order{};
        auto sort_at = [&](int per) {
            for (int i = 0; i < nb; ++i) order[i] = i;
            std::stable_sort(order.begin(), order.begin() + nb, [&](int x, int y) { return length_at(x, per) > length_at(y, per); });
        };
        // the tiles that the last SM has done when stretches of `per` go out, longest first, to SMs as these get free
        auto end_at = [&](int per) {
            struct Free {
                int64_t at, sms;
            };
            std::vector<Free> free{{0, slots}};               // (the last is the first to be free)
            bool cut = false;
            sort_at(per);
            for (int k = 0; k < nb; ++k) {
                const int i = order[k], s = splits_at(i, per);
                cut = cut || s > 1;
                for (int64_t n = (int64_t)s * X.a.req[i].tiles * c.hkv; n > 0;) {
                    const Free f = free.back();
                    const int64_t m = std::min(n, f.sms);
                    free.back().sms -= m;
                    if (free.back().sms == 0) free.pop_back();
                    const Free then{f.at + kItemTiles + length_at(i, per), m};
                    free.insert(std::find_if(free.begin(), free.end(), [&](const Free& x) { return x.at <= then.at; }), then);
                    n -= m;
                }
            }
            return free.front().at + (cut ? kJoinTiles : 0);
        };
        int per = longest;
        int64_t end = end_at(per);
        for (int p = (int)std::max<int64_t>(kLeastTiles, work / slots / 3); p < longest; p = std::max(p + 1, p * 6 / 5)) {
            const int64_t e = end_at(p);
            if (e < end) end = e, per = p;
        }
        auto splits_of = [&](int i) { return splits_at(i, per); };
        sort_at(per);
        {
            const std::array<int, kReq> was = tiles;
            std::vector<PagedReq> reqs(X.a.req, X.a.req + nb);
            for (int k = 0; k < nb; ++k) {
                tiles[k] = was[order[k]];
                X.a.req[k] = reqs[order[k]];
            }
        }
        int64_t items = 0, units = 0;
        int most = 1;
        auto lay_out = [&](bool cut) {
            items = units = 0;
            most = 1;
            for (int i = 0; i < nb; ++i) {
                PagedReq& q = X.a.req[i];
                q.splits = cut ? splits_of(i) : 1;
                q.item0 = (int32_t)items;
                q.unit0 = (int32_t)units;
                if (q.splits > 1) {
                    units += (int64_t)q.tiles * c.hkv;
                    most = std::max(most, q.splits);
                }
                items += (int64_t)q.tiles * c.hkv * q.splits;
            }
        };
        lay_out(true);
        // (partials are stored 32 bytes at a time)
        const size_t odd_bytes = ((size_t)notes * c.hkv * sizeof(uint4) + 255) / 256 * 256;
        std::optional<Workspace> scratch;
        size_t o_bytes = units > 0 ? (size_t)items * BM * D * 4 : 0;
        scratch.emplace(c.ctx, odd_bytes + o_bytes + (units > 0 ? (size_t)items * BM * 4 : 0), 0);
        if (scratch->err == cudaErrorMemoryAllocation && units > 0) {     // no room for partials: keys are not cut, slower
            (void)cudaGetLastError();
            lay_out(false);
            o_bytes = 0;
            scratch.emplace(c.ctx, odd_bytes, 0);
        }
        if (scratch->err == cudaErrorMemoryAllocation) {                  // nor for a note a key tile
            (void)cudaGetLastError();
            e = launch_paged_mma(c, req + b0, nb, D, kCodes, s);
            if (e != cudaSuccess) return e;
            continue;
        }
        if (scratch->err != cudaSuccess) return scratch->err;
        char* const base = static_cast<char*>(scratch->p);
        X.odd = reinterpret_cast<uint4*>(base);
        X.part_o = reinterpret_cast<float*>(base + odd_bytes);
        X.part_lse = reinterpret_cast<float*>(base + odd_bytes + o_bytes);
        const int box_rows = std::min(BN, 1 << c.pg.page_shift), box = kCodes ? D : 64;
        const auto swizzle = kCodes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
        if (!encode_page_map(&X.tm_k, c.pg.k, c.pg, c.hkv, D, kCodes, box, box_rows, swizzle) ||
            !encode_page_map(&X.tm_v, c.pg.v, c.pg, c.hkv, D, kCodes, box, box_rows, swizzle))
            return cudaErrorInvalidValue;
        e = launch_overlapped(kernel, (unsigned)items, kDirThreads, kSmem, s, X);
        if (e == cudaSuccess && units > 0)
            e = launch_overlapped(paged_join_kernel<D, BM, true, DirectLaunch<kReq>>, (unsigned)(units * (BM / join_rows(D))), kJoinThreads,
                                  (size_t)most * join_rows(D) * 4, s, X);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_paged_direct(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? launch<128, true, kPagedFew>(c, req, n, s) : launch<128, false, kPagedFew>(c, req, n, s);
    return codes ? launch<64, true, kPagedFew>(c, req, n, s) : launch<64, false, kPagedFew>(c, req, n, s);
}

}  // namespace c2kv
