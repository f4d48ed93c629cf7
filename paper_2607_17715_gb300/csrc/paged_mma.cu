// Paged attention of few query rows: one to a few tokens of each request (c2kv_paged_attend).
//
// The rows of a (request, KV head) -- its tokens times the group's heads -- meet every key once, so
// the call is bound by reading the pages.  One CTA takes 8 NT rows and a stretch of keys, dealt to its
// four warps in blocks of 32.  Each warp runs alone: a ring of TMA stages of its own, its own running
// maximum and sum.  The warps' results join in shared memory, the stretches' in the CTA that ends last.
//
// The products are mma.sync (a tcgen05 tile of 128 rows would be mostly empty, and would need the 8-bit
// codes converted through shared memory instead of in registers), turned over: S^T = K.Q^T and
// O^T = V^T.P^T, keys and channels in the 16 rows of an operand, query rows in its columns of 8, so that
// a token of four heads wastes half a tile and not three quarters.  P^T comes out of S^T's registers by
// 8 x 8 transposes (movmatrix).
//
// E4M3 codes become f16 in registers, exactly: half of them by the conversion instruction, which takes a
// quarter of its lanes a clock and bound the kernel alone (a block 2350 clocks a warp), half by shifts
// and masks, which leave 2^-8 of the value; the queries' channels, or O's, give that back.  Scales stay
// in fp32: a key's K scale multiplies its row of S^T, its V scale its row of P^T.  P must fit f16, so V
// scales are taken relative to a power of two, the largest of them so far, that O is counted in; it moves
// like the running maximum does.  The largest weight is 2^15, so that f16 keeps 11 bits of weight times scale
// down to 2^-29 of the largest of both (with a largest weight of one a row whose value is 2^10 times the others',
// whatever its own weight, left nothing of weights of 2^-15).  Queries are f16 too, each row scaled by a power of two so that its
// largest value is near 2^6 (2^14 where codes are short of 2^8): their rounding is at most 2^-11 of a value.  Over
// 16-bit pages operands are bf16, and the queries two terms of it each: one alone, 8 bits of a value that
// RoPE turned, made two thirds of the output's error over long contexts (5.6e-3 of it, against 2e-3).
//
// Values that are not finite (16-bit pages): 0 times one of V would be NaN for rows that do not see it, and a
// query's second term makes NaN of an infinity of K.  A warp looks at its sums every eight blocks, and where
// they show one it begins again with care: such values of V become zero, which rows see them is noted, and
// they are taken in when the warps join; keys of infinities meet the first terms alone.  That is about twice
// the time at most, where rows computed again key by key took 14 ms for 0.3 (64 requests over 8192 rows).
// Over 8-bit pages a row that is no number has scale NaN, and a hidden key's weight is set to zero after it
// meets that.
//
// Operand layouts.  The contraction over channels does not care for their order, so a lane takes the
// channels that lie next to one another in its row: 16-byte shared loads, conflict-free under the
// 128-byte swizzle, with no transpose of V (a lane loads the same channels of four keys and pairs them).
//
// Measured (32 / 8 heads): one token over 131000 rows of 16 bits, 537 MB in 87 us (6.2 TB/s); one token of
// 16 requests over 500 to 2000 rows of codes, 37 MB in 12 us, of which first loads and the two joins
// are half; five tokens of eight requests with groups of eight (40 rows), 46 MB in 30 us, bound by the issue of
// the warps' chains: each of two tiles of 24 rows converts the codes for itself.
#include "paged.cuh"
#include "per_device.cuh"
#include "ptx.cuh"
#include "rope.cuh"

#include <algorithm>
#include <cuda_fp16.h>
#include <optional>
#include <type_traits>

namespace c2kv {
namespace {

constexpr int kWarps = 4;
constexpr int kBlk = 32;                 // keys of a warp's block

constexpr int kMostEights = 4;           // eights of query rows a CTA: what its registers hold (40 rows: two tiles of
                                         // three eights 33 us, one of five, which spills, 44)

// Blocks in flight a warp (kStages) and CTAs an SM (kCtas): three CTAs of two blocks where registers and
// shared memory hold them (8-bit codes and eight rows), the warps' chains of dependent instructions being
// what takes the time then; else two of three blocks, or one of heads of 128 channels in 16 bits.
template <int D, bool kCodes, int NT>
struct Lay {
    static constexpr int EB = kCodes ? 1 : 2;
    static constexpr int BC = kCodes ? D : 64;         // channels of a TMA box
    static constexpr int NB = D / BC;                  // boxes a row
    static constexpr int RB = BC * EB;                 // bytes of a box row (64 or 128)
    static constexpr int CQ = BC / 4;                  // channels of K a lane takes of a box row
    static constexpr int KS = D / 16;                  // k-steps of S
    static constexpr int CV = BC / 8;                  // channels of V a lane takes of a box row
    static constexpr int kBox = kBlk * RB;             // bytes of a box of a block
    static constexpr int kSide = NB * kBox;            // K (or V) of a block
    static constexpr int kStages = kCodes && NT == 1 ? 2 : 3;
    static constexpr int kStage = 2 * kSide;
    static constexpr int kScale = kCodes ? 2 * kBlk * 4 : 0;       // bytes of a block's scales
    static constexpr int kRing = kWarps * kStages * kStage;
    static constexpr int kSmem = 1024 /*align*/ + kRing + kWarps * kStages * kScale;
    static constexpr int kCtas = kCodes && NT == 1 ? 3 : kSmem <= 108 * 1024 ? 2 : 1;
    static constexpr int kPitch = D + 4;               // floats between rows of the joined results
};
static_assert(Lay<128, false, kMostEights>::kSmem + 24 * 1024 <= 227 * 1024 && 3 * (Lay<128, true, 1>::kSmem + 5 * 1024) <= 227 * 1024,
              "shared memory of an SM");

// log2 of the largest weight: what the reference lies below a row's largest score so far (P: f16 or bf16).
template <bool kCodes>
__host__ __device__ constexpr float top_weight() {
    return kCodes ? 15.f : 0.f;
}

constexpr int kMaxStretches = 128;       // of one unit's keys: their weights join in shared memory

template <int kReq>
struct MmaLaunch {
    CUtensorMap tm_k, tm_v;              // [n_pages][Hkv][page_size][d], boxes of min(page_size, 32) rows
    int32_t box_rows;
    float* part_o;                       // [item][8 * NT][D] normalised
    float* part_lse;                     // [item][8 * NT] log2 domain
    uint32_t* tickets;                   // [unit], zero between launches
    PagedAttn<kReq> a;
};

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool kHalf>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (kHalf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool kHalf>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The two E4M3 codes of 16 bits as f16.
__device__ __forceinline__ uint32_t half2_of(uint16_t w) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
    return h;
}
__device__ __forceinline__ uint32_t lo_half2(uint32_t w) { return half2_of((uint16_t)w); }
__device__ __forceinline__ uint32_t hi_half2(uint32_t w) { return half2_of((uint16_t)(w >> 16)); }

// Shared memory by ordinary loads, which the compiler may move between the barriers.
__device__ __forceinline__ void lds4(const uint8_t* a, uint32_t& x, uint32_t& y, uint32_t& z, uint32_t& w) {
    const uint4 v = *reinterpret_cast<const uint4*>(a);
    x = v.x;
    y = v.y;
    z = v.z;
    w = v.w;
}
__device__ __forceinline__ void lds2(const uint8_t* a, uint32_t& x, uint32_t& y) {
    const uint2 v = *reinterpret_cast<const uint2*>(a);
    x = v.x;
    y = v.y;
}
__device__ __forceinline__ float lds_f(const uint8_t* a) { return *reinterpret_cast<const float*>(a); }

// The four codes of a word as two pairs of f16, 2^-8 of their values: bytes 0 and 2, bytes 1 and 3.
__device__ __forceinline__ uint32_t masked_pair(uint32_t w) {
    return (w & 0x80008000u) | ((w >> 1) & 0x3f803f80u);
}
__device__ __forceinline__ uint32_t odd_pair(uint32_t w) { return masked_pair(w); }
__device__ __forceinline__ uint32_t even_pair(uint32_t w) { return masked_pair(w << 8); }

// An 8 x 8 matrix of 16-bit values, a row in four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// K-step s of S (four channels a lane): by shifts and masks, or by the conversion instruction.
__host__ __device__ constexpr bool by_masks(bool codes, int s) { return codes && (s & 1); }

// Where channel ch of query row `row` lies in the fragments of Q^T: index of its 16 bits.
template <int D, bool kCodes, int NT>
__device__ __forceinline__ int q_place(int row, int ch) {
    using L = Lay<D, kCodes, NT>;
    const int box = ch / L::BC, in = ch % L::BC, c = in / L::CQ, s = box * (L::CQ / 4) + in % L::CQ / 4, e = in % 4;
    const int reg = by_masks(kCodes, s) ? e & 1 : e >> 1, half = by_masks(kCodes, s) ? e >> 1 : e & 1;
    return (((s * NT + row / 8) * 32 + (row % 8) * 4 + c) * 2 + reg) * 2 + half;
}

// 16-bit values that are not finite become zero: an exponent of ones carries into the bit above it.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t finite(uint32_t w) { return w & ~((not_finite(w) >> 15) * 0xffffu); }

// The scores of a block of 16-bit keys among which some value is not finite, the queries' second terms taken
// times the finite ones alone: of an infinity times a query, its first term says all.
template <int NT>
struct Scores {
    float x[NT][2][4];
};
template <int D, int NT>
__device__ __noinline__ Scores<NT> scores_of_infinities(const uint8_t* sk, const uint8_t* q_at, int g, int c) {
    using L = Lay<D, false, NT>;
    Scores<NT> r;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) r.x[t][h][e] = 0.f;
#pragma unroll 1
    for (int s = 0; s < L::KS; ++s) {                          // (words 2 s, 2 s + 1 of the lane's channels of a key)
        const int b = s / (L::CQ / 4), u = s % (L::CQ / 4);
        uint32_t a[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                lds2(sk + b * L::kBox + (16 * h + 8 * k + g) * L::RB + ((2 * c + u / 2) ^ g) * 16 + u % 2 * 8, a[h][k], a[h][2 + k]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 1; x >= 0; --x) {
                uint32_t q0, q1;
                lds2(q_at + x * (L::KS * NT * 256) + (s * NT + t) * 256, q0, q1);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t y[4] = {x ? finite(a[h][0]) : a[h][0], x ? finite(a[h][1]) : a[h][1], x ? finite(a[h][2]) : a[h][2],
                                           x ? finite(a[h][3]) : a[h][3]};
                    mma16816<false>(r.x[t][h], y, q0, q1);
                }
            }
    }
    return r;
}

// Values of a block's V (16 bits) that are not finite become zero in shared memory, and are noted for the rows
// that see them: a byte a channel in odd[row][D / 4], 1 infinity, 2 minus it, 4 NaN.
// A key with an infinity of K too scores -inf where the row's sum is a number: 0 times its infinities is NaN.
template <int D, class Sees>
__device__ __noinline__ void set_aside(uint8_t* sv, int key0, uint32_t has, int k_lo, int k_hi, const Sees sees, int live, uint32_t* odd,
                                       int lane) {
    using L = Lay<D, false, 1>;
    constexpr int kLanes = D / 4, kStep = 32 / kLanes;         // 8 bytes a lane: four channels
    const int b = lane % kLanes / 16, u = lane % 16;
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < kBlk; j += kStep) {
        const uint2 w = *(reinterpret_cast<const uint2*>(sv + b * L::kBox + (j + lane / kLanes) * L::RB) + u);
        any |= not_finite(w.x) | not_finite(w.y);
    }
    if (!__any_sync(0xffffffffu, any != 0u)) return;
#pragma unroll 1
    for (int j = lane / kLanes; j < kBlk; j += kStep) {
        const int key = key0 + j;
        uint2* const at = reinterpret_cast<uint2*>(sv + b * L::kBox + j * L::RB) + u;
        const uint2 w = *at, y = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(at) - L::kSide);   // (K's)
        const uint32_t of_k = __ballot_sync(0xffffffffu, (not_finite(y.x) | not_finite(y.y)) != 0u) >> (lane & ~(kLanes - 1));
        if (key < k_lo || key >= k_hi || !(has >> (j >> 4) & 1u)) continue;
        if ((not_finite(w.x) | not_finite(w.y)) == 0u) continue;
        const bool no_weight = (of_k & (0xffffffffu >> (32 - kLanes))) != 0u;
        uint32_t is = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = (e < 2 ? w.x : w.y) >> (16 * (e & 1)) & 0xffffu;
            if ((x & 0x7f80u) == 0x7f80u) is |= ((x & 0x7fu) || no_weight ? 4u : (x & 0x8000u) ? 2u : 1u) << (8 * e);
        }
        const int word = b * 16 + ((u / 2) ^ (j & 7)) * 2 + u % 2;       // (16-byte lines of a row are swapped)
        for (int row = 0; row < live; ++row)
            if (sees(row, key)) atomicOr(odd + row * (D / 4) + word, is);
        *at = make_uint2(finite(w.x), finite(w.y));
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // (TMA writes there next)
    __syncwarp();
}

// Whether a query row sees a key that is there: rows up to its own, or its way to the root of its tree.
struct RowsBefore {
    const int* end;          // [row]: the last key it sees
    int window;
    __device__ __forceinline__ bool operator()(int row, int key) const { return key <= end[row] && (!window || key > end[row] - window); }
};
struct RowsOfTree {
    const int* start;        // [row]: the last key before the tree that it does not see
    const uint32_t* bits;    // [row][kTreeWords]
    int before;
    __device__ __forceinline__ bool operator()(int row, int key) const { return tree_sees(key, before, start[row], bits + row * kTreeWords); }
};

template <int D, bool kCodes, int NT, int kReq, bool kTree>
__global__ void __launch_bounds__(kWarps * 32, Lay<D, kCodes, NT>::kCtas > 1 ? Lay<D, kCodes, NT>::kCtas : 2) paged_mma_kernel(const __grid_constant__ MmaLaunch<kReq> X) {
    using L = Lay<D, kCodes, NT>;
    using T = __nv_bfloat16;
    constexpr int kStages = L::kStages;
    constexpr int kRows = 8 * NT, MT = D / 16;         // query rows; 16-channel tiles of O^T
    constexpr bool kHeldQ = NT == 1;                   // Q^T in registers
    constexpr int kTerms = kCodes ? 1 : 2;             // of a query's value
    const PagedAttn<kReq>& P = X.a;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kStages];
    __shared__ __align__(16) uint16_t s_q[kTerms][L::KS * NT * 32 * 4];
    __shared__ __align__(8) float s_rs[kRows];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ int s_unit[kWarps];       // (codes) V's scales are below 2^this
    __shared__ int s_end[kRows];         // (trees: the last key before the tree that a row does not see)
    __shared__ uint32_t s_bits[kTree ? kRows * kTreeWords : 1];
    __shared__ uint32_t s_abort, s_last;
    // (16-bit pages) values that are not finite, of keys that a row sees: a byte a channel, 1 infinity, 2 minus
    // it, 4 NaN
    __shared__ uint32_t s_odd[kCodes ? 1 : kRows * (D / 4)];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
    uint8_t* const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&X.tm_k)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&X.tm_v)) : "memory");
    }
    // the work item: (request, stretch, KV head, row tile)
    int r = 0;
    for (int hi = P.batch; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.req[mid].item0 <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    const PagedReq R = P.req[r];
    const uint32_t G = P.group, n_tiles = R.tiles, n_split = R.splits;
    uint32_t it = blockIdx.x - R.item0, rt = 0;
    if (n_tiles > 1) {
        rt = it % n_tiles;
        it /= n_tiles;
    }
    const uint32_t sp = it / (uint32_t)P.hkv;
    const int hk = (int)(it - sp * P.hkv);
    const uint32_t row0 = rt * kRows;
    const int live = min(kRows, (int)(R.nq * G - row0));
    // keys that any row of the tile sees: [k_lo, k_hi); every row sees up to `first` (from its window on)
    const int before = R.n_keys - R.nq, first = kTree ? before - 1 : before + (int)(row0 / G), k_hi = before + (int)((row0 + live - 1) / G) + 1;
    const int k_lo = P.window ? max(0, (kTree ? before : first) - P.window + 1) : 0;      // (a tree's root has the least depth)
    const int b_lo = k_lo / kBlk, b_n = max(0, (k_hi + kBlk - 1) / kBlk - b_lo);
    const uint32_t each = (uint32_t)b_n / n_split, rest = (uint32_t)b_n - each * n_split;   // the first `rest` stretches: one more
    const int b0 = b_lo + (int)(each * sp + min(sp, rest)), b1 = b0 + (int)(each + (sp < rest));
    const int n_it = b1 - b0 > warp ? (b1 - b0 - warp + kWarps - 1) / kWarps : 0;

    // a warp's barriers are its own: a block is there when its tiles are, and each lane's scales
    if (lane < kStages) mbar_init(smem_u32(&s_full[warp][lane]), kCodes ? 33 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    if (threadIdx.x == 0) s_abort = 0;
    if constexpr (!kCodes)
        for (int i = threadIdx.x; i < kRows * (D / 4); i += kWarps * 32) s_odd[i] = 0;

    after_kernels_before();
    // the warp's query rows, on their way before the keys are: behind a ring's worth of tiles they took 4 us
    constexpr int C = D / 64, kMine = (kRows + kWarps - 1) / kWarps;   // channels of each half a lane; rows a warp
    uint32_t q_raw[kMine][2];
    int q_pos[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const uint32_t rr = row0 + min(warp + i * kWarps, live - 1), tok = rr / G;
        const T* q = static_cast<const T*>(P.q) + (int64_t)(R.q0 + tok) * P.q_stride + (int64_t)(hk * G + rr - tok * G) * D + lane * C;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if constexpr (C == 2) q_raw[i][half] = ld_after(reinterpret_cast<const uint32_t*>(q + half * (D / 2)));
            else q_raw[i][half] = ld_after(reinterpret_cast<const uint16_t*>(q + half * (D / 2)));
        }
        q_pos[i] = P.turn ? ld_after(P.turn + R.q0 + tok) : 0;
    }
    uint64_t turn[C] = {};
    if (P.turn) {
#pragma unroll
        for (int e = 0; e < C; ++e) turn[e] = lane_turn(P.rope.turn, lane * C + e);
    }

    const uint32_t ring = smem_u32(smem) + warp * kStages * L::kStage;
    const uint32_t scales = smem_u32(smem) + L::kRing + warp * kStages * L::kScale;
    const int32_t* const table = P.pg.table + (int64_t)R.row * P.pg.table_stride;
    const int box_rows = X.box_rows, boxes = kBlk / box_rows;      // pages a block spans: 1, or 2 of 16 rows
    // Pages of 32 of the warp's blocks, one a lane, looked up together; -1 for one that is none, or
    // that holds no key of the tile (the second half of a last block).
    int pages0 = -1, pages1 = -1;
    auto look_up = [&](int i0) {
        pages0 = pages1 = -1;
        if (i0 + lane >= n_it) return;
        const int key = (b0 + warp + (i0 + lane) * kWarps) * kBlk;
        // (a page that a window has left behind may be gone from the table)
        const bool one = boxes == 1 || key + 16 > k_lo, two = boxes == 2 && key + 16 < k_hi;
        if (one) pages0 = ld_after(table + (key >> P.pg.page_shift));
        if (two) pages1 = ld_after(table + ((key + 16) >> P.pg.page_shift));
        if (one && (pages0 < 0 || pages0 >= P.pg.n_pages)) {
            atomicOr(P.err, 1);
            pages0 = -1;
        }
        if (two && (pages1 < 0 || pages1 >= P.pg.n_pages)) {
            atomicOr(P.err, 1);
            pages1 = -1;
        }
    };
    // Block i of the warp into a stage; returns which halves of its keys are loaded (bits 0 and 1).
    auto issue = [&](int i, int stage) -> uint32_t {
        const int p0 = __shfl_sync(0xffffffffu, pages0, i & 31), p1 = __shfl_sync(0xffffffffu, pages1, i & 31);
        const int off = ((b0 + warp + i * kWarps) * kBlk) & ((1 << P.pg.page_shift) - 1);
        if (lane == 0) {
            const uint32_t bar = smem_u32(&s_full[warp][stage]), dst = ring + stage * L::kStage;
            mbar_expect_tx(bar, ((p0 >= 0) + (p1 >= 0)) * box_rows * 2 * D * L::EB);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int page = k ? p1 : p0, at_row = k ? 0 : off;
                if (page < 0) continue;
#pragma unroll
                for (int b = 0; b < L::NB; ++b) {
                    const uint32_t to = dst + b * L::kBox + k * 16 * L::RB;
                    tma_load_4d(to, &X.tm_k, b * L::BC, at_row, hk, page, bar);
                    tma_load_4d(to + L::kSide, &X.tm_v, b * L::BC, at_row, hk, page, bar);
                }
            }
        }
        if constexpr (kCodes) {          // a key's scales a lane (held in registers they were waited for at once)
            const bool second = boxes == 2 && lane >= 16;
            const int page = second ? p1 : p0;
            const uint32_t to = scales + stage * L::kScale + lane * 4;
            if (page >= 0) {
                const int64_t at = (int64_t)page * P.pg.scale_stride + ((int64_t)hk << P.pg.page_shift) + (second ? lane - 16 : off + lane);
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(P.pg.k_scale + at) : "memory");
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + kBlk * 4), "l"(P.pg.v_scale + at) : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&s_full[warp][stage])) : "memory");
        }
        return boxes == 1 ? (p0 >= 0 ? 3u : 0u) : (p0 >= 0 ? 1u : 0u) | (p1 >= 0 ? 2u : 0u);
    };
    look_up(0);
    uint32_t loaded[kStages];            // of the blocks in flight, the next one to be used first
#pragma unroll
    for (int i = 0; i < kStages; ++i) loaded[i] = i < n_it ? issue(i, i) : 0u;
    if constexpr (kTree) {               // the rows' ways through the tree, where the stretch meets it or a window
        if (threadIdx.x < kRows) {
            const int row = threadIdx.x;
#pragma unroll
            for (int i = 0; i < kTreeWords; ++i) s_bits[row * kTreeWords + i] = 0u;
            s_end[row] = -1;
            if (b1 * kBlk > before || P.window)
                s_end[row] = tree_bits(P.parent + R.q0, (int)((row0 + min(row, live - 1)) / G), before, P.window, P.err, s_bits + row * kTreeWords);
        }
    }

    // the tile's queries: turned, as fragments of Q^T
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int row = warp + i * kWarps;
        if (row >= kRows) break;
        float x[2 * C];
        const bool there = row < live;
        const uint32_t tok = (row0 + min(row, live - 1)) / G;
#pragma unroll
        for (int e = 0; e < C; ++e) {
            x[e] = there ? __uint_as_float(e == 0 ? q_raw[i][0] << 16 : q_raw[i][0] & 0xffff0000u) : 0.f;
            x[C + e] = there ? __uint_as_float(e == 0 ? q_raw[i][1] << 16 : q_raw[i][1] & 0xffff0000u) : 0.f;
        }
        if (P.turn) {
#pragma unroll
            for (int e = 0; e < C; ++e) {
                float a, b;
                rotate1(x[e], x[C + e], turn_cs_fast(turn[e], q_pos[i]), a, b);
                x[e] = a;
                x[C + e] = b;
            }
        }
        float back = 1.f, f = 1.f;
        if constexpr (kCodes) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 2 * C; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            top = __reduce_max_sync(0xffffffffu, top);
            // largest value to [2^6, 2^7); zero and non-finite rows as they are
            const int ex = (int)(top >> 23) - 127;
            if (top < 0x7f800000u && ex > -100) {
                f = pow2i(6 - ex);
                back = pow2i(ex - 6);
            }
        }
        if (lane == 0) {
            s_rs[row] = back * P.scale_log2;
            if constexpr (!kTree) s_end[row] = before + (int)tok;
        }
#pragma unroll
        for (int e = 0; e < 2 * C; ++e) {
            const int ch = (e / C) * (D / 2) + lane * C + e % C;
            const bool masks = by_masks(kCodes, (ch % L::BC) % L::CQ / 4);
            const uint32_t v = pack2<kCodes>(masks ? x[e] * f * 256.f : x[e] * f, 0.f);
            const int at = q_place<D, kCodes, NT>(row, ch);
            s_q[0][at] = (uint16_t)v;
            if constexpr (kTerms == 2) {                       // (what is left of an infinity is nothing)
                const float left = x[e] - __uint_as_float(v << 16);
                s_q[kTerms - 1][at] = (uint16_t)pack2<kCodes>(fabsf(left) < 3.0e38f ? left : 0.f, 0.f);
            }
        }
    }
    __syncthreads();

    // O^T: channel tile m of 16 (lane: channels g and g + 8 of it), rows 2c and 2c + 1 of each eight
    float o[NT][MT][4], m[NT][2], l[NT][2];
    auto start = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int n = 0; n < MT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][n][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[t][e] = -INFINITY;
                l[t][e] = 0.f;
            }
        }
    };
    start();
    int unit = -127;                     // O counts in 2^unit (E4M3)
    uint32_t qf[kTerms][kHeldQ ? L::KS : 1][2];
    const uint8_t* const q_at = reinterpret_cast<const uint8_t*>(s_q) + lane * 8;
    constexpr int kTermBytes = L::KS * NT * 256;
    if constexpr (kHeldQ) {
#pragma unroll
        for (int x = 0; x < kTerms; ++x)
#pragma unroll
            for (int s = 0; s < L::KS; ++s) lds2(q_at + x * kTermBytes + s * 256, qf[x][s][0], qf[x][s][1]);
    }

    const auto sees = [&] {
        if constexpr (kTree) return RowsOfTree{s_end, s_bits, before};
        else return RowsBefore{s_end, P.window};
    }();
    int stage = 0, parity = 0;
    auto advance = [&] {
        if (++stage == kStages) {
            stage = 0;
            parity ^= 1;
        }
    };
    // The warp's blocks.  Without care it may stop early, and returns how many it has done, where a sum is not
    // finite (16-bit pages); else -1.
    auto blocks = [&](auto care) -> int {
        constexpr bool kCare = decltype(care)::value;
        for (int i = 0; i < n_it; ++i) {
            const int key0 = (b0 + warp + i * kWarps) * kBlk;
            const uint8_t* const sk = smem + (warp * kStages + stage) * L::kStage;
            const uint8_t* const sv = sk + L::kSide;
            const uint8_t* const ssc = smem + L::kRing + (warp * kStages + stage) * L::kScale;
            const uint32_t has = loaded[0];
            // some key is hidden from some row, or was not loaded: then every key is asked
            const bool edge = has != 3 || key0 + kBlk - 1 > first || (P.window && key0 <= k_hi - 1 - P.window);
            // key j of the block is there, and some row of the tile sees it
            auto there = [&](int j) { return key0 + j < k_hi && key0 + j >= k_lo && (has >> (j >> 4) & 1u); };
            mbar_wait(smem_u32(&s_full[warp][stage]), parity, P.err, &s_abort);

            // S^T of keys 16 h + g (e = 0, 1) and + 8 (2, 3), rows 8 t + 2c and + 1
            float s[NT][2][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][h][e] = 0.f;
#pragma unroll
            for (int b = 0; b < L::NB; ++b) {
                constexpr int KW = L::CQ * L::EB / 4;              // words of the lane's channels of a key
                uint32_t w[2][2][KW];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint8_t* const at = sk + b * L::kBox + (n * 8 + g) * L::RB;
                    uint32_t* const to = w[n >> 1][n & 1];
#pragma unroll
                    for (int u = 0; u < KW / 4; ++u)
                        lds4(at + (L::RB == 128 ? ((2 * c + u) ^ g) * 16 : c * 16), to[4 * u], to[4 * u + 1], to[4 * u + 2], to[4 * u + 3]);
                }
#pragma unroll
                for (int ks = 0; ks < L::CQ / 4; ++ks) {
                    uint32_t a[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {              // rows g and g + 8 of the 16 keys
                            const uint32_t x = w[h][k][kCodes ? ks : (2 * ks) % KW];
                            if constexpr (kCodes) {
                                a[h][k] = by_masks(true, ks) ? even_pair(x) : lo_half2(x);
                                a[h][2 + k] = by_masks(true, ks) ? odd_pair(x) : hi_half2(x);
                            } else {
                                a[h][k] = x;
                                a[h][2 + k] = w[h][k][(2 * ks + 1) % KW];
                            }
                        }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int s_i = b * (L::CQ / 4) + ks;
#pragma unroll
                        for (int x = kTerms - 1; x >= 0; --x) {
                            uint32_t q0, q1;
                            if constexpr (kHeldQ) {
                                q0 = qf[x][s_i][0];
                                q1 = qf[x][s_i][1];
                            } else {
                                lds2(q_at + x * kTermBytes + (s_i * NT + t) * 256, q0, q1);
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) mma16816<kCodes>(s[t][h], a[h], q0, q1);
                        }
                    }
                }
            }
            if constexpr (kCare) {
                float z = 0.f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) z += s[t][h][e];
                if (__any_sync(0xffffffffu, isnan(z))) {
                    const Scores<NT> r = scores_of_infinities<D, NT>(sk, q_at, g, c);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[t][h][e] = r.x[t][h][e];
                }
            }
            // scales: K's on the scores; V's relative to the unit that O counts in
            float vs[2][2], shift = 1.f;
            if constexpr (kCodes) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float f = lds_f(ssc + (16 * h + 8 * k + g) * 4);
                        vs[h][k] = lds_f(ssc + (kBlk + 16 * h + 8 * k + g) * 4);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            s[t][h][2 * k] *= f;
                            s[t][h][2 * k + 1] *= f;
                        }
                    }
                uint32_t top = __float_as_uint(lds_f(ssc + (kBlk + lane) * 4)) & 0x7fffffffu;
                if (top >= 0x7f800000u || (edge && !there(lane))) top = 0;
                top = __reduce_max_sync(0xffffffffu, top);
                const int u = max(unit, min((int)(top >> 23) - 126, 126));     // every scale below 2^u
                shift = pow2i(unit - u);
                unit = u;
                const float inv = pow2i(-u);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) vs[h][k] *= inv;
            }
            uint32_t pf[NT][2][2];           // P^T as fragments, 16 keys each
            bool moved = shift != 1.f;
            float grow[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float2 rs = *reinterpret_cast<const float2*>(s_rs + t * 8 + 2 * c);
                if (edge) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int row = t * 8 + 2 * c + k;
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const int j = n * 8 + g, key = key0 + j;
                            const bool seen = sees(row, key) && (has >> (j >> 4) & 1);
                            if (!seen) s[t][n >> 1][(n & 1) * 2 + k] = -INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float f = k ? rs.y : rs.x;
                    float top = fmaxf(fmaxf(s[t][0][k], s[t][0][2 + k]), fmaxf(s[t][1][k], s[t][1][2 + k]));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    const float high = fmaxf(m[t][k], fmaf(top, f, -top_weight<kCodes>()));
                    const float base = high == -INFINITY ? 0.f : high;     // nothing seen yet: weights 2^-inf
                    const float a = ex2f(m[t][k] - base);
                    moved |= high != m[t][k];
                    m[t][k] = high;
                    grow[t][k] = a * shift;
                    float sum = 0.f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        float& x = s[t][n >> 1][(n & 1) * 2 + k];
                        float p = ex2f(fmaf(x, f, -base));
                        sum += p;
                        // a hidden key's scale may be anything
                        if constexpr (kCodes) p = edge && x == -INFINITY ? 0.f : p * vs[n >> 1][n & 1];
                        x = p;
                    }
                    l[t][k] = fmaf(l[t][k], a, sum);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    pf[t][h][0] = transposed(pack2<kCodes>(s[t][h][0], s[t][h][1]));
                    pf[t][h][1] = transposed(pack2<kCodes>(s[t][h][2], s[t][h][3]));
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int n = 0; n < MT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][n][e] *= grow[t][e & 1];
            }
            if constexpr (kCare) set_aside<D>(const_cast<uint8_t*>(sv), key0, has, k_lo, k_hi, sees, live, s_odd, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int b = 0; b < L::NB; ++b) {
                    constexpr int VW = L::CV * L::EB / 4;          // words of the lane's V of a key: 4 or 2
                    uint32_t w[4][VW];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {                  // keys 2c, 2c + 1, 2c + 8, 2c + 9
                        const int row = h * 16 + 2 * c + (k & 1) + (k >> 1) * 8;
                        const uint8_t* const at = sv + b * L::kBox + row * L::RB;
                        if constexpr (VW == 4) lds4(at + (g ^ (row & 7)) * 16, w[k][0], w[k][1], w[k][2], w[k][3]);
                        else lds2(at + g * 8, w[k][0], w[k][1]);
                        if (edge && !there(row))       // whatever lies there: 0 times it must be 0
#pragma unroll
                            for (int e = 0; e < VW; ++e) w[k][e] = 0;
                    }
                    // a[m]: channels 2m (rows g of the tile) and 2m + 1 (rows g + 8) of the lane's, four keys
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        constexpr int kTiles = kCodes ? 2 : 1;     // a word's channels in pairs
                        uint32_t a[kTiles][4];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {              // keys 2c, 2c + 1, then + 8
                            const uint32_t x = w[2 * k][e], y = w[2 * k + 1][e];
                            if constexpr (!kCodes) {
                                a[0][2 * k] = __byte_perm(x, y, 0x5410);
                                a[0][2 * k + 1] = __byte_perm(x, y, 0x7632);
                            } else if (by_masks(true, e)) {
                                const uint32_t ex = even_pair(x), ey = even_pair(y), ox = odd_pair(x), oy = odd_pair(y);
                                a[0][2 * k] = __byte_perm(ex, ey, 0x5410);
                                a[0][2 * k + 1] = __byte_perm(ox, oy, 0x5410);
                                a[kTiles - 1][2 * k] = __byte_perm(ex, ey, 0x7632);
                                a[kTiles - 1][2 * k + 1] = __byte_perm(ox, oy, 0x7632);
                            } else {
                                const uint32_t lo = __byte_perm(x, y, 0x5140), hi = __byte_perm(x, y, 0x7362);
                                a[0][2 * k] = lo_half2(lo);
                                a[0][2 * k + 1] = hi_half2(lo);
                                a[kTiles - 1][2 * k] = lo_half2(hi);
                                a[kTiles - 1][2 * k + 1] = hi_half2(hi);
                            }
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int n = 0; n < kTiles; ++n)
                                mma16816<kCodes>(o[t][b * (L::CV / 2) + kTiles * e + n], a[n], pf[t][h][0], pf[t][h][1]);
                    }
                }
            }
            __syncwarp();                    // every lane has read the stage
            const int next = i + kStages;
            if (next < n_it && (next & 31) == 0) look_up(next);
#pragma unroll
            for (int k = 0; k + 1 < kStages; ++k) loaded[k] = loaded[k + 1];
            loaded[kStages - 1] = next < n_it ? issue(next, stage) : 0u;
            advance();
            if constexpr (!kCodes && !kCare) {
                if ((i & 7) == 7 || i + 1 == n_it) {
                    float z[4] = {};         // zero, or NaN where a sum is not finite
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
#pragma unroll
                        for (int n = 0; n < MT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[e] = fmaf(o[t][n][e], 0.f, z[e]);
                        z[t & 3] = fmaf(l[t][0] + l[t][1], 0.f, z[t & 3]);
                    }
                    if (__any_sync(0xffffffffu, (z[0] + z[1]) + (z[2] + z[3]) != 0.f)) return i + 1;
                }
            }
        }
        return -1;
    };
    const int stopped = blocks(std::false_type{});
    if constexpr (!kCodes)
        if (stopped >= 0) {
            for (int k = min(kStages, n_it - stopped); k > 0; --k) {         // what is on its way lands first
                mbar_wait(smem_u32(&s_full[warp][stage]), parity, P.err, &s_abort);
                advance();
            }
            __syncwarp();
            start();
            look_up(0);
#pragma unroll
            for (int k = 0; k < kStages; ++k) loaded[k] = k < n_it ? issue(k, (stage + k) % kStages) : 0u;
            blocks(std::true_type{});
        }

    // the warps' results join: O in units of one, rows [row][channel], lines of 16 bytes swapped within
    // groups of eight so that lanes meet fewer banks
    if (kCodes && lane == 0) s_unit[warp] = unit;
    __syncthreads();                     // every stage has been read
    // (O is its weights' sum times the output, up to 2^54: of large values in units of 2^lift until it is divided by it)
    int lift = 0;
    if constexpr (kCodes) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) lift = max(lift, s_unit[w] - 40);
    }
    float* const joined = reinterpret_cast<float*>(smem);
    auto line = [](int f) { return f ^ (2 * (f >> 3 & 3)); };
    const float one = kCodes ? pow2i(unit - lift) : 1.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float sum = l[t][k];
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            const int row = t * 8 + 2 * c + k;
            if (g == 0) {
                s_m[warp][row] = m[t][k];
                s_l[warp][row] = sum;
            }
            float* const to = joined + (warp * kRows + row) * L::kPitch;
#pragma unroll
            for (int b = 0; b < L::NB; ++b)
#pragma unroll
                for (int q4 = 0; q4 < L::CV / 4; ++q4) {       // the lane's channels 4 q4 .. + 3 of the box
                    const int n = b * (L::CV / 2) + 2 * q4;
                    const float f = by_masks(kCodes, q4) ? one * 256.f : one;
                    *reinterpret_cast<float4*>(to + line((b * L::BC + g * L::CV) / 4 + q4) * 4) =
                        make_float4(o[t][n][k] * f, o[t][n][2 + k] * f, o[t][n + 1][k] * f, o[t][n + 1][2 + k] * f);
                }
        }
    __syncthreads();
    const bool whole = n_split == 1;
    T* const out = static_cast<T*>(P.out);
    float* const part_o = X.part_o + (int64_t)blockIdx.x * kRows * D;
    float* const part_lse = X.part_lse + (int64_t)blockIdx.x * kRows;
    // row `row`'s four channels from 4 f on, and its log2 normaliser, to where they belong
    auto put = [&](int row, int f, float4 x, float lse2) {
        if (whole) {
            const int64_t tok = R.q0 + (row0 + row) / G;
            const int h = hk * G + (row0 + row) % G;
            *reinterpret_cast<uint2*>(out + (tok * P.hq + h) * D + 4 * f) = make_uint2(pack2<false>(x.x, x.y), pack2<false>(x.z, x.w));
            if (f == 0 && P.lse) P.lse[(int64_t)h * P.n_tokens + tok] = lse2 * 0.69314718055994531f;
        } else {
            *reinterpret_cast<float4*>(part_o + row * D + 4 * f) = x;
            if (f == 0) part_lse[row] = lse2;
        }
    };
    // of a row of no weight; a stretch's is zero, and the others' decide
    auto none = [&](int row) { return whole ? of_no_weight<kTree>(P, R, (int)((row0 + row) / G)) : 0.f; };
    for (int i = threadIdx.x; i < live * (D / 4); i += kWarps * 32) {
        const int row = i / (D / 4), f = i % (D / 4);
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][row]);
        const float base = top == -INFINITY ? 0.f : top;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float a = ex2f(s_m[w][row] - base);
            sum = fmaf(s_l[w][row], a, sum);
            const float4 y = *reinterpret_cast<const float4*>(joined + (w * kRows + row) * L::kPitch + line(f) * 4);
            x.x = fmaf(y.x, a, x.x);
            x.y = fmaf(y.y, a, x.y);
            x.z = fmaf(y.z, a, x.z);
            x.w = fmaf(y.w, a, x.w);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (sum == 0.f) x.x = x.y = x.z = x.w = none(row);
        else x = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        if constexpr (kCodes) {
            const float up = pow2i(lift);
            x = make_float4(x.x * up, x.y * up, x.z * up, x.w * up);
        }
        if constexpr (!kCodes) {         // values that are not finite, of keys that the row sees
            const uint32_t odd = s_odd[row * (D / 4) + f];
            if (odd != 0u && sum < INFINITY) {
                auto take_in = [&](float& y, uint32_t is) {
                    if (is != 0u) y = is == 1u ? INFINITY : is == 2u ? -INFINITY : __uint_as_float(0x7fc00000u);
                };
                take_in(x.x, odd & 7u);
                take_in(x.y, odd >> 8 & 7u);
                take_in(x.z, odd >> 16 & 7u);
                take_in(x.w, odd >> 24 & 7u);
            }
        }
        put(row, f, x, sum == 0.f ? -INFINITY : top + log2f(sum));
    }
    if (whole) return;
    // the stretch that ends last joins them all: every partial is visible before its ticket is taken
    const int unit_id = R.unit0 + hk * (int)n_tiles + (int)rt;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();                 // (cumulative: of what the CTA's threads wrote before the barrier)
        const uint32_t t = atomicAdd(X.tickets + unit_id, 1u);
        s_last = t == n_split - 1;
        if (s_last) X.tickets[unit_id] = 0;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    // items of this unit's stretches, `step` apart; a thread's sixteen at a time on their way at once
    const int64_t step = (int64_t)P.hkv * n_tiles, item0 = R.item0 + (int64_t)hk * n_tiles + rt;
    for (int i = threadIdx.x; i < live * (D / 4); i += kWarps * 32) {
        const int row = i / (D / 4), f = i % (D / 4);
        const float* const from = X.part_o + (item0 * kRows + row) * D + 4 * f;
        const float* const from_lse = X.part_lse + item0 * kRows + row;
        float top = -INFINITY, sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kBatch = 16;
        constexpr float kLow = 1.f / kMaxStretches;      // (of values near the largest no sum overflows; a power of two changes nothing else)
        for (int k0 = 0; k0 < (int)n_split; k0 += kBatch) {
            float e[kBatch];
            float4 y[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (k0 + k >= (int)n_split) {
                    e[k] = -INFINITY;
                    y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    continue;
                }
                e[k] = __ldcg(from_lse + (k0 + k) * step * kRows);
                y[k] = __ldcg(reinterpret_cast<const float4*>(from + (k0 + k) * step * kRows * D));
            }
            float now = top;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) now = fmaxf(now, e[k]);
            const float base = now == -INFINITY ? 0.f : now, a = ex2f(top - base);
            top = now;
            sum *= a;
            x = make_float4(x.x * a, x.y * a, x.z * a, x.w * a);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const float w = ex2f(e[k] - base) * kLow;
                sum += w;
                x.x = fmaf(y[k].x, w, x.x);
                x.y = fmaf(y[k].y, w, x.y);
                x.z = fmaf(y[k].z, w, x.z);
                x.w = fmaf(y[k].w, w, x.w);
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (sum == 0.f) x.x = of_no_weight<kTree>(P, R, (int)((row0 + row) / G)), x.y = x.z = x.w = x.x;
        const uint32_t tok = (row0 + row) / G, h = hk * G + row0 + row - tok * G;
        *reinterpret_cast<uint2*>(out + ((int64_t)(R.q0 + tok) * P.hq + h) * D + 4 * f) =
            make_uint2(pack2<false>(x.x * inv, x.y * inv), pack2<false>(x.z * inv, x.w * inv));
        if (f == 0 && P.lse) P.lse[(int64_t)h * P.n_tokens + R.q0 + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum / kLow)) * 0.69314718055994531f;
    }
}

// ------------------------------------------------------------------ host side

template <int D, bool kCodes, int NT, int kReq, bool kTree>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    using L = Lay<D, kCodes, NT>;
    constexpr int kRows = 8 * NT;
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_mma_kernel<D, kCodes, NT, kReq, kTree>;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, L::kSmem);
    if (e != cudaSuccess) return e;
    for (int b0 = 0; b0 < n; b0 += kReq) {
        const int nb = std::min(n - b0, kReq);
        MmaLaunch<kReq> X;
        fill_paged(X.a, c, D, req + b0, nb);
        // Stretches: as many blocks each as make one wave of CTAs of all of them, but at least one for
        // each warp (one token over 500 rows: 8.3 us, with two each 9.4).
        const int slots = device_sms() * L::kCtas, G = c.hq / c.hkv;
        auto blocks_of = [&](const PagedReq& q) {
            const int64_t keys = c.window ? std::min<int64_t>(q.n_keys, (int64_t)c.window + q.nq + kBlk) : q.n_keys;
            return (int)((keys + kBlk - 1) / kBlk);
        };
        auto tiles_of = [&](const PagedReq& q) { return (q.nq * G + kRows - 1) / kRows; };
        auto splits_of = [&](const PagedReq& q, int per) {
            return std::max(1, std::min((blocks_of(q) + per - 1) / per, kMaxStretches));
        };
        int64_t total = 0;
        for (int i = 0; i < nb; ++i) total += (int64_t)blocks_of(X.a.req[i]) * tiles_of(X.a.req[i]) * c.hkv;
        int per = (int)std::max<int64_t>(kWarps, (total + slots - 1) / slots);
        for (int tries = 0; tries < 64; ++tries) {
            int64_t items = 0;
            for (int i = 0; i < nb; ++i) items += (int64_t)splits_of(X.a.req[i], per) * tiles_of(X.a.req[i]) * c.hkv;
            if (items <= slots) break;
            const int more = std::max(per + 1, (int)((int64_t)per * 33 / 32));
            bool any = false;
            for (int i = 0; i < nb; ++i) any = any || splits_of(X.a.req[i], per) > 1;
            if (!any) break;
            per = more;
        }
        int64_t items = 0, units = 0;
        bool split = false;
        auto lay_out = [&](bool cut) {
            items = units = 0;
            split = false;
            for (int i = 0; i < nb; ++i) {
                PagedReq& q = X.a.req[i];
                q.splits = cut ? splits_of(q, per) : 1;
                split = split || q.splits > 1;
                q.item0 = (int32_t)items;
                q.unit0 = (int32_t)units;
                q.tiles = tiles_of(q);
                units += (int64_t)q.tiles * c.hkv;
                items += (int64_t)q.tiles * c.hkv * q.splits;
            }
        };
        lay_out(true);
        X.box_rows = std::min(1 << c.pg.page_shift, kBlk);
        X.part_o = X.part_lse = nullptr;
        X.tickets = nullptr;
        std::optional<Workspace> work;
        if (split) {
            const size_t o_bytes = (size_t)items * kRows * D * 4;
            work.emplace(c.ctx, o_bytes + (size_t)items * kRows * 4, (size_t)units);
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
        const auto swizzle = L::RB == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE;
        if (!encode_page_map(&X.tm_k, c.pg.k, c.pg, c.hkv, D, kCodes, L::BC, X.box_rows, swizzle) ||
            !encode_page_map(&X.tm_v, c.pg.v, c.pg, c.hkv, D, kCodes, L::BC, X.box_rows, swizzle))
            return cudaErrorInvalidValue;
        e = launch_overlapped(kernel, (unsigned)items, kWarps * 32, L::kSmem, s, X);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// As few row tiles as hold the largest request's rows, and as few eights of rows a tile as make them up:
// a tile's keys are loaded and converted once for all its rows.
template <int D, bool kCodes, bool kTree>
cudaError_t by_rows(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    int rows = 1;
    for (int i = 0; i < n; ++i) rows = std::max(rows, req[i].nq * (c.hq / c.hkv));
    const int hold = c.eights ? c.eights : kMostEights;
    const int eights = (rows + 7) / 8, tiles = (eights + hold - 1) / hold, nt = (eights + tiles - 1) / tiles;
    // (trees have kernels of the small block alone: a launch for every 32 requests)
    const bool small = kTree || n <= kPagedFew;
    constexpr int kLarge = kTree ? kPagedFew : kPagedMany;
    if (nt == 1) return small ? launch<D, kCodes, 1, kPagedFew, kTree>(c, req, n, s) : launch<D, kCodes, 1, kLarge, kTree>(c, req, n, s);
    if (nt == 2) return small ? launch<D, kCodes, 2, kPagedFew, kTree>(c, req, n, s) : launch<D, kCodes, 2, kLarge, kTree>(c, req, n, s);
    if (nt == 3) return launch<D, kCodes, 3, kPagedFew, kTree>(c, req, n, s);
    return launch<D, kCodes, 4, kPagedFew, kTree>(c, req, n, s);
}

template <bool kTree>
cudaError_t by_kind(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? by_rows<128, true, kTree>(c, req, n, s) : by_rows<128, false, kTree>(c, req, n, s);
    return codes ? by_rows<64, true, kTree>(c, req, n, s) : by_rows<64, false, kTree>(c, req, n, s);
}

}  // namespace

// This file is compiled twice: trees of tokens are paged_mma_tree.cu's.
#ifndef C2KV_TREES

bool encode_page_map(CUtensorMap* tm, const void* base, const PageView& pg, int hkv, int d, bool codes, int box_channels, int box_rows,
              CUtensorMapSwizzle swizzle) {
    const cuuint64_t eb = codes ? 1 : 2, rows = 1ull << pg.page_shift;
    const cuuint64_t dims[4] = {(cuuint64_t)d, rows, (cuuint64_t)hkv, (cuuint64_t)pg.n_pages};
    const cuuint64_t strides[3] = {d * eb, rows * d * eb, (cuuint64_t)pg.page_stride * eb};
    const cuuint32_t box[4] = {(cuuint32_t)box_channels, (cuuint32_t)box_rows, 1, 1};
    return encode_tensor_map(tm, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides,
                             box, swizzle);
}

cudaError_t launch_paged_mma(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return c.parent ? launch_paged_mma_tree(c, req, n, d, codes, s) : by_kind<false>(c, req, n, d, codes, s);
}

#else

cudaError_t launch_paged_mma_tree(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return by_kind<true>(c, req, n, d, codes, s);
}

template <int D, bool kCodes>
int ctas_of(int eights) {
    return eights == 1 ? Lay<D, kCodes, 1>::kCtas : eights == 2 ? Lay<D, kCodes, 2>::kCtas : Lay<D, kCodes, kMostEights>::kCtas;
}

int paged_mma_tree_ctas(int d, bool codes, int eights) {
    if (d == 128) return codes ? ctas_of<128, true>(eights) : ctas_of<128, false>(eights);
    return codes ? ctas_of<64, true>(eights) : ctas_of<64, false>(eights);
}

#endif

}  // namespace c2kv
