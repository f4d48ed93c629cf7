// Paged attention of few query rows: one to a few tokens of each request (c2kv_paged_attend).
//
// The rows of a (request, KV head) -- its tokens times the group's heads -- meet every key once, so
// the call is bound by reading the pages.  One CTA takes 16 * MT rows and a stretch of keys, dealt to
// its four warps in blocks of 32.  Each warp runs alone: a ring of TMA stages of its own, S = Q.K^T and
// P.V on mma.sync (16 rows fill its M; a tcgen05 tile of 128 rows would be mostly empty, and would need
// the 8-bit codes converted through shared memory instead of in registers), its own running maximum and
// sum.  The warps' results join in shared memory, the stretches' in the CTA that ends last.
//
// E4M3 codes become f16 in registers (exact); their scales stay in fp32: a key's K scale multiplies its
// column of S, its V scale its column of P.  P must fit f16, so V scales are taken relative to a power
// of two, the largest of them so far, that O is counted in; it moves like the running maximum does.
// Queries are f16 too, each row scaled by a power of two so that its largest value is near 2^14: their
// rounding is 2^-12 of a value.  Over 16-bit pages queries and weights are bf16.
//
// Operand layouts.  The contraction over channels does not care for their order, so a lane of B takes
// the channels that lie next to one another in its row: 16-byte shared loads, conflict-free under the
// 128-byte swizzle, with no transpose of V (a lane loads the same channels of four keys and pairs them).
#include "paged.cuh"
#include "paged_row.cuh"
#include "per_device.cuh"
#include "ptx.cuh"

#include <algorithm>
#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int kWarps = 4;
constexpr int kBlk = 32;                 // keys of a warp's block
constexpr int kStages = 3;               // blocks in flight a warp

template <int D, bool kCodes>
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
    static constexpr int kStage = 2 * kSide;
    static constexpr int kScales = kCodes ? 2 * kBlk * 4 : 0;      // bytes of a block's scales
    static constexpr int kRing = kWarps * kStages * kStage;
    static constexpr int kSmem = 1024 /*align*/ + kRing + kWarps * kStages * kScales;
    static constexpr int kCtas = kSmem <= 108 * 1024 ? 2 : 1;      // an SM
    static constexpr int kPitch = D + 4;               // floats between rows of the joined results
};
static_assert(Lay<128, false>::kSmem + 12 * 1024 <= 227 * 1024, "shared memory of a CTA");

constexpr int kMaxStretches = 128;       // of one unit's keys: their weights join in shared memory

template <int kReq>
struct MmaLaunch {
    CUtensorMap tm_k, tm_v;              // [n_pages][Hkv][page_size][d], boxes of min(page_size, 32) rows
    int32_t box_rows;
    float* part_o;                       // [item][16 * MT][D] normalised
    float* part_lse;                     // [item][16 * MT] log2 domain
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

__device__ __forceinline__ void lds4(uint32_t a, uint32_t& x, uint32_t& y, uint32_t& z, uint32_t& w) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x), "=r"(y), "=r"(z), "=r"(w) : "r"(a) : "memory");
}
__device__ __forceinline__ void lds2(uint32_t a, uint32_t& x, uint32_t& y) {
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory");
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float lds_f(uint32_t a) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// Where channel pair (ch, ch + 1) of tile row `row` lies in the fragments of Q: word of lane, register.
template <int D, bool kCodes>
__device__ __forceinline__ int q_word(int row, int ch) {
    using L = Lay<D, kCodes>;
    const int box = ch / L::BC, in = ch % L::BC, c = in / L::CQ, s = box * (L::CQ / 4) + in % L::CQ / 4;
    const int reg = (in % 4 / 2) * 2 + (row % 16) / 8;
    return ((row / 16 * L::KS + s) * 32 + (row % 8) * 4 + c) * 4 + reg;
}

template <int D, bool kCodes, int MT, int kReq>
__global__ void __launch_bounds__(kWarps * 32, 2) paged_mma_kernel(const __grid_constant__ MmaLaunch<kReq> X) {
    using L = Lay<D, kCodes>;
    using T = __nv_bfloat16;
    constexpr int kRows = 16 * MT;
    const PagedAttn<kReq>& P = X.a;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kStages];
    __shared__ __align__(16) uint32_t s_q[MT * L::KS * 32 * 4];
    __shared__ float s_rs[kRows], s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ uint32_t s_abort, s_bad, s_last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
    uint8_t* const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);

    // the work item: (request, stretch, KV head, row tile)
    int r = 0;
    for (int hi = P.batch; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.req[mid].item0 <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    const PagedReq R = P.req[r];
    const int G = P.hq / P.hkv, n_rows = R.nq * G, n_tiles = (n_rows + kRows - 1) / kRows;
    int it = blockIdx.x - R.item0;
    const int rt = it % n_tiles;
    it /= n_tiles;
    const int hk = it % P.hkv, sp = it / P.hkv, n_split = R.splits;
    const int row0 = rt * kRows, live = min(kRows, n_rows - row0);
    // keys that any row of the tile sees: [k_lo, k_hi); the first row sees up to `first`
    const int first = R.n_keys - R.nq + row0 / G, k_hi = R.n_keys - R.nq + (row0 + live - 1) / G + 1;
    const int k_lo = P.window ? max(0, first - P.window + 1) : 0;
    const int b_lo = k_lo / kBlk, b_n = max(0, (k_hi + kBlk - 1) / kBlk - b_lo);
    const int b0 = b_lo + (int)((int64_t)b_n * sp / n_split), b1 = b_lo + (int)((int64_t)b_n * (sp + 1) / n_split);
    const int n_it = b1 - b0 > warp ? (b1 - b0 - warp + kWarps - 1) / kWarps : 0;

    if (threadIdx.x == 0) {
        s_abort = s_bad = 0;
        for (int w = 0; w < kWarps; ++w)
            for (int s = 0; s < kStages; ++s) mbar_init(smem_u32(&s_full[w][s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    const uint32_t ring = smem_u32(smem) + warp * kStages * L::kStage;
    const uint32_t scales = smem_u32(smem) + L::kRing + warp * kStages * L::kScales;
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
        if (one) pages0 = __ldg(table + (key >> P.pg.page_shift));
        if (two) pages1 = __ldg(table + ((key + 16) >> P.pg.page_shift));
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
        if (lane == 0) {
            const uint32_t bar = smem_u32(&s_full[warp][stage]), dst = ring + stage * L::kStage, ssc = scales + stage * L::kScales;
            const int off = ((b0 + warp + i * kWarps) * kBlk) & ((1 << P.pg.page_shift) - 1);
            const int n = (p0 >= 0) + (p1 >= 0);
            mbar_expect_tx(bar, n * box_rows * (2 * D * L::EB + (kCodes ? 8 : 0)));
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
                if constexpr (kCodes) {
                    const int64_t at = (int64_t)page * P.pg.scale_stride + ((int64_t)hk << P.pg.page_shift) + at_row;
                    bulk_load(ssc + k * 16 * 4, P.pg.k_scale + at, box_rows * 4, bar);
                    bulk_load(ssc + (kBlk + k * 16) * 4, P.pg.v_scale + at, box_rows * 4, bar);
                }
            }
        }
        return boxes == 1 ? (p0 >= 0 ? 3u : 0u) : (p0 >= 0 ? 1u : 0u) | (p1 >= 0 ? 2u : 0u);
    };
    look_up(0);
    uint32_t loaded[kStages];            // of the blocks in flight, the next one to be used first
#pragma unroll
    for (int i = 0; i < kStages; ++i) loaded[i] = i < n_it ? issue(i, i) : 0;

    // the tile's queries: turned, as fragments of A
    uint64_t turn[D / 64] = {};
    if (P.turn) {
#pragma unroll
        for (int e = 0; e < D / 64; ++e) turn[e] = lane_turn(P.rope.turn, lane * (D / 64) + e);
    }
    for (int row = warp; row < kRows; row += kWarps) {
        float x[D / 32];                 // channels 2 lane (+ 1) of the lower half, and of the upper
        const bool there = row < live;
        const int tok = R.q0 + (row0 + row) / G, h = hk * G + (row0 + row) % G;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) x[e] = 0.f;
        constexpr int C = D / 64;        // channels of each half a lane
        if (there) {
            const T* q = static_cast<const T*>(P.q) + (int64_t)tok * P.q_stride + (int64_t)h * D + lane * C;
#pragma unroll
            for (int e = 0; e < C; ++e) {
                x[e] = static_cast<float>(q[e]);
                x[C + e] = static_cast<float>(q[D / 2 + e]);
            }
            if (P.turn) {
                const int64_t pos = __ldg(P.turn + tok);
#pragma unroll
                for (int e = 0; e < C; ++e) {
                    float a, b;
                    rotate1(x[e], x[C + e], turn_cs_fast(turn[e], pos), a, b);
                    x[e] = a;
                    x[C + e] = b;
                }
            }
        }
        float back = 1.f;
        if constexpr (kCodes) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            top = __reduce_max_sync(0xffffffffu, top);
            // largest value to [2^14, 2^15); zero and non-finite rows as they are
            const int ex = (int)(top >> 23) - 127;
            if (top != 0 && top < 0x7f800000u && ex > -100) {
                const float f = exp2f((float)(14 - ex));
                back = exp2f((float)(ex - 14));
#pragma unroll
                for (int e = 0; e < D / 32; ++e) x[e] *= f;
            }
        }
        if (lane == 0) s_rs[row] = back * P.scale_log2;
        if constexpr (C == 2) {
            s_q[q_word<D, kCodes>(row, 2 * lane)] = pack2<kCodes>(x[0], x[1]);
            s_q[q_word<D, kCodes>(row, D / 2 + 2 * lane)] = pack2<kCodes>(x[2], x[3]);
        } else {                         // one channel of each half a lane: pairs from even lanes
            const float y0 = __shfl_down_sync(0xffffffffu, x[0], 1), y1 = __shfl_down_sync(0xffffffffu, x[1], 1);
            if (!(lane & 1)) {
                s_q[q_word<D, kCodes>(row, lane)] = pack2<kCodes>(x[0], y0);
                s_q[q_word<D, kCodes>(row, D / 2 + lane)] = pack2<kCodes>(x[1], y1);
            }
        }
    }
    __syncthreads();

    float o[MT][D / 8][4], m[MT][2], l[MT][2], rs[MT][2];
    int last_key[MT][2];                 // the last key that rows g and g + 8 of each 16 see
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][n][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            m[t][e] = -INFINITY;
            l[t][e] = 0.f;
            rs[t][e] = s_rs[t * 16 + e * 8 + g];
            last_key[t][e] = R.n_keys - R.nq + (row0 + t * 16 + e * 8 + g) / G;
        }
    }
    int unit = -127;                     // O counts in 2^unit (E4M3)
    uint32_t qf[MT == 1 ? L::KS : 1][4];
    if constexpr (MT == 1) {
#pragma unroll
        for (int s = 0; s < L::KS; ++s) lds4(smem_u32(s_q) + (s * 32 + lane) * 16, qf[s][0], qf[s][1], qf[s][2], qf[s][3]);
    }

    int stage = 0, parity = 0;
    for (int i = 0; i < n_it; ++i) {
        const int key0 = (b0 + warp + i * kWarps) * kBlk;
        const uint32_t sk = ring + stage * L::kStage, sv = sk + L::kSide, ssc = scales + stage * L::kScales;
        const uint32_t has = loaded[0];
        // some key is hidden from some row, or was not loaded: then every key is asked
        const bool edge = has != 3 || key0 + kBlk - 1 > first || (P.window && key0 <= k_hi - 1 - P.window);
        // key j of the block is there, and some row of the tile sees it
        auto there = [&](int j) { return key0 + j < k_hi && key0 + j >= k_lo && (has >> (j >> 4) & 1); };
        mbar_wait(smem_u32(&s_full[warp][stage]), parity, P.err, &s_abort);

        float s[MT][4][4];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][n][e] = 0.f;
#pragma unroll
        for (int b = 0; b < L::NB; ++b) {
            constexpr int KW = L::CQ * L::EB / 4;              // words of the lane's channels of a key
            uint32_t w[4][KW];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const uint32_t at = sk + b * L::kBox + (n * 8 + g) * L::RB;
#pragma unroll
                for (int u = 0; u < KW / 4; ++u)
                    lds4(at + (L::RB == 128 ? ((2 * c + u) ^ g) * 16 : c * 16), w[n][4 * u], w[n][4 * u + 1], w[n][4 * u + 2], w[n][4 * u + 3]);
            }
#pragma unroll
            for (int ks = 0; ks < L::CQ / 4; ++ks) {
                uint32_t f[4][2];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    f[n][0] = kCodes ? lo_half2(w[n][ks]) : w[n][(2 * ks) % KW];
                    f[n][1] = kCodes ? hi_half2(w[n][ks]) : w[n][(2 * ks + 1) % KW];
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    uint32_t a[4];
                    if constexpr (MT == 1) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = qf[b * (L::CQ / 4) + ks][e];
                    } else {
                        lds4(smem_u32(s_q) + ((t * L::KS + b * (L::CQ / 4) + ks) * 32 + lane) * 16, a[0], a[1], a[2], a[3]);
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n) mma16816<kCodes>(s[t][n], a, f[n][0], f[n][1]);
                }
            }
        }
        // scales: K's on the scores; V's relative to the unit that O counts in
        float vs[4][2], shift = 1.f;
        if constexpr (kCodes) {
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float2 a = lds_f2(ssc + (n * 8 + 2 * c) * 4), b = lds_f2(ssc + (kBlk + n * 8 + 2 * c) * 4);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    s[t][n][0] *= a.x;
                    s[t][n][1] *= a.y;
                    s[t][n][2] *= a.x;
                    s[t][n][3] *= a.y;
                }
                vs[n][0] = b.x;
                vs[n][1] = b.y;
            }
            uint32_t top = __float_as_uint(lds_f(ssc + (kBlk + lane) * 4)) & 0x7fffffffu;
            if (top >= 0x7f800000u || (edge && !there(lane))) top = 0;
            top = __reduce_max_sync(0xffffffffu, top);
            const int u = max(unit, min((int)(top >> 23) - 126, 126));     // every scale below 2^u
            shift = unit == u ? 1.f : exp2f((float)max(unit - u, -250));
            unit = u;
            const float inv = exp2f((float)-u);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                vs[n][0] *= inv;
                vs[n][1] *= inv;
            }
        }
        uint32_t pf[MT][2][4];           // P as fragments of A, 16 keys each
        float grow[MT][2];
        bool moved = shift != 1.f;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (edge) {
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = n * 8 + 2 * c + (e & 1), key = key0 + j, end = last_key[t][e >> 1];
                        const bool seen = key <= end && (!P.window || key > end - P.window) && (has >> (j >> 4) & 1);
                        if (!seen) s[t][n][e] = -INFINITY;
                    }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = -INFINITY;
#pragma unroll
                for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(s[t][n][2 * e], s[t][n][2 * e + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const float now = fmaxf(m[t][e], top * rs[t][e]);
                const float base = now == -INFINITY ? 0.f : now;       // nothing seen yet: weights 2^-inf
                const float f = ex2f(m[t][e] - base);
                moved |= now != m[t][e];
                m[t][e] = now;
                grow[t][e] = f * shift;
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < 4; ++n) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float p = ex2f(fmaf(s[t][n][2 * e + k], rs[t][e], -base));
                        sum += p;
                        // a hidden key's scale may be anything
                        if constexpr (kCodes) p = edge && s[t][n][2 * e + k] == -INFINITY ? 0.f : p * vs[n][k];
                        s[t][n][2 * e + k] = p;
                    }
                }
                l[t][e] = fmaf(l[t][e], f, sum);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    pf[t][h][e] = pack2<kCodes>(s[t][2 * h][2 * e], s[t][2 * h][2 * e + 1]);
                    pf[t][h][2 + e] = pack2<kCodes>(s[t][2 * h + 1][2 * e], s[t][2 * h + 1][2 * e + 1]);
                }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int n = 0; n < D / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][n][e] *= grow[t][e >> 1];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int b = 0; b < L::NB; ++b) {
                constexpr int VW = L::CV * L::EB / 4;          // words of the lane's V of a key: 4 or 2
                uint32_t w[4][VW];
#pragma unroll
                for (int k = 0; k < 4; ++k) {                  // keys 2c, 2c + 1, 2c + 8, 2c + 9
                    const int row = h * 16 + 2 * c + (k & 1) + (k >> 1) * 8;
                    const uint32_t at = sv + b * L::kBox + row * L::RB;
                    if constexpr (VW == 4) lds4(at + (g ^ (row & 7)) * 16, w[k][0], w[k][1], w[k][2], w[k][3]);
                    else lds2(at + g * 8, w[k][0], w[k][1]);
                    if (edge && !there(row))       // whatever lies there: 0 times it must be 0
#pragma unroll
                        for (int e = 0; e < VW; ++e) w[k][e] = 0;
                }
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    if constexpr (kCodes) {
                        const uint32_t x0 = __byte_perm(w[0][e], w[1][e], 0x5140), x1 = __byte_perm(w[0][e], w[1][e], 0x7362);
                        const uint32_t y0 = __byte_perm(w[2][e], w[3][e], 0x5140), y1 = __byte_perm(w[2][e], w[3][e], 0x7362);
                        const uint32_t f[4] = {lo_half2(x0), hi_half2(x0), lo_half2(x1), hi_half2(x1)};
                        const uint32_t h2[4] = {lo_half2(y0), hi_half2(y0), lo_half2(y1), hi_half2(y1)};
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int k = 0; k < 4; ++k) mma16816<kCodes>(o[t][4 * e + k], pf[t][h], f[k], h2[k]);
                    } else {
                        const uint32_t f[2] = {__byte_perm(w[0][e], w[1][e], 0x5410), __byte_perm(w[0][e], w[1][e], 0x7632)};
                        const uint32_t h2[2] = {__byte_perm(w[2][e], w[3][e], 0x5410), __byte_perm(w[2][e], w[3][e], 0x7632)};
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int k = 0; k < 2; ++k) mma16816<kCodes>(o[t][b * L::CV + 2 * e + k], pf[t][h], f[k], h2[k]);
                    }
                }
            }
        }
        __syncwarp();                    // every lane has read the stage
        const int next = i + kStages;
        if (next < n_it && (next & 31) == 0) look_up(next);
#pragma unroll
        for (int k = 0; k + 1 < kStages; ++k) loaded[k] = loaded[k + 1];
        loaded[kStages - 1] = next < n_it ? issue(next, stage) : 0;
        if (++stage == kStages) {
            stage = 0;
            parity ^= 1;
        }
    }

    // the warps' results join: O in units of one, rows [row][channel], lines of 16 bytes swapped within
    // groups of eight so that the four lanes of a row meet different banks
    __syncthreads();                     // every stage has been read
    float* const joined = reinterpret_cast<float*>(smem);
    auto line = [](int f) { return f ^ (2 * (f >> 3 & 3)); };
    const float one = kCodes ? exp2f((float)unit) : 1.f;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[t][e];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            const int row = t * 16 + e * 8 + g;
            if (c == 0) {
                s_m[warp][row] = m[t][e];
                s_l[warp][row] = sum;
            }
            float* const to = joined + (warp * kRows + row) * L::kPitch;
#pragma unroll
            for (int b = 0; b < L::NB; ++b)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int q4 = 0; q4 < L::CV / 4; ++q4) {
                        const int n = b * L::CV + 4 * q4;
                        const int f = (b * L::BC + (2 * c + k) * L::CV) / 4 + q4;
                        *reinterpret_cast<float4*>(to + line(f) * 4) =
                            make_float4(o[t][n][2 * e + k] * one, o[t][n + 1][2 * e + k] * one, o[t][n + 2][2 * e + k] * one,
                                        o[t][n + 3][2 * e + k] * one);
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
        if constexpr (!kCodes)           // infinity or NaN in V may belong to keys that this row does not see
            if (!(fabsf(x.x) <= 3.0e38f && fabsf(x.y) <= 3.0e38f && fabsf(x.z) <= 3.0e38f && fabsf(x.w) <= 3.0e38f))
                atomicOr(&s_bad, 1u << row);
        put(row, f, sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv),
            sum == 0.f ? -INFINITY : top + log2f(sum));
    }
    if constexpr (!kCodes) {
        __syncthreads();
        for (uint32_t bad = s_bad; bad; bad &= bad - 1) {      // those rows again, key by key
            const int row = __ffs(bad) - 1;
            if (row % kWarps != warp) continue;
            const int end = R.n_keys - R.nq + (row0 + row) / G;
            const int lo = max(b0 * kBlk, P.window ? end - P.window + 1 : 0), hi = min(b1 * kBlk, end + 1);
            float q[D / 32], x[D / 32], rm, rl;
            lane_query<T, D>(P, R.q0 + (row0 + row) / G, hk * G + (row0 + row) % G, lane, q);
            row_attend<T, D, kCodes>(P, q, R.row, hk, lo, hi, 1, lane, rm, rl, x);
            const float inv = rl == 0.f ? 0.f : 1.f / rl;
            float4 y = make_float4(x[0] * inv, x[1] * inv, 0.f, 0.f);
            if constexpr (D == 128) {
                y.z = x[2] * inv;
                y.w = x[3] * inv;
                put(row, lane, y, rl == 0.f ? -INFINITY : rm + log2f(rl));
            } else {
                const float z = __shfl_down_sync(0xffffffffu, y.x, 1), w = __shfl_down_sync(0xffffffffu, y.y, 1);
                if (!(lane & 1)) put(row, lane / 2, make_float4(y.x, y.y, z, w), rl == 0.f ? -INFINITY : rm + log2f(rl));
            }
        }
    }
    if (whole) return;
    // the stretch that ends last joins them all: every partial is visible before its ticket is taken
    const int unit_id = R.unit0 + hk * n_tiles + rt;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t t = atomicAdd(X.tickets + unit_id, 1u);
        s_last = t == (uint32_t)n_split - 1;
        if (s_last) X.tickets[unit_id] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    const int64_t step = (int64_t)P.hkv * n_tiles, item0 = R.item0 + (int64_t)hk * n_tiles + rt;   // items of this unit
    float* const weight = joined;        // [stretch][row]
    for (int i = threadIdx.x; i < n_split * live; i += kWarps * 32) {
        const int k = i / live, row = i % live;
        weight[k * kRows + row] = __ldcg(X.part_lse + (item0 + k * step) * kRows + row);
    }
    __syncthreads();
    if (threadIdx.x < live) {
        const int row = threadIdx.x;
        float top = -INFINITY, sum = 0.f;
        for (int k = 0; k < n_split; ++k) top = fmaxf(top, weight[k * kRows + row]);
        const float base = top == -INFINITY ? 0.f : top;
        for (int k = 0; k < n_split; ++k) sum += ex2f(weight[k * kRows + row] - base);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        for (int k = 0; k < n_split; ++k) weight[k * kRows + row] = ex2f(weight[k * kRows + row] - base) * inv;
        if (P.lse) {
            const int64_t tok = R.q0 + (row0 + row) / G;
            P.lse[(int64_t)(hk * G + (row0 + row) % G) * P.n_tokens + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < live * (D / 4); i += kWarps * 32) {
        const int row = i / (D / 4), f = i % (D / 4);
        const float* from = X.part_o + (item0 * kRows + row) * D + 4 * f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < n_split; ++k) {
            const float a = weight[k * kRows + row];
            const float4 y = __ldcg(reinterpret_cast<const float4*>(from + k * step * kRows * D));
            x.x = fmaf(y.x, a, x.x);
            x.y = fmaf(y.y, a, x.y);
            x.z = fmaf(y.z, a, x.z);
            x.w = fmaf(y.w, a, x.w);
        }
        const int64_t tok = R.q0 + (row0 + row) / G;
        *reinterpret_cast<uint2*>(out + (tok * P.hq + hk * G + (row0 + row) % G) * D + 4 * f) =
            make_uint2(pack2<false>(x.x, x.y), pack2<false>(x.z, x.w));
    }
}

// ------------------------------------------------------------------ host side

template <int D, bool kCodes, int MT, int kReq>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    using L = Lay<D, kCodes>;
    constexpr int kRows = 16 * MT;
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_mma_kernel<D, kCodes, MT, kReq>;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, L::kSmem);
    if (e != cudaSuccess) return e;
    for (int b0 = 0; b0 < n; b0 += kReq) {
        const int nb = std::min(n - b0, kReq);
        MmaLaunch<kReq> X;
        fill_paged(X.a, c, D, req + b0, nb);
        // Stretches: as many blocks each as make one wave of CTAs of all of them, but at least two
        // rounds of the four warps.
        const int slots = device_sms() * L::kCtas, G = c.hq / c.hkv;
        auto blocks_of = [&](const PagedReq& q) {
            const int keys = c.window ? std::min(q.n_keys, c.window + q.nq + kBlk) : q.n_keys;
            return (keys + kBlk - 1) / kBlk;
        };
        auto tiles_of = [&](const PagedReq& q) { return (q.nq * G + kRows - 1) / kRows; };
        auto splits_of = [&](const PagedReq& q, int per) {
            return std::max(1, std::min((blocks_of(q) + per - 1) / per, kMaxStretches));
        };
        int64_t total = 0;
        for (int i = 0; i < nb; ++i) total += (int64_t)blocks_of(X.a.req[i]) * tiles_of(X.a.req[i]) * c.hkv;
        int per = (int)std::max<int64_t>(2 * kWarps, (total + slots - 1) / slots);
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
        for (int i = 0; i < nb; ++i) {
            PagedReq& q = X.a.req[i];
            q.splits = splits_of(q, per);
            split = split || q.splits > 1;
            q.item0 = (int32_t)items;
            q.unit0 = (int32_t)units;
            units += (int64_t)tiles_of(q) * c.hkv;
            items += (int64_t)tiles_of(q) * c.hkv * q.splits;
        }
        X.box_rows = std::min(1 << c.pg.page_shift, kBlk);
        X.part_o = X.part_lse = nullptr;
        X.tickets = nullptr;
        if (split) {
            void* p = nullptr;
            const size_t o_bytes = (size_t)items * kRows * D * 4;
            e = context_workspace(c.ctx, o_bytes + (size_t)items * kRows * 4, (size_t)units, &p, &X.tickets);
            if (e != cudaSuccess) return e;
            X.part_o = static_cast<float*>(p);
            X.part_lse = reinterpret_cast<float*>(static_cast<char*>(p) + o_bytes);
        }
        const auto swizzle = L::RB == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE;
        if (!encode_page_map(&X.tm_k, c.pg.k, c.pg, c.hkv, D, kCodes, L::BC, X.box_rows, swizzle) ||
            !encode_page_map(&X.tm_v, c.pg.v, c.pg, c.hkv, D, kCodes, L::BC, X.box_rows, swizzle))
            return cudaErrorInvalidValue;
        kernel<<<(unsigned)items, kWarps * 32, L::kSmem, s>>>(X);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool kCodes>
cudaError_t by_rows(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    int rows = 0;
    for (int i = 0; i < n; ++i) rows = std::max(rows, req[i].nq * (c.hq / c.hkv));
    if (rows <= 16)
        return n <= kPagedFew ? launch<D, kCodes, 1, kPagedFew>(c, req, n, s) : launch<D, kCodes, 1, kPagedMany>(c, req, n, s);
    return n <= kPagedFew ? launch<D, kCodes, 2, kPagedFew>(c, req, n, s) : launch<D, kCodes, 2, kPagedMany>(c, req, n, s);
}

}  // namespace

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
    if (d == 128) return codes ? by_rows<128, true>(c, req, n, s) : by_rows<128, false>(c, req, n, s);
    return codes ? by_rows<64, true>(c, req, n, s) : by_rows<64, false>(c, req, n, s);
}

}  // namespace c2kv
