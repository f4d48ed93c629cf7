// Paged attention of many query rows: chunks of a prompt (c2kv_paged_attend).
//
// The rows of a (request, KV head) are taken 256 at a time, two tiles A and B of 128 in a CTA, over all
// the keys that they see: S = Q.K^T and P.V are tcgen05 products of 128 x 128 keys, S and O stay in
// tensor memory, and each tile's softmax (a warpgroup, a row a thread) runs beside the other tile's
// products.  The tensor cores bound it, four products of 2 M multiply-adds a key tile and CTA.
//
// The keys come by TMA from key tiles, f16 relative to a power of two of their own (paged_expand.cu).  The
// tiles' powers of two come back in the softmax: K's as a factor of the scores, V's as an offset of the
// exponent (the running reference is of score + offset, so that weights of every tile fit f16; the sum of
// weights takes the offset back).  Queries are f16 too, each row scaled by a power of two.
//
// Measured: 2048 tokens over 30720 rows (32 / 8 heads) 866 us with the tiles' making and the join, 1.23
// PFLOP/s; a key tile takes a CTA 1.7 us where its products alone would take 1.33 (the weights of a tile
// lie where its next scores go, so a tile's softmax and its own products follow one another, and only the
// other tile's run beside them).  A CTA's start and end are 8 us: chunks of four prompts, 64 equal units on
// 152 SMs, 86 us.
#include "paged.cuh"
#include "paged_row.cuh"
#include "per_device.cuh"
#include "ptx.cuh"
#include "rope.cuh"
#include "tcgen05.cuh"

#include <math_constants.h>

#include <algorithm>
#include <optional>
#include <type_traits>
#include <utility>
#include <vector>

namespace c2kv {
namespace {

constexpr int BM = 128;                  // rows of a query tile
constexpr int BN = 128;                  // keys of a tile
constexpr int kPair = 2 * BM;
constexpr int kUnits = 8;                // tiles whose notes are kept: more than K has stages

// Warp 0 issues the products, warp 1 loads, 4..7 and 8..11 are the softmax of tiles A and B, which holds
// a row of scores in registers.
constexpr int kThreads = 384;
constexpr int kLaunchRegs = 168, kRegsLow = 136, kRegsSoftmax = 184;
static_assert(128 * kRegsLow + 256 * kRegsSoftmax <= kThreads * kLaunchRegs, "register split");

constexpr uint32_t kTmemCols = 512;      // S_A, S_B (P over their first halves), O_A, O_B
constexpr uint32_t kColO = 256;

template <int D>
struct Tc {
    static constexpr int kK = 3, kV = 2;                   // stages of K and of V tiles
    static constexpr int kTile = BN * D * 2;               // bytes of a tile
    static constexpr int kHalf = BN * 128;                 // of its 64-channel block
    // barriers: tile landed / free (K, V), scores, weights, O, queries
    static constexpr int KF = 0, KE = KF + kK, VF = KE + kK, VE = VF + kV, S = VE + kV, P = S + 2, O = P + 2, Q = O + 1, kBars = Q + 1;
    static constexpr int kTiles = (2 + kK + kV) * kTile;
    static constexpr int kNotes = kTiles + (8 * kBars + 15) / 16 * 16;
    static constexpr int kBack = kNotes + 32 * kUnits;     // powers of two of the queries' rows: a byte each
    static constexpr int kSlot = kBack + kPair;
    static constexpr int kSmem = 1024 /*align*/ + kSlot + 16;
};
static_assert(Tc<128>::kSmem <= 232448, "shared memory of a CTA");

// What the softmax needs to know of a key tile: K's power of two, V's exponent, which of its eight groups of
// 16 keys lie in pages (bits), and which rows of V have values that are not finite (zero in the tile).
struct __align__(16) TileNote {
    float k_unit;
    float v_exp;
    uint32_t there;
    uint32_t pad;
    uint4 odd;
};

template <int kReq>
struct TcLaunch {
    CUtensorMap tm_k, tm_v;              // key tiles [n * Hkv][128][d], boxes of 64 channels
    const float2* unit;                  // [n][Hkv]
    const uint32_t* there;               // [n]
    const uint4* odd;                    // [n][Hkv]
    float* part_o;                       // [item][256][D] normalised
    float* part_lse;                     // [item][256] log2 domain
    PagedAttn<kReq> a;
};

// kind::f16 with f16 operands, D fp32, A K-major, B K- or MN-major.
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major) {
    return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The CTA's work: rows [row0, row0 + live) of request R's KV head hk, key tiles [j0, j0 + n).
struct Item {
    PagedReq R;
    int hk, sp, row0, live, j0, n;
    int k_lo, k_hi;                      // keys that some row sees: [k_lo, k_hi)
};

template <int kReq>
__device__ __forceinline__ Item find_item(const PagedAttn<kReq>& P) {
    Item w;
    int r = 0;
    for (int hi = P.batch; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.req[mid].item0 <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    w.R = P.req[r];
    const int G = P.hq / P.hkv, n_rows = w.R.nq * G;
    int i = blockIdx.x - w.R.item0;
    // the last rows first: they see the most keys
    w.hk = i % P.hkv;
    i /= P.hkv;
    w.sp = i % w.R.splits;
    const int pr = w.R.tile0 + w.R.tiles - 1 - i / w.R.splits;
    w.row0 = pr * kPair;
    w.live = min(kPair, n_rows - w.row0);
    const int before = w.R.n_keys - w.R.nq;
    w.k_hi = before + (w.row0 + w.live - 1) / G + 1;
    w.k_lo = P.window ? max(0, before + w.row0 / G - P.window + 1) : 0;
    const int t_lo = w.k_lo / BN, t_n = max(0, (w.k_hi + BN - 1) / BN - t_lo);
    w.j0 = t_lo + (int)((int64_t)t_n * w.sp / w.R.splits);
    w.n = t_lo + (int)((int64_t)t_n * (w.sp + 1) / w.R.splits) - w.j0;
    return w;
}

// ------------------------------------------------------------------ loaders

// One thread brings K and V tiles, and the softmax's notes of them.
template <int D, int kReq>
__device__ __forceinline__ void load_tiles(const TcLaunch<kReq>& X, const Item& w, uint32_t sK, uint32_t sV, uint32_t bars,
                                           TileNote* notes, volatile uint32_t* abort) {
    using C = Tc<D>;
    const PagedAttn<kReq>& P = X.a;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int t0 = w.R.scratch + w.j0;
    asm volatile("griddepcontrol.wait;" ::: "memory");           // the key tiles are complete and visible
    float2 unit = ld_after(X.unit + (int64_t)t0 * P.hkv + w.hk);
    uint32_t there = ld_after(X.there + t0);
    uint4 odd = ld_after(X.odd + (int64_t)t0 * P.hkv + w.hk);
    for (int j = 0; j < w.n; ++j) {
        const int at = (t0 + j) * P.hkv + w.hk;
        notes[j & (kUnits - 1)] = TileNote{unit.x, unit.y, there, 0u, odd};
        if (j + 1 < w.n) {               // (the next tile's: on their way while this one's are)
            unit = ld_after(X.unit + (int64_t)at + P.hkv);
            there = ld_after(X.there + t0 + j + 1);
            odd = ld_after(X.odd + (int64_t)at + P.hkv);
        }
        const int ks = j % C::kK, vs = j % C::kV;
        if (j >= C::kK) mbar_wait(bar(C::KE + ks), (uint32_t)(j / C::kK - 1) & 1u, P.err, abort);
        mbar_expect_tx(bar(C::KF + ks), C::kTile);
#pragma unroll
        for (int b = 0; b < D / 64; ++b) tma_load_3d(sK + ks * C::kTile + b * C::kHalf, &X.tm_k, b * 64, 0, at, bar(C::KF + ks));
        if (j >= C::kV) mbar_wait(bar(C::VE + vs), (uint32_t)(j / C::kV - 1) & 1u, P.err, abort);
        mbar_expect_tx(bar(C::VF + vs), C::kTile);
#pragma unroll
        for (int b = 0; b < D / 64; ++b) tma_load_3d(sV + vs * C::kTile + b * C::kHalf, &X.tm_v, b * 64, 0, at, bar(C::VF + vs));
    }
}

// ------------------------------------------------------------------ products

// Issue order per key tile: PV_A(j - 1), S_A(j), PV_B(j - 1), S_B(j): a tile's next scores follow the
// product that read the weights they overwrite, and each tile's softmax runs beside the other's products.
template <int D>
__device__ __forceinline__ void issue_products(uint32_t tmem, uint32_t sQ, uint32_t sK, uint32_t sV, uint32_t bars, int n, bool has_b,
                                               int32_t* err, volatile uint32_t* abort) {
    constexpr uint32_t idS = idesc_f16(BM, BN, false), idO = idesc_f16(BM, D, true);
    using C = Tc<D>;
    constexpr uint64_t kTileDesc = (uint64_t)(C::kTile >> 4);
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto wait = [&](int i, uint32_t parity) {
        mbar_wait(bar(i), parity, err, abort);
        tc_fence_after();
    };
    const uint64_t dQa = sw128_desc(sQ, 16, 1024), dQb = sw128_desc(sQ + C::kTile, 16, 1024);
    const uint64_t dK0 = sw128_desc(sK, 16, 1024), dV0 = sw128_desc(sV, C::kHalf, 1024);
    auto scores = [&](uint64_t dq, uint64_t dk, uint32_t d) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t off = (uint64_t)(((kk >> 2) * C::kHalf + (kk & 3) * 32) >> 4);
            mma_bf16(d, dq + off, dk + off, idS, kk > 0 ? 1u : 0u);
        }
    };
    auto values = [&](uint32_t p, uint64_t dv, uint32_t o, uint32_t acc) {
#pragma unroll
        for (int kk = 0; kk < BN / 16; ++kk)
            mma_bf16_ts(o, p + (uint32_t)kk * 8u, dv + (uint64_t)((kk * 16 * 128) >> 4), idO, kk > 0 ? 1u : acc);
    };
    const uint32_t tSa = tmem, tSb = tmem + BN, tOa = tmem + kColO, tOb = tOa + D;
    int ks = 0, vs = 0;
    uint32_t kp = 0, vp = 0;
    wait(C::Q, 0);
    wait(C::KF, 0);
    scores(dQa, dK0, tSa);
    mma_commit(bar(C::S));
    if (has_b) {
        scores(dQb, dK0, tSb);
        mma_commit(bar(C::S + 1));
    }
    mma_commit(bar(C::KE));
    for (int j = 1; j <= n; ++j) {
        const bool more = j < n;
        if (++ks == C::kK) {
            ks = 0;
            kp ^= 1u;
        }
        const uint64_t dk = dK0 + (uint64_t)ks * kTileDesc, dv = dV0 + (uint64_t)vs * kTileDesc;
        const uint32_t acc = j > 1 ? 1u : 0u, pp = (uint32_t)(j - 1) & 1u;
        wait(C::P, pp);
        wait(C::VF + vs, vp);
        values(tSa, dv, tOa, acc);
        if (more) {
            wait(C::KF + ks, kp);
            scores(dQa, dk, tSa);
            mma_commit(bar(C::S));
        }
        if (has_b) {
            wait(C::P + 1, pp);
            values(tSb, dv, tOb, acc);
        }
        mma_commit(bar(C::VE + vs));
        if (more) {
            if (has_b) {
                scores(dQb, dk, tSb);
                mma_commit(bar(C::S + 1));
            }
            mma_commit(bar(C::KE + ks));
        }
        if (++vs == C::kV) {
            vs = 0;
            vp ^= 1u;
        }
    }
    mma_commit(bar(C::O));
}

// ------------------------------------------------------------------ softmax

// The pair's queries, turned, into their tiles (128-byte swizzle), by the eight softmax warps, 32 rows
// each: copied as they are, all on their way at once and before the CTA is set up (fetch), then turned and
// made f16 in place, eight rows at a time (a row after the other is a chain of dependent instructions).  A
// row's largest value goes to [2^14, 2^15) before it turns, which keeps it below 2^15.5: its scores come
// back by 2^back.
template <int D>
struct QueryRows {
    static constexpr int E = D / 64;                     // channels of each half a lane
    uint64_t turn[E];
    int pos;                                             // of row `lane`
};

template <int D, int kReq>
__device__ __forceinline__ QueryRows<D> fetch_queries(const PagedAttn<kReq>& P, const Item& w, int warp, int lane, uint32_t sQ) {
    using T = __nv_bfloat16;
    using C = Tc<D>;
    const int G = P.hq / P.hkv;
    const int r0 = warp * 32, n = max(0, min(32, w.live - r0));
    const uint32_t tile = sQ + (r0 / BM) * C::kTile + (r0 % BM) * 128;
    // lane i knows where row i lies; a copy takes whole rows, 16 bytes a lane
    const int row = w.row0 + r0 + min(lane, max(0, n - 1)), tok = row / G;
    const int64_t at = (w.R.q0 + tok) * P.q_stride + ((int64_t)w.hk * G + row - tok * G) * D;
    constexpr int kChunks = D / 8, kStep = 32 / kChunks;
    const int q = lane % kChunks;
    const T* const base = static_cast<const T*>(P.q) + q * 8;
#pragma unroll
    for (int i0 = 0; i0 < 32; i0 += kStep) {
        const int i = i0 + lane / kChunks;
        const uint32_t to = tile + (uint32_t)((q >> 3) * C::kHalf + i * 128 + (((q & 7) ^ (i & 7)) << 4));
        cp_async16_or_zero(to, base + __shfl_sync(0xffffffffu, at, i), i < n);   // zero past the rows: a number
    }
    cp_async_commit();
    QueryRows<D> k;
    k.pos = 0;
#pragma unroll
    for (int e = 0; e < k.E; ++e) k.turn[e] = 0;
    if (P.turn && n > 0) {
#pragma unroll
        for (int e = 0; e < k.E; ++e) k.turn[e] = lane_turn(P.rope.turn, lane * k.E + e);
        k.pos = ld_after(P.turn + w.R.q0 + tok);
    }
    return k;
}

template <int D, int kReq>
__device__ __forceinline__ void turn_queries(const PagedAttn<kReq>& P, const QueryRows<D>& k, int warp, int lane, uint32_t sQ, int8_t* s_back) {
    using C = Tc<D>;
    constexpr int E = QueryRows<D>::E, kBatch = 8;       // rows in flight
    const int r0 = warp * 32;
    const int c = lane * E, q0 = c >> 3, q1 = (D / 2 + c) >> 3;
    const uint32_t tile = sQ + (r0 / BM) * C::kTile + (r0 % BM) * 128;
    float2 cs[E];
    int pos_cs = __shfl_sync(0xffffffffu, k.pos, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) cs[e] = turn_cs_fast(k.turn[e], pos_cs);
    cp_async_wait<0>();
    __syncwarp();
#pragma unroll 1
    for (int i0 = 0; i0 < 32; i0 += kBatch) {
        uint32_t x0[kBatch], x1[kBatch];
        const uint32_t a0 = (c & 7) * 2 + (q0 >> 3) * C::kHalf + tile + i0 * 128, a1 = (c & 7) * 2 + (q1 >> 3) * C::kHalf + tile + i0 * 128;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {               // (i0 is a multiple of 8: the rows swap as rows 0 .. 7 do)
            const uint32_t s0 = a0 + i * 128 + (((q0 & 7) ^ i) << 4), s1 = a1 + i * 128 + (((q1 & 7) ^ i) << 4);
            if constexpr (E == 2) {
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x0[i]) : "r"(s0));
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x1[i]) : "r"(s1));
            } else {
                uint16_t y0, y1;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y0) : "r"(s0));
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y1) : "r"(s1));
                x0[i] = y0;
                x1[i] = y1;
            }
        }
        float f[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t m = __vmaxu2(x0[i] & 0x7fff7fffu, x1[i] & 0x7fff7fffu);
            const uint32_t top = __reduce_max_sync(0xffffffffu, max(m & 0xffff0000u, m << 16));
            const int ex = (int)(top >> 23) - 127;       // zero and non-finite rows stay as they are
            const bool scaled = top < 0x7f800000u && ex > -100;
            f[i] = scaled ? pow2i(14 - ex) : 1.f;
            if (lane == i) s_back[r0 + i0 + i] = (int8_t)(scaled ? ex - 14 : 0);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            float x[E], y[E], lo[E], hi[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = __uint_as_float(e == 0 ? x0[i] << 16 : x0[i] & 0xffff0000u) * f[i];
                y[e] = __uint_as_float(e == 0 ? x1[i] << 16 : x1[i] & 0xffff0000u) * f[i];
                lo[e] = x[e];
                hi[e] = y[e];
            }
            if (P.turn) {
                const int pos = __shfl_sync(0xffffffffu, k.pos, i0 + i);
                if (pos != pos_cs) {                     // the heads of a token share its angles
#pragma unroll
                    for (int e = 0; e < E; ++e) cs[e] = turn_cs_fast(k.turn[e], pos);
                    pos_cs = pos;
                }
                rotate<E>(x, y, cs, lo, hi);
            }
            x0[i] = pack_f16(lo[0], E == 2 ? lo[E - 1] : 0.f);
            x1[i] = pack_f16(hi[0], E == 2 ? hi[E - 1] : 0.f);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t s0 = a0 + i * 128 + (((q0 & 7) ^ i) << 4), s1 = a1 + i * 128 + (((q1 & 7) ^ i) << 4);
            if constexpr (E == 2) {
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(s0), "r"(x0[i]));
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(s1), "r"(x1[i]));
            } else {
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(s0), "h"((uint16_t)x0[i]));
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(s1), "h"((uint16_t)x1[i]));
            }
        }
    }
}

// Of 32 keys key0 .. whose bits are `keys`, those in (start, end].
__device__ __forceinline__ uint32_t within(uint32_t keys, int key0, int start, int end) {
    const int lo = max(0, start + 1 - key0), hi = min(31, end - key0);
    return lo > hi ? 0u : keys & (0xffffffffu << lo) & (0xffffffffu >> (31 - hi));
}

// Rows that see values of V which are not finite (bits of `bad`, a lane a row from row0 on): of a channel's
// infinities and NaN nothing is left but which there are, and nothing else matters there.  The warp looks the
// noted keys up once for all its rows.  (Computed again key by key, a chunk of 256 tokens over one such row
// of 8192 took 28 ms for 70 us.)
template <int D, bool kCodes, int kReq>
__device__ __forceinline__ void take_in(const TcLaunch<kReq>& X, const Item& w, uint32_t bad, int start, int end, int row0, int lane, uint8_t* q_tiles) {
    using T = __nv_bfloat16;
    constexpr int E = D / 32;                                    // channels a lane, a byte each: 1 infinity, 2 minus it, 4 NaN
    constexpr uint32_t kNan = E == 4 ? 0x04040404u : 0x0404u;
    using Word = typename std::conditional<E == 4, uint32_t, uint16_t>::type;
    const PagedAttn<kReq>& P = X.a;
    const int G = P.hq / P.hkv, size = 1 << P.pg.page_shift;
    const int32_t* const table = P.pg.table + (int64_t)w.R.row * P.pg.table_stride;
    Word* const of_row = reinterpret_cast<Word*>(q_tiles + row0 * D) + lane;      // (the products have read the queries)
    for (int i = 0; i < 32; ++i) of_row[i * 32] = 0;
    after_kernels_before();                                      // (the notes in memory: this thread has not waited)
    uint32_t common = 0;                                         // of keys that all of the rows see
    bool rest = true;
    for (int j0 = 0; j0 < w.n && rest; j0 += 32) {
        uint4 odd = make_uint4(0u, 0u, 0u, 0u);
        if (j0 + lane < w.n) odd = ld_after(X.odd + (int64_t)(w.R.scratch + w.j0 + j0 + lane) * P.hkv + w.hk);
        for (uint32_t tiles = __ballot_sync(0xffffffffu, (odd.x | odd.y | odd.z | odd.w) != 0u); tiles && rest; tiles &= tiles - 1) {
            const int j = __ffs(tiles) - 1;
#pragma unroll 1
            for (int k = 0; k < 4 && rest; ++k) {
                uint32_t keys = __shfl_sync(0xffffffffu, k == 0 ? odd.x : k == 1 ? odd.y : k == 2 ? odd.z : odd.w, j);
                for (; keys && rest; keys &= keys - 1) {
                    const int key = (w.j0 + j0 + j) * BN + 32 * k + __ffs(keys) - 1;
                    uint32_t rows = __ballot_sync(0xffffffffu, key > start && key <= end) & bad;
                    if (rows == 0u) continue;
                    const int64_t page = ld_after(table + (key >> P.pg.page_shift)), in_page = (int64_t)w.hk * size + (key & (size - 1));
                    float v[E];
                    lane_row<T, D, kCodes>(P.pg.v, page * P.pg.page_stride + in_page * D,
                                           kCodes ? ld_after(P.pg.v_scale + page * P.pg.scale_stride + in_page) : 1.f, lane, v);
                    // a key with an infinity of K too scores -inf, the row's sum being a number: 0 times it is NaN
                    float y[E];
                    lane_row<T, D, kCodes>(P.pg.k, page * P.pg.page_stride + in_page * D,
                                           kCodes ? ld_after(P.pg.k_scale + page * P.pg.scale_stride + in_page) : 1.f, lane, y);
                    bool odd_k = false;
#pragma unroll
                    for (int e = 0; e < E; ++e) odd_k = odd_k || !(fabsf(y[e]) < CUDART_INF_F);
                    const bool no_weight = __any_sync(0xffffffffu, odd_k);
                    uint32_t is = 0;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (!(fabsf(v[e]) < CUDART_INF_F))
                            is |= (isnan(v[e]) || no_weight ? 4u : v[e] > 0.f ? 1u : 2u) << (8 * e);
                    if (rows == bad) {
                        common |= is;
                        rest = __any_sync(0xffffffffu, (common & kNan) != kNan);
                    } else {
                        for (; rows; rows &= rows - 1) of_row[(__ffs(rows) - 1) * 32] |= (Word)is;
                    }
                }
            }
        }
    }
    const bool whole = w.R.splits == 1;
    __syncwarp();                                                // (after the rows' own stores)
    for (; bad; bad &= bad - 1) {
        const int i = __ffs(bad) - 1, rr = w.row0 + row0 + i;
        const uint32_t is = common | of_row[i * 32];
        const int64_t at = whole ? ((w.R.q0 + rr / G) * (int64_t)P.hq + w.hk * G + rr % G) * D : ((int64_t)blockIdx.x * kPair + row0 + i) * D;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t f = is >> (8 * e) & 7u;
            if (f == 0u) continue;
            const float y = f == 1u ? CUDART_INF_F : f == 2u ? -CUDART_INF_F : CUDART_NAN_F;
            if (whole) static_cast<T*>(P.out)[at + lane * E + e] = static_cast<T>(y);
            else X.part_o[at + lane * E + e] = y;
        }
    }
}

// One softmax thread: row r of tile x over the CTA's key tiles, then its output.
//
// Weights are 2^(score + offset - ref) with the reference of the tiles before: the tile's own maximum need
// not be known first, and is found after the weights are handed over, beside the products.  A reference is
// set 2^8 below the maximum, so that a long tail of small weights keeps f16's 11 bits down to 2^-22 of the
// largest (and a tile of equal weights, 2^15 together, passes for what the guard lets through).  O and the sum
// are scaled to a new one, before the next tile, only when weights have passed 2^14.  Where a sum shows
// weights near f16's largest (or the row has no reference yet) the maximum comes first after all.
constexpr float kBelow = 8.f, kRoom = 14.f, kMostSum = 61440.f;

template <int D, bool kCodes, int kReq>
__device__ __forceinline__ void softmax_rows(const TcLaunch<kReq>& X, const Item& w, uint32_t tmem, uint32_t bars, int x, int quad, int lane,
                                             const TileNote* notes, const int8_t* s_back, volatile uint32_t* abort, uint8_t* q_tiles) {
    using T = __nv_bfloat16;
    using C = Tc<D>;
    const PagedAttn<kReq>& P = X.a;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int G = P.hq / P.hkv;
    const int r = quad * 32 + lane, row = x * BM + r;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t colS = tmem + lane_addr + (uint32_t)(x * BN), colO = tmem + lane_addr + kColO + (uint32_t)(x * D);
    const bool there = row < w.live;
    const int my = min(row, w.live - 1);
    const int end = w.R.n_keys - w.R.nq + (w.row0 + my) / G;     // the last key the row sees
    const int start = P.window ? end - P.window : -1;            // and the last that it does not, before them
    const float rs = P.scale_log2 * pow2i(s_back[row]);
    float ref = -CUDART_INF_F, top = -CUDART_INF_F, l = 0.f;
    bool touched = false;                // by values that are not finite
    auto scale_o = [&](float alpha) {
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
    for (int j = 0; j < w.n; ++j) {
        mbar_wait(bar(C::S + x), (uint32_t)j & 1u, P.err, abort);
        tc_fence_after();
        uint32_t sv[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(colS + c * 32, sv[c]);
        // scores of tile j are complete, so is every product before them: O may be scaled
        const bool moves = top > ref + kRoom;
        float alpha = 1.0f;
        if (__any_sync(0xffffffffu, moves)) {
            if (moves) {
                alpha = ex2(ref - (top - kBelow));               // (0 from no reference at all)
                ref = top - kBelow;
            }
            if (j > 0) scale_o(alpha);
            l *= alpha;
        }
        const TileNote nt = notes[j & (kUnits - 1)];
        const uint32_t groups = nt.there;
        // (kept within fp32's normal range: hidden scores of -inf times zero, or scores of zero times infinity,
        // would be no number)
        const float f = fminf(fmaxf(rs * nt.k_unit, 0x1p-126f), 0x1.fffffep127f), ve = nt.v_exp;
        const int key0 = (w.j0 + j) * BN;
        if (nt.odd.x | nt.odd.y | nt.odd.z | nt.odd.w)
            touched = touched || within(nt.odd.x, key0, start, end) || within(nt.odd.y, key0 + 32, start, end) ||
                      within(nt.odd.z, key0 + 64, start, end) || within(nt.odd.w, key0 + 96, start, end);
        tmem_ld_wait();
        if (key0 + BN - 1 > end || key0 <= start || groups != 0xffu) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const int key = key0 + c * 32 + e;
                    if (key > end || key <= start || !(groups >> (2 * c + e / 16) & 1u)) sv[c][e] = __float_as_uint(-CUDART_INF_F);
                }
        }
        auto find_top = [&]() {
            float top4[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float m = fmaxf(__uint_as_float(sv[c][0]), __uint_as_float(sv[c][1]));
#pragma unroll
                for (int e = 2; e < 32; e += 2) m = fmax3(m, __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
                top4[c] = m;
            }
            top = fmaf(fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])), f, ve);
        };
        auto weigh = [&]() {
            float ps[4] = {0.f, 0.f, 0.f, 0.f};
            const float off = ref == -CUDART_INF_F ? ve : ve - ref;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t pk[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float a0, a1;
                    ffma2(a0, a1, __uint_as_float(sv[c][2 * i]), __uint_as_float(sv[c][2 * i + 1]), f, off);
                    a0 = ex2(a0);
                    a1 = ex2(a1);
                    if (i & 1) fadd2(ps[2], ps[3], a0, a1);
                    else fadd2(ps[0], ps[1], a0, a1);
                    pk[i] = pack_f16(a0, a1);
                }
                tmem_st16(colS + c * 16, pk);
            }
            return (ps[0] + ps[1]) + (ps[2] + ps[3]);
        };
        float sum = 0.f;
        bool high = ref == -CUDART_INF_F;
        if (!__all_sync(0xffffffffu, high)) {
            sum = weigh();
            high = high || !(sum < kMostSum);
        }
        if (__any_sync(0xffffffffu, high)) {
            find_top();
            alpha = 1.0f;
            if (high && top - kBelow > ref) {
                alpha = ex2(ref - (top - kBelow));
                ref = top - kBelow;
            }
            if (j > 0) scale_o(alpha);
            l *= alpha;
            sum = weigh();
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(bar(C::P + x));
        l = fmaf(sum, ex2(-ve), l);
        find_top();
    }
    if (w.n > 0) {
        mbar_wait(bar(C::O), 0u, P.err, abort);
        tc_fence_after();
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const float lse2 = l == 0.f ? -CUDART_INF_F : ref + log2f(l);
    const int64_t tok = w.R.q0 + (w.row0 + my) / G;
    const int h = w.hk * G + (w.row0 + my) % G;
    const bool whole = w.R.splits == 1;
    T* const orow = static_cast<T*>(P.out) + (tok * P.hq + h) * D;
    float* const prow = X.part_o + ((int64_t)blockIdx.x * kPair + row) * D;
    const bool wide = (reinterpret_cast<uintptr_t>(P.out) & 31u) == 0;
    const float none = there && whole && l == 0.f ? of_no_weight(P, w.R.row, end) : 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        uint32_t ov[32];
        if (w.n > 0) {
            tmem_ld32(colO + c * 32, ov);
            tmem_ld_wait();
        } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) ov[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            ov[e] = l == 0.f ? __float_as_uint(none) : __float_as_uint(__uint_as_float(ov[e]) * inv);
        }
        if (!there) continue;
        if (whole) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t o8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o8[e] = pack_bf16(__uint_as_float(ov[16 * k + 2 * e]), __uint_as_float(ov[16 * k + 2 * e + 1]));
                if (wide) {
                    stg256(orow + c * 32 + k * 16, o8);
                } else {
                    *reinterpret_cast<uint4*>(orow + c * 32 + k * 16) = make_uint4(o8[0], o8[1], o8[2], o8[3]);
                    *reinterpret_cast<uint4*>(orow + c * 32 + k * 16 + 8) = make_uint4(o8[4], o8[5], o8[6], o8[7]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) stg256(prow + c * 32 + k * 8, ov + 8 * k);
        }
    }
    if (there) {
        if (!whole) X.part_lse[(int64_t)blockIdx.x * kPair + row] = lse2;
        else if (P.lse) P.lse[(int64_t)h * P.n_tokens + tok] = lse2 * 0.69314718055994531f;
    }
    const uint32_t bad = __ballot_sync(0xffffffffu, there && touched && l < CUDART_INF_F);
    if (bad) take_in<D, kCodes>(X, w, bad, start, end, x * BM + quad * 32, lane, q_tiles);
}

// ------------------------------------------------------------------ kernel

template <int D, bool kCodes, int kReq>
__global__ void __launch_bounds__(kThreads, 1) paged_tc_kernel(const __grid_constant__ TcLaunch<kReq> X) {
    const PagedAttn<kReq>& P = X.a;
    using C = Tc<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sQ = smem_u32(smem), sK = sQ + 2 * C::kTile, sV = sK + C::kK * C::kTile;
    const uint32_t bars = sQ + C::kTiles;
    TileNote* const notes = reinterpret_cast<TileNote*>(smem + C::kNotes);
    int8_t* const s_back = reinterpret_cast<int8_t*>(smem + C::kBack);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(smem + C::kSlot);
    volatile uint32_t* const abort = slot + 1;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Item w = find_item(P);
    const bool has_b = w.live > BM;
    QueryRows<D> rows;
    if (warp >= 4) rows = fetch_queries<D>(P, w, warp - 4, lane, sQ);

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kK; ++s) {
            mbar_init(bar(C::KF + s), 1);
            mbar_init(bar(C::KE + s), 1);
        }
        for (int s = 0; s < C::kV; ++s) {
            mbar_init(bar(C::VF + s), 1);
            mbar_init(bar(C::VE + s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::S + i), 1);
            mbar_init(bar(C::P + i), 128);
        }
        mbar_init(bar(C::O), 1);
        mbar_init(bar(C::Q), 256);
        *abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;
    // the kernel that joins cut keys may be set up from here on: it waits for this grid to end
    if (threadIdx.x == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLow));
        if (warp == 1 && lane == 0 && w.n > 0) load_tiles<D>(X, w, sK, sV, bars, notes, abort);
        else if (warp == 0 && lane == 0 && w.n > 0) issue_products<D>(tmem, sQ, sK, sV, bars, w.n, has_b, P.err, abort);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        turn_queries<D>(P, rows, warp - 4, lane, sQ, s_back);
        fence_proxy_async();
        asm volatile("bar.sync 1, 256;" ::: "memory");           // (the rows' powers of two)
        mbar_arrive(bar(C::Q));
        const int x = warp >= 8;
        if (x == 0 || has_b) softmax_rows<D, kCodes>(X, w, tmem, bars, x, warp & 3, lane, notes, s_back, abort, smem);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// The stretches of cut keys joined: 32 rows of a unit a CTA, eight rows a thread on their way at once.
// (Joined by the last stretch of a unit instead, 19 partials of 128 KB came through one SM: 72 us for 64
// tokens over 30000 rows, where this takes 4 of them.)
constexpr int kJoinThreads = 128, kJoinRows = 32;

template <int D, int kReq>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const __grid_constant__ TcLaunch<kReq> X) {
    const PagedAttn<kReq>& P = X.a;
    extern __shared__ float weight[];                            // [stretch][row]
    constexpr int kSlices = kPair / kJoinRows;
    const int u = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
    int r = 0;
    while (r + 1 < P.batch && P.req[r + 1].unit0 <= u) ++r;      // (entries that are not cut have no units)
    asm volatile("griddepcontrol.wait;" ::: "memory");           // the partials are complete and visible
    const PagedReq R = P.req[r];
    const int G = P.hq / P.hkv, S = R.splits, k0 = u - R.unit0, hk = k0 % P.hkv, pr = R.tile0 + k0 / P.hkv;
    const int first = slice * kJoinRows, live = min(kJoinRows, R.nq * G - pr * kPair - first);
    if (live <= 0) return;
    // items of the unit's stretch k: see find_item
    const int64_t item0 = R.item0 + ((int64_t)(R.tile0 + R.tiles - 1 - pr) * S) * P.hkv + hk;
    for (int row = threadIdx.x; row < live; row += kJoinThreads) {
        float top = -CUDART_INF_F, sum = 0.f;
        for (int k = 0; k < S; ++k) {
            const float e = ld_after_l2(X.part_lse + (item0 + (int64_t)k * P.hkv) * kPair + first + row);
            weight[k * kJoinRows + row] = e;
            top = fmaxf(top, e);
        }
        const float base = top == -CUDART_INF_F ? 0.f : top;
        for (int k = 0; k < S; ++k) sum += ex2(weight[k * kJoinRows + row] - base);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const float none = sum == 0.f ? of_no_weight(P, R.row, R.n_keys - R.nq + (pr * kPair + first + row) / G) : 0.f;
        for (int k = 0; k < S; ++k) weight[k * kJoinRows + row] = ex2(weight[k * kJoinRows + row] - base) * inv + none;
        if (P.lse) {
            const int all = pr * kPair + first + row;
            P.lse[(int64_t)(hk * G + all % G) * P.n_tokens + R.q0 + all / G] = sum == 0.f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
        }
    }
    __syncthreads();
    constexpr int kLines = D / 4, kStep = kJoinThreads / kLines, kRows = kJoinRows / kStep;
    const int f = threadIdx.x % kLines, row0 = threadIdx.x / kLines;
    float4 o[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < S; ++k) {
        const float* const from = X.part_o + ((item0 + (int64_t)k * P.hkv) * kPair + first) * D + 4 * f;
        float4 y[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) y[i] = ld_after_l2(reinterpret_cast<const float4*>(from + (int64_t)min(row0 + i * kStep, live - 1) * D));
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float a = weight[k * kJoinRows + min(row0 + i * kStep, live - 1)];
            o[i].x = fmaf(y[i].x, a, o[i].x);
            o[i].y = fmaf(y[i].y, a, o[i].y);
            o[i].z = fmaf(y[i].z, a, o[i].z);
            o[i].w = fmaf(y[i].w, a, o[i].w);
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int row = row0 + i * kStep;
        if (row >= live) continue;
        const int all = pr * kPair + first + row;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.out) + ((int64_t)(R.q0 + all / G) * P.hq + hk * G + all % G) * D + 4 * f) =
            make_uint2(pack_bf16(o[i].x, o[i].y), pack_bf16(o[i].z, o[i].w));
    }
}

// ------------------------------------------------------------------ host side

// Work items and their order.  A pair of row tiles over all its keys is one item, or its keys are cut
// into stretches whose partials are joined: a stretch costs its own start and end (about as much as
// kStart key tiles) and 128 KB written and read.  So keys are cut only where the schedule gets shorter:
// where units are fewer than SMs, where one request's are much longer than the others', and in the last
// round of many equal units.  The schedules compared are estimated by dealing items, longest first, to
// the SMs that are free first, as the hardware does.
constexpr double kStart = 6.0, kCutStart = 11.0;

struct Deal {
    // SMs by their load: (load, how many)
    std::vector<std::pair<double, int>> sms;
    explicit Deal(int n) { sms.push_back({0.0, n}); }
    void items(double cost, int64_t count) {
        while (count > 0) {
            auto low = std::min_element(sms.begin(), sms.end());
            // whole rounds over equally loaded SMs at once
            if (sms.size() == 1 && count >= low->second) {
                const int64_t rounds = count / low->second;
                low->first += cost * rounds;
                count -= rounds * low->second;
                continue;
            }
            const int take = (int)std::min<int64_t>(low->second, count);
            const double to = low->first + cost;
            low->second -= take;
            if (low->second == 0) sms.erase(low);
            auto same = std::find_if(sms.begin(), sms.end(), [&](const auto& x) { return x.first == to; });
            if (same != sms.end()) same->second += take;
            else sms.push_back({to, take});
            count -= take;
        }
    }
    double longest() const { return std::max_element(sms.begin(), sms.end())->first; }
};

// Entries of the launch: requests, or parts of them that are cut alike; longest items first.
std::vector<PagedReq> plan(const PagedAttnCall& c, const PagedReq* req, int n) {
    const int slots = device_sms(), G = c.hq / c.hkv;
    auto pairs_of = [&](const PagedReq& q) { return (int)(((int64_t)q.nq * G + kPair - 1) / kPair); };
    auto keys_of = [&](const PagedReq& q, int pr) {      // key tiles of a pair
        const int last = (int)std::min<int64_t>((int64_t)(pr + 1) * kPair, (int64_t)q.nq * G) - 1;
        const int hi = q.n_keys - q.nq + last / G + 1, lo = c.window ? std::max(0, q.n_keys - q.nq + pr * kPair / G - c.window + 1) : 0;
        return std::max(1, (hi + BN - 1) / BN - lo / BN);
    };
    auto piece = [](const PagedReq& e, int keys) { return (keys + e.splits - 1) / e.splits + (e.splits > 1 ? kCutStart : kStart); };
    int64_t units = 0;
    int longest = 1;
    for (int i = 0; i < n; ++i) {
        units += (int64_t)pairs_of(req[i]) * c.hkv;
        longest = std::max(longest, keys_of(req[i], pairs_of(req[i]) - 1));
    }
    std::vector<PagedReq> best;
    double best_cost = 0;
    // at: stretches of at most this many key tiles; rest > 0: only the last round's units are cut, into rest
    auto consider = [&](int at, int rest) {
        std::vector<PagedReq> e;
        const int64_t cut_units = rest ? units - units / slots * slots : 0;
        int64_t left = (cut_units + c.hkv - 1) / c.hkv;   // pairs still to be cut
        for (int i = n - 1; i >= 0; --i) {
            PagedReq q = req[i];
            const int pairs = pairs_of(q);
            if (!rest) {
                q.tile0 = 0;
                q.tiles = pairs;
                q.splits = (keys_of(q, pairs - 1) + at - 1) / at;
                e.push_back(q);
                continue;
            }
            const int cut = (int)std::min<int64_t>(left, pairs);          // the first pairs: those of fewest keys
            left -= cut;
            if (pairs > cut) {
                q.tile0 = cut;
                q.tiles = pairs - cut;
                q.splits = 1;
                e.push_back(q);
            }
            if (cut > 0) {
                q.tile0 = 0;
                q.tiles = cut;
                q.splits = std::max(1, std::min(rest, keys_of(q, cut - 1)));
                e.push_back(q);
            }
        }
        std::stable_sort(e.begin(), e.end(), [&](const PagedReq& a, const PagedReq& b) {
            return piece(a, keys_of(a, a.tile0 + a.tiles - 1)) > piece(b, keys_of(b, b.tile0 + b.tiles - 1));
        });
        Deal d(slots);
        for (const PagedReq& q : e) {
            // up to four groups of pairs, each as long as its longest
            for (int g = std::min(4, q.tiles), hi = q.tile0 + q.tiles; g > 0; --g) {
                const int lo = q.tile0 + q.tiles * (g - 1) / std::min(4, q.tiles);
                d.items(piece(q, keys_of(q, hi - 1)), (int64_t)(hi - lo) * c.hkv * q.splits);
                hi = lo;
            }
        }
        if (best.empty() || d.longest() < best_cost * 0.97) {     // (ties go to fewer cuts)
            best_cost = d.longest();
            best = std::move(e);
        }
    };
    consider(longest, 0);
    if (units < 8 * (int64_t)slots) {
        for (const int k : {2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            const int at = (longest + k - 1) / k;
            if (at < 2 || units * k > 16 * (int64_t)slots) break;
            consider(at, 0);
        }
        if (units < slots) consider((int)std::max<int64_t>(2, (longest * units + slots - 1) / slots), 0);   // (one round of equal stretches)
        if (units > slots && units % slots)
            for (const int k : {2, 3, 4, 5, 6, 7, 8}) consider(longest, k);
    }
    return best;
}

template <int D, bool kCodes, int kReq>
cudaError_t launch(const PagedAttnCall& c, const KeyTiles& tiles, const std::vector<PagedReq>& entries, cudaStream_t s) {
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_tc_kernel<D, kCodes, kReq>;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, Tc<D>::kSmem);
    if (e != cudaSuccess) return e;
    for (size_t b0 = 0; b0 < entries.size(); b0 += kReq) {
        const int nb = (int)std::min<size_t>(entries.size() - b0, kReq);
        TcLaunch<kReq> X;
        fill_paged(X.a, c, D, entries.data() + b0, nb);
        int64_t items = 0, units = 0;
        int32_t most = 1;
        auto lay_out = [&](bool cut) {
            items = units = 0;
            most = 1;
            for (int i = 0; i < nb; ++i) {
                PagedReq& q = X.a.req[i];
                if (!cut) q.splits = 1;
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
        X.part_o = X.part_lse = nullptr;
        std::optional<Workspace> work;
        if (units > 0) {
            const size_t o_bytes = (size_t)items * kPair * D * 4;
            work.emplace(c.ctx, o_bytes + (size_t)items * kPair * 4, 0);
            if (work->err == cudaErrorMemoryAllocation) {        // no room for partials: keys are not cut, slower
                (void)cudaGetLastError();
                lay_out(false);
            } else if (work->err != cudaSuccess) {
                return work->err;
            } else {
                X.part_o = static_cast<float*>(work->p);
                X.part_lse = reinterpret_cast<float*>(static_cast<char*>(work->p) + o_bytes);
            }
        }
        const cuuint64_t dims[3] = {D, kTileKeys, (cuuint64_t)std::max(1, tiles.n) * c.hkv}, strides[2] = {D * 2, kTileKeys * D * 2};
        const cuuint32_t box[3] = {64, kTileKeys, 1};
        if (!encode_tensor_map(&X.tm_k, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, tiles.k, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
            !encode_tensor_map(&X.tm_v, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, tiles.v, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B))
            return cudaErrorInvalidValue;
        X.unit = tiles.unit;
        X.there = tiles.there;
        X.odd = tiles.odd;
        // each starts while the kernel before it ends, and waits for it where it reads what that wrote
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)items);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = Tc<D>::kSmem;
        cfg.stream = s;
        cfg.attrs = &at;
        cfg.numAttrs = b0 == 0 && tiles.n > 0;   // (after another kernel than the tiles' it waits for all of that)
        e = cudaLaunchKernelEx(&cfg, kernel, X);
        if (e == cudaSuccess && units > 0) {
            cfg.gridDim = dim3((unsigned)(units * (kPair / kJoinRows)));
            cfg.blockDim = dim3(kJoinThreads);
            cfg.dynamicSmemBytes = (size_t)most * kJoinRows * 4;
            cfg.numAttrs = 1;
            e = cudaLaunchKernelEx(&cfg, paged_join_kernel<D, kReq>, X);
        }
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool kCodes>
cudaError_t by_count(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, cudaStream_t s) {
    const std::vector<PagedReq> entries = plan(c, req, n);
    return (int)entries.size() <= kPagedFew ? launch<D, kCodes, kPagedFew>(c, tiles, entries, s) : launch<D, kCodes, kPagedMany>(c, tiles, entries, s);
}

}  // namespace

cudaError_t launch_paged_tc(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? by_count<128, true>(c, tiles, req, n, s) : by_count<128, false>(c, tiles, req, n, s);
    return codes ? by_count<64, true>(c, tiles, req, n, s) : by_count<64, false>(c, tiles, req, n, s);
}

}  // namespace c2kv
