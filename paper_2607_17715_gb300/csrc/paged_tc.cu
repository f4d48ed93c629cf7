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
#include "paged_tile.cuh"

#include <algorithm>
#include <optional>
#include <type_traits>
#include <utility>
#include <vector>

namespace c2kv {
namespace {

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
struct Tc : TileOf<D> {
    using TileOf<D>::kTile;
    using TileOf<D>::kHalf;
    static constexpr int kK = 3, kV = 2;                   // stages of K and of V tiles
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

// One softmax thread: row r of tile x over the CTA's key tiles, then its output.
//
// Weights are 2^(score + offset - ref) with the reference of the tiles before: the tile's own maximum need
// not be known first, and is found after the weights are handed over, beside the products.  A reference is
// set 2^8 below the maximum, so that a long tail of small weights keeps f16's 11 bits down to 2^-22 of the
// largest (and a tile of equal weights, 2^15 together, passes for what the guard lets through).  O and the sum
// are scaled to a new one, before the next tile, only when weights have passed 2^14.  Where a sum shows
// weights near f16's largest (or the row has no reference yet) the maximum comes first after all.
constexpr float kBelow = 8.f, kRoom = 14.f, kMostSum = 61440.f;

template <int D, bool kCodes, bool kTree, int kReq>
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
    const Sight<kTree> sight(P, w, (w.row0 + my) / G);
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
            touched = touched || (nt.odd.x & sight.of32(key0)) || (nt.odd.y & sight.of32(key0 + 32)) || (nt.odd.z & sight.of32(key0 + 64)) ||
                      (nt.odd.w & sight.of32(key0 + 96));
        tmem_ld_wait();
        if (!sight.sees_tile(key0) || groups != 0xffu) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t seen = sight.of32(key0 + c * 32) & ((groups >> (2 * c) & 1u ? 0xffffu : 0u) | (groups >> (2 * c + 1) & 1u ? 0xffff0000u : 0u));
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (!(seen >> e & 1u)) sv[c][e] = __float_as_uint(-CUDART_INF_F);
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
    const float none = there && whole && l == 0.f ? of_no_weight<kTree>(P, w.R, (w.row0 + my) / G) : 0.f;
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
    if (bad) take_in<D, kCodes, kPair>(X, w, bad, sight, x * BM + quad * 32, lane, q_tiles);
}

// ------------------------------------------------------------------ kernel

template <int D, bool kCodes, int kReq, bool kTree>
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
    const Item w = find_item<kTree, kPair>(P, (int)blockIdx.x);
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
        if (x == 0 || has_b) softmax_rows<D, kCodes, kTree>(X, w, tmem, bars, x, warp & 3, lane, notes, s_back, abort, smem);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
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
        const int hi = q.n_keys - q.nq + last / G + 1, lo = c.window ? std::max(0, q.n_keys - q.nq + (c.parent ? 0 : pr * kPair / G) - c.window + 1) : 0;
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

template <int D, bool kCodes, int kReq, bool kTree>
cudaError_t launch(const PagedAttnCall& c, const KeyTiles& tiles, const std::vector<PagedReq>& entries, cudaStream_t s) {
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_tc_kernel<D, kCodes, kReq, kTree>;
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
            cfg.gridDim = dim3((unsigned)(units * (kPair / join_rows(D))));
            cfg.blockDim = dim3(kJoinThreads);
            cfg.dynamicSmemBytes = (size_t)most * join_rows(D) * 4;
            cfg.numAttrs = 1;
            e = cudaLaunchKernelEx(&cfg, paged_join_kernel<D, kPair, kTree, TcLaunch<kReq>>, X);
        }
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool kCodes, bool kTree>
cudaError_t by_count(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, cudaStream_t s) {
    const std::vector<PagedReq> entries = plan(c, req, n);
    constexpr int kLarge = kTree ? kPagedFew : kPagedMany;       // (trees: a launch for every 32 requests)
    return (int)entries.size() <= kPagedFew ? launch<D, kCodes, kPagedFew, kTree>(c, tiles, entries, s)
                                            : launch<D, kCodes, kLarge, kTree>(c, tiles, entries, s);
}

template <bool kTree>
cudaError_t by_kind(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? by_count<128, true, kTree>(c, tiles, req, n, s) : by_count<128, false, kTree>(c, tiles, req, n, s);
    return codes ? by_count<64, true, kTree>(c, tiles, req, n, s) : by_count<64, false, kTree>(c, tiles, req, n, s);
}

}  // namespace

// This file is compiled twice: trees of tokens are paged_tc_tree.cu's.
#ifndef C2KV_TREES

cudaError_t launch_paged_tc(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return c.parent ? launch_paged_tc_tree(c, tiles, req, n, d, codes, s) : by_kind<false>(c, tiles, req, n, d, codes, s);
}

#else

cudaError_t launch_paged_tc_tree(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    return by_kind<true>(c, tiles, req, n, d, codes, s);
}

#endif

}  // namespace c2kv
