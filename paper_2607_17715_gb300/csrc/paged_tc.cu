// Paged attention of many query rows: chunks of a prompt (c2kv_paged_attend).
//
// The rows of a (request, KV head) are taken 256 at a time, two tiles A and B of 128 in a CTA, over all
// the keys that they see: S = Q.K^T and P.V are tcgen05 products of 128 x 128 keys, S and O stay in
// tensor memory, and each tile's softmax (a warpgroup, a row a thread) runs beside the other tile's
// products.  The tensor cores bound it, four products of 2 M multiply-adds a key tile and CTA.
//
// Loader threads bring the keys, not TMA: a tile of 128 keys is gathered from up to eight pages, rows
// that no query may feel (past the last key, or of a page that is none) have to be zero in V whatever
// memory holds, and E4M3 codes are turned to f16 on the way.  A row's scale is applied there, relative
// to the power of two above the largest scale of its tile: f16 keeps 11 bits, and the tiles' powers of
// two come back in the softmax, K's as a factor of the scores, V's as an offset of the exponent (the
// running maximum is of score + offset, so that weights of every tile fit f16; the sum of weights
// takes the offset back).  Queries are scaled to f16's range a row.  16-bit pages keep bf16 throughout.
#include "paged.cuh"
#include "paged_row.cuh"
#include "per_device.cuh"
#include "ptx.cuh"
#include "rope.cuh"
#include "tcgen05.cuh"

#include <math_constants.h>

#include <algorithm>
#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int BM = 128;                  // rows of a query tile
constexpr int BN = 128;                  // keys of a tile
constexpr int kPair = 2 * BM;
constexpr int kK = 3, kV = 2;            // stages of K and of V tiles
constexpr int kUnits = 8;                // tiles whose powers of two are kept: more than K's stages

// Warps 0..3 load, 4..7 and 8..11 are the softmax of tiles A and B, warp 12 issues the products.  The
// softmax holds a row of scores in registers: 160 a thread, which warps 12..15 give.
constexpr int kThreads = 512;
constexpr int kRegsSoftmax = 160, kRegsLoad = 128, kRegsRest = 64;
static_assert(128 * kRegsLoad + 256 * kRegsSoftmax + 128 * kRegsRest <= kThreads * 128, "register split");

constexpr uint32_t kTmemCols = 512;      // S_A, S_B (P over their first halves), O_A, O_B
constexpr uint32_t kColO = 256;

enum { kBarKF = 0, kBarKE = kBarKF + kK, kBarVF = kBarKE + kK, kBarVE = kBarVF + kV, kBarS = kBarVE + kV, kBarP = kBarS + 2,
       kBarO = kBarP + 2, kBarQ, kBars };

template <int D>
struct Tc {
    static constexpr int kTile = BN * D * 2;               // bytes of a 16-bit tile
    static constexpr int kHalf = BN * 128;                 // of its 64-channel block
    static constexpr int kTail = 8 * kBars + 16 + 16 * kUnits + 4 * kPair;
    static constexpr int kSmem = 1024 /*align*/ + (2 + kK + kV) * kTile + kTail;
};
static_assert(Tc<128>::kSmem <= 232448, "shared memory of a CTA");

// What the loaders say of a key tile: K's power of two as a factor, V's as an exponent, and which of its
// eight groups of 16 keys are in pages (bits).
struct TileNote {
    float k_unit;
    float v_exp;
    uint32_t there;
    uint32_t pad;
};

template <int kReq>
struct TcLaunch {
    float* part_o;                       // [item][256][D] normalised
    float* part_lse;                     // [item][256] log2 domain
    uint32_t* tickets;                   // [unit], zero between launches
    PagedAttn<kReq> a;
};

// kind::f16 with A and B both f16 or both bf16, D fp32, A K-major, B K- or MN-major.
__host__ __device__ constexpr uint32_t idesc16(bool half, int m, int n, bool b_mn_major) {
    return (1u << 4) | (half ? 0u : 1u << 7 | 1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}

template <bool kHalf>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t r;
    if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two E4M3 codes times a scale, as f16.
__device__ __forceinline__ uint32_t scaled2(uint32_t codes, uint32_t scale2) {
    uint32_t h, r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(scale2));
    return r;
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The CTA's work: rows [row0, row0 + live) of request R's KV head hk, key tiles [j0, j0 + n).
struct Item {
    PagedReq R;
    int hk, sp, row0, live, j0, n, unit;
    int first, k_lo, k_hi;               // the first row's last key; keys that some row sees: [k_lo, k_hi)
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
    const int G = P.hq / P.hkv, n_rows = w.R.nq * G, pairs = (n_rows + kPair - 1) / kPair;
    int i = blockIdx.x - w.R.item0;
    // the last rows first: they see the most keys
    w.hk = i % P.hkv;
    i /= P.hkv;
    w.sp = i % w.R.splits;
    const int pr = pairs - 1 - i / w.R.splits;
    w.unit = w.R.unit0 + pr * P.hkv + w.hk;
    w.row0 = pr * kPair;
    w.live = min(kPair, n_rows - w.row0);
    const int before = w.R.n_keys - w.R.nq;
    w.first = before + w.row0 / G;
    w.k_hi = before + (w.row0 + w.live - 1) / G + 1;
    w.k_lo = P.window ? max(0, w.first - P.window + 1) : 0;
    const int t_lo = w.k_lo / BN, t_n = max(0, (w.k_hi + BN - 1) / BN - t_lo);
    w.j0 = t_lo + (int)((int64_t)t_n * w.sp / w.R.splits);
    w.n = t_lo + (int)((int64_t)t_n * (w.sp + 1) / w.R.splits) - w.j0;
    return w;
}

// ------------------------------------------------------------------ loaders

// 128 threads bring K and V tiles, K one stage ahead: rows thread / kChunks + kStep * i, one 16-byte
// chunk of each.
template <int D, bool kCodes, int kReq>
__device__ __forceinline__ void load_tiles(const PagedAttn<kReq>& P, const Item& w, int thread, uint32_t sK, uint32_t sV,
                                           uint32_t bars, TileNote* notes, volatile uint32_t* abort) {
    constexpr int EB = kCodes ? 1 : 2;
    constexpr int kChunks = D * EB / 16, kStep = 128 / kChunks, kPasses = kChunks;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int lane = thread % 32, chunk = thread % kChunks, row_t = thread / kChunks;
    const int ps = P.pg.page_shift;
    const int32_t* const table = P.pg.table + (int64_t)w.R.row * P.pg.table_stride;
    const int64_t head = ((int64_t)w.hk << ps);                  // rows of a page before the head's
    // page of 16-key group `lane` (0..7) of a tile; -1 for none
    auto look_up = [&](int j) {
        const int key = (w.j0 + j) * BN + (lane & 7) * 16;
        int page = -1;
        if (j < w.n && key < w.k_hi) {
            page = __ldg(table + (key >> ps));
            if (page < 0 || page >= P.pg.n_pages) {
                if (thread < 8) atomicOr(P.err, 1);
                page = -1;
            }
        }
        return page;
    };
    // element offset of the thread's chunk of row `row` of a tile, and whether the row counts
    auto row_at = [&](int j, int row, int pages, int64_t& at, int64_t& sat) {
        const int page = __shfl_sync(0xffffffffu, pages, row >> 4);
        const int key = (w.j0 + j) * BN + row;
        const int64_t in_page = head + (key & ((1 << ps) - 1));
        at = (int64_t)page * P.pg.page_stride + in_page * D + chunk * (16 / EB);
        sat = (int64_t)page * P.pg.scale_stride + in_page;
        return page >= 0 && key < w.k_hi && key >= w.k_lo;
    };
    // where 8 channels (16 bytes) from channel 8 * q on of row `row` lie in a tile
    auto place = [](int row, int q) { return (uint32_t)((q >> 3) * (BN * 128) + row * 128 + (((q & 7) ^ (row & 7)) << 4)); };
    auto note = [&](int j, int pages, float k_unit, float v_exp) {
        const uint32_t there = __ballot_sync(0xffffffffu, pages >= 0) & 0xffu;
        if (thread == 0) notes[j & (kUnits - 1)] = TileNote{k_unit, v_exp, there, 0u};
    };
    int pages = look_up(0);
    if constexpr (kCodes) {
        // a row's codes wait in registers while the other operand's tile is converted
        uint4 rk[kPasses], rv[kPasses];
        float sk = 0.f, sv = 0.f, sk4 = 0.f, sv4 = 0.f;          // the lane's row's scale; the largest of four others
        const uint8_t* const pk = static_cast<const uint8_t*>(P.pg.k);
        const uint8_t* const pv = static_cast<const uint8_t*>(P.pg.v);
        constexpr int kRowsW = 32 / kChunks;                     // rows of a warp in a pass
        auto fetch = [&](const uint8_t* base, const float* scales, int j, int pg, uint4 (&raw)[kPasses], float& mine, float& top) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                int64_t at, sat;
                const bool ok = row_at(j, row_t + kStep * i, pg, at, sat);
                raw[i] = ok ? __ldg(reinterpret_cast<const uint4*>(base + at)) : make_uint4(0u, 0u, 0u, 0u);
            }
            // scales: lane i * kRowsW + r has that of the warp's row r of pass i; the tile's largest comes
            // from four rows a lane (32 lanes have all 128)
            int64_t at, sat;
            const int row = (thread / 32) * kRowsW + lane % kRowsW + kStep * (lane / kRowsW);
            mine = row_at(j, row, pg, at, sat) ? __ldg(scales + sat) : 0.f;
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (row_at(j, lane + 32 * i, pg, at, sat)) {
                    const uint32_t b = __float_as_uint(__ldg(scales + sat)) & 0x7fffffffu;
                    if (b < 0x7f800000u) m = max(m, b);
                }
            }
            top = __uint_as_float(m);
        };
        auto unit_of = [&](float top) {                          // every scale of the tile is below 2^unit
            const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
            return max(-100, min(100, (int)(m >> 23) - 126));
        };
        auto convert = [&](uint32_t tile, const uint4 (&raw)[kPasses], float mine, int unit) {
            const float s = mine * exp2f((float)-unit);
            const uint32_t s2 = pack16<true>(s, s);
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int row = row_t + kStep * i;
                const uint32_t f = __shfl_sync(0xffffffffu, s2, i * kRowsW + lane / kChunks);
                const uint32_t x[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    h[2 * e] = scaled2(x[e], f);
                    h[2 * e + 1] = scaled2(x[e] >> 16, f);
                }
                sts128_(tile + place(row, 2 * chunk), make_uint4(h[0], h[1], h[2], h[3]));
                sts128_(tile + place(row, 2 * chunk + 1), make_uint4(h[4], h[5], h[6], h[7]));
            }
        };
        if (w.n > 0) {
            fetch(pk, P.pg.k_scale, 0, pages, rk, sk, sk4);
            fetch(pv, P.pg.v_scale, 0, pages, rv, sv, sv4);
        }
        for (int j = 0; j < w.n; ++j) {
            const int next = look_up(j + 1);
            const int uk = unit_of(sk4), uv = unit_of(sv4);
            note(j, pages, exp2f((float)uk), (float)uv);
            const int ks = j % kK, vs = j % kV;
            if (j >= kK) mbar_wait(bar(kBarKE + ks), (uint32_t)(j / kK - 1) & 1u, P.err, abort);
            convert(sK + ks * Tc<D>::kTile, rk, sk, uk);
            fence_proxy_async();
            mbar_arrive(bar(kBarKF + ks));
            if (j + 1 < w.n) fetch(pk, P.pg.k_scale, j + 1, next, rk, sk, sk4);
            if (j >= kV) mbar_wait(bar(kBarVE + vs), (uint32_t)(j / kV - 1) & 1u, P.err, abort);
            convert(sV + vs * Tc<D>::kTile, rv, sv, uv);
            fence_proxy_async();
            mbar_arrive(bar(kBarVF + vs));
            if (j + 1 < w.n) fetch(pv, P.pg.v_scale, j + 1, next, rv, sv, sv4);
            pages = next;
        }
    } else {
        using T = __nv_bfloat16;
        auto fetch = [&](const void* base, uint32_t tile, int j, int pg) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int row = row_t + kStep * i;
                int64_t at, sat;
                const bool ok = row_at(j, row, pg, at, sat);
                cp_async16_or_zero(tile + place(row, chunk), static_cast<const T*>(base) + (ok ? at : 0), ok);
            }
            cp_async_commit();
        };
        // three tiles on their way: K(j), V(j), K(j + 1); one is handed over when the next two are asked for
        auto hand_over = [&](int f) {
            fence_proxy_async();
            mbar_arrive(bar(f));
        };
        for (int j = 0; j < w.n; ++j) {
            const int next = look_up(j + 1);
            note(j, pages, 1.f, 0.f);
            const int ks = j % kK, vs = j % kV;
            if (j >= kK) mbar_wait(bar(kBarKE + ks), (uint32_t)(j / kK - 1) & 1u, P.err, abort);
            fetch(P.pg.k, sK + ks * Tc<D>::kTile, j, pages);
            if (j > 0) {
                cp_async_wait<2>();
                hand_over(kBarKF + (j - 1) % kK);
            }
            if (j >= kV) mbar_wait(bar(kBarVE + vs), (uint32_t)(j / kV - 1) & 1u, P.err, abort);
            fetch(P.pg.v, sV + vs * Tc<D>::kTile, j, pages);
            if (j > 0) {
                cp_async_wait<2>();
                hand_over(kBarVF + (j - 1) % kV);
            }
            pages = next;
        }
        if (w.n > 0) {
            cp_async_wait<1>();
            hand_over(kBarKF + (w.n - 1) % kK);
            cp_async_wait<0>();
            hand_over(kBarVF + (w.n - 1) % kV);
        }
    }
}

// ------------------------------------------------------------------ products

// Issue order per key tile: PV_A(j - 1), S_A(j), PV_B(j - 1), S_B(j): a tile's next scores follow the
// product that read the weights they overwrite, and each tile's softmax runs beside the other's products.
template <int D, bool kHalf>
__device__ __forceinline__ void issue_products(uint32_t tmem, uint32_t sQ, uint32_t sK, uint32_t sV, uint32_t bars, int n, bool has_b,
                                               int32_t* err, volatile uint32_t* abort) {
    constexpr uint32_t idS = idesc16(kHalf, BM, BN, false), idO = idesc16(kHalf, BM, D, true);
    constexpr uint64_t kTileDesc = (uint64_t)(Tc<D>::kTile >> 4);
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto wait = [&](int i, uint32_t parity) {
        mbar_wait(bar(i), parity, err, abort);
        tc_fence_after();
    };
    const uint64_t dQa = sw128_desc(sQ, 16, 1024), dQb = sw128_desc(sQ + Tc<D>::kTile, 16, 1024);
    const uint64_t dK0 = sw128_desc(sK, 16, 1024), dV0 = sw128_desc(sV, Tc<D>::kHalf, 1024);
    auto scores = [&](uint64_t dq, uint64_t dk, uint32_t d) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t off = (uint64_t)(((kk >> 2) * Tc<D>::kHalf + (kk & 3) * 32) >> 4);
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
    wait(kBarQ, 0);
    wait(kBarKF, 0);
    scores(dQa, dK0, tSa);
    mma_commit(bar(kBarS));
    if (has_b) {
        scores(dQb, dK0, tSb);
        mma_commit(bar(kBarS + 1));
    }
    mma_commit(bar(kBarKE));
    for (int j = 1; j <= n; ++j) {
        const bool more = j < n;
        if (++ks == kK) {
            ks = 0;
            kp ^= 1u;
        }
        const uint64_t dk = dK0 + (uint64_t)ks * kTileDesc, dv = dV0 + (uint64_t)vs * kTileDesc;
        const uint32_t acc = j > 1 ? 1u : 0u, pp = (uint32_t)(j - 1) & 1u;
        wait(kBarP, pp);
        wait(kBarVF + vs, vp);
        values(tSa, dv, tOa, acc);
        if (more) {
            wait(kBarKF + ks, kp);
            scores(dQa, dk, tSa);
            mma_commit(bar(kBarS));
        }
        if (has_b) {
            wait(kBarP + 1, pp);
            values(tSb, dv, tOb, acc);
        }
        mma_commit(bar(kBarVE + vs));
        if (more) {
            if (has_b) {
                scores(dQb, dk, tSb);
                mma_commit(bar(kBarS + 1));
            }
            mma_commit(bar(kBarKE + ks));
        }
        if (++vs == kV) {
            vs = 0;
            vp ^= 1u;
        }
    }
    mma_commit(bar(kBarO));
}

// ------------------------------------------------------------------ softmax

// The pair's queries, turned, into their tiles (128-byte swizzle), by the eight softmax warps: a warp
// takes a token, whose angles serve the heads of the group.
template <int D, bool kHalf, int kReq>
__device__ __forceinline__ void put_queries(const PagedAttn<kReq>& P, const Item& w, int warp, int lane, uint32_t sQ, float* s_rs) {
    using T = __nv_bfloat16;
    const int G = P.hq / P.hkv;
    constexpr int C = D / 64;                            // channels of each half a lane
    const int c = lane * C;
    auto put = [&](int row, int ch, float a, float b) {  // channels ch and ch + 1
        const uint32_t at = sQ + (row / BM) * Tc<D>::kTile + (ch >> 6) * Tc<D>::kHalf + (row % BM) * 128 +
                            ((((ch >> 3) & 7) ^ (row & 7)) << 4) + (ch & 7) * 2;
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(pack16<kHalf>(a, b)) : "memory");
    };
    const int tok0 = w.row0 / G, tok1 = (w.row0 + w.live - 1) / G;
    for (int tk = tok0 + warp; tk <= tok1; tk += 8) {
        float2 cs[C];
        const int64_t t = w.R.q0 + tk;
        if (P.turn) {
            const int64_t pos = __ldg(P.turn + t);
#pragma unroll
            for (int e = 0; e < C; ++e) cs[e] = turn_cs(P.rope.turn[c + e], pos);
        }
        const int r0 = max(tk * G, w.row0), r1 = min((tk + 1) * G, w.row0 + w.live);
        const T* q = static_cast<const T*>(P.q) + t * P.q_stride + (int64_t)w.hk * G * D + c;
#pragma unroll 4
        for (int rr = r0; rr < r1; ++rr) {
            const T* p = q + (rr - tk * G) * D;
            float lo[C], hi[C];
#pragma unroll
            for (int e = 0; e < C; ++e) {
                lo[e] = static_cast<float>(p[e]);
                hi[e] = static_cast<float>(p[D / 2 + e]);
                if (P.turn) rotate1(lo[e], hi[e], cs[e], lo[e], hi[e]);
            }
            float back = 1.f;
            if constexpr (kHalf) {       // the row's largest value to [2^14, 2^15); zero and non-finite rows as they are
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < C; ++e) top = max(top, max(__float_as_uint(lo[e]) & 0x7fffffffu, __float_as_uint(hi[e]) & 0x7fffffffu));
                top = __reduce_max_sync(0xffffffffu, top);
                const int ex = (int)(top >> 23) - 127;
                if (top < 0x7f800000u && ex > -100) {
                    const float f = exp2f((float)(14 - ex));
                    back = exp2f((float)(ex - 14));
#pragma unroll
                    for (int e = 0; e < C; ++e) {
                        lo[e] *= f;
                        hi[e] *= f;
                    }
                }
            }
            const int row = rr - w.row0;
            if (lane == 0) s_rs[row] = back * P.scale_log2;
            if constexpr (C == 2) {
                put(row, c, lo[0], lo[1]);
                put(row, D / 2 + c, hi[0], hi[1]);
            } else {
                const float y0 = __shfl_down_sync(0xffffffffu, lo[0], 1), y1 = __shfl_down_sync(0xffffffffu, hi[0], 1);
                if (!(lane & 1)) {
                    put(row, c, lo[0], y0);
                    put(row, D / 2 + c, hi[0], y1);
                }
            }
        }
    }
    // rows of no query: zero, so that what they hold is a number
    for (int row = w.live + warp; row < kPair; row += 8) {
        if (lane == 0) s_rs[row] = P.scale_log2;
        for (int ch = 2 * lane; ch < D; ch += 64) put(row, ch, 0.f, 0.f);
    }
}

// One softmax thread: row r of tile x over the CTA's key tiles, then its output.
template <int D, bool kCodes, int kReq>
__device__ __forceinline__ void softmax_rows(const TcLaunch<kReq>& X, const Item& w, uint32_t tmem, uint32_t bars, int x, int quad, int lane,
                                             const TileNote* notes, const float* s_rs, volatile uint32_t* abort) {
    using T = __nv_bfloat16;
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
    const float rs = s_rs[row];
    float ref = -CUDART_INF_F, l = 0.f;
    for (int j = 0; j < w.n; ++j) {
        mbar_wait(bar(kBarS + x), (uint32_t)j & 1u, P.err, abort);
        tc_fence_after();
        uint32_t sv[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(colS + c * 32, sv[c]);
        const TileNote nt = notes[j & (kUnits - 1)];
        const float f = kCodes ? rs * nt.k_unit : rs, ve = kCodes ? nt.v_exp : 0.f;
        tmem_ld_wait();
        const int key0 = (w.j0 + j) * BN;
        if (key0 + BN - 1 > end || key0 <= start || nt.there != 0xffu) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const int key = key0 + c * 32 + e;
                    if (key > end || key <= start || !(nt.there >> (2 * c + e / 16) & 1u)) sv[c][e] = __float_as_uint(-CUDART_INF_F);
                }
        }
        float top4[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float m = fmaxf(__uint_as_float(sv[c][0]), __uint_as_float(sv[c][1]));
#pragma unroll
            for (int e = 2; e < 32; e += 2) m = fmax3(m, __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
            top4[c] = m;
        }
        const float top = fmaf(fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])), f, ve);
        // the reference moves only when weights would pass 2^8: a rescale of O reads and writes it all
        const bool moves = top > ref + 8.0f;
        const float now = moves ? top : ref;
        const float alpha = moves ? ex2(ref - now) : 1.0f;
        const float base = now == -CUDART_INF_F ? 0.f : now;     // nothing seen yet
        if (j >= 1 && __any_sync(0xffffffffu, moves)) {
            // scores of tile j are complete, so is every product before them: O may be scaled
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
                uint32_t ov[16];
                tmem_ld16(colO + c * 16, ov);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
                tmem_st16(colO + c * 16, ov);
            }
        }
        float ps[4] = {0.f, 0.f, 0.f, 0.f};
        const float off = ve - base;
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
                pk[i] = pack16<kCodes>(a0, a1);
            }
            tmem_st16(colS + c * 16, pk);
        }
        tmem_st_wait();
        const float sum = (ps[0] + ps[1]) + (ps[2] + ps[3]);
        l = l * alpha + (kCodes ? sum * ex2(-ve) : sum);
        ref = now;
        tc_fence_before();
        mbar_arrive(bar(kBarP + x));
    }
    if (w.n > 0) {
        mbar_wait(bar(kBarO), 0u, P.err, abort);
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
    float fin = 0.f;                     // zero, or NaN where O is not finite
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
            fin = fmaf(__uint_as_float(ov[e]), 0.f, fin);
            ov[e] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(ov[e]) * inv);
        }
        if (!there) continue;
        if (whole) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t o8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o8[e] = pack16<false>(__uint_as_float(ov[16 * k + 2 * e]), __uint_as_float(ov[16 * k + 2 * e + 1]));
                if (wide) {
                    stg256(orow + c * 32 + k * 16, o8);
                } else {
                    *reinterpret_cast<uint4*>(orow + c * 32 + k * 16) = make_uint4(o8[0], o8[1], o8[2], o8[3]);
                    *reinterpret_cast<uint4*>(orow + c * 32 + k * 16 + 8) = make_uint4(o8[4], o8[5], o8[6], o8[7]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                *reinterpret_cast<uint4*>(prow + c * 32 + k * 4) = make_uint4(ov[4 * k], ov[4 * k + 1], ov[4 * k + 2], ov[4 * k + 3]);
        }
    }
    if (there) {
        if (!whole) X.part_lse[(int64_t)blockIdx.x * kPair + row] = lse2;
        else if (P.lse) P.lse[(int64_t)h * P.n_tokens + tok] = lse2 * 0.69314718055994531f;
    }
    // Rows whose O is not finite though their weights' sum is: a value that is not finite may belong to
    // keys that the row does not see (0 times it is NaN).  Those rows again, key by key, in fp32.
    uint32_t bad = __ballot_sync(0xffffffffu, there && fin != 0.f && l < CUDART_INF_F);
    for (; bad; bad &= bad - 1) {
        const int i = __ffs(bad) - 1, rr = w.row0 + x * BM + quad * 32 + i;
        const int last = w.R.n_keys - w.R.nq + rr / G;
        const int lo = max(w.j0 * BN, P.window ? last - P.window + 1 : 0), hi = min((w.j0 + w.n) * BN, last + 1);
        const int64_t t = w.R.q0 + rr / G;
        const int hh = w.hk * G + rr % G;
        float q[D / 32], o[D / 32], m, sum;
        lane_query<T, D>(P, t, hh, lane, q);
        row_attend<T, D, kCodes>(P, q, w.R.row, w.hk, lo, hi, 1, lane, m, sum, o);
        const float iv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
            const int ch = lane * (D / 32) + e;
            if (whole) static_cast<T*>(P.out)[(t * P.hq + hh) * D + ch] = static_cast<T>(o[e] * iv);
            else X.part_o[((int64_t)blockIdx.x * kPair + rr - w.row0) * D + ch] = o[e] * iv;
        }
        if (!whole && lane == 0) X.part_lse[(int64_t)blockIdx.x * kPair + rr - w.row0] = sum == 0.f ? -CUDART_INF_F : m + log2f(sum);
    }
}

// ------------------------------------------------------------------ kernel

template <int D, bool kCodes, int kReq>
__global__ void __launch_bounds__(kThreads, 1) paged_tc_kernel(const __grid_constant__ TcLaunch<kReq> X) {
    const PagedAttn<kReq>& P = X.a;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t s_last;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sQ = smem_u32(smem), sK = sQ + 2 * Tc<D>::kTile, sV = sK + kK * Tc<D>::kTile;
    const uint32_t bars = sV + kV * Tc<D>::kTile;
    uint8_t* const tail = smem + (size_t)(2 + kK + kV) * Tc<D>::kTile + 8 * kBars;
    uint32_t* const slot = reinterpret_cast<uint32_t*>(tail);
    volatile uint32_t* const abort = slot + 1;
    TileNote* const notes = reinterpret_cast<TileNote*>(tail + 16);
    float* const s_rs = reinterpret_cast<float*>(tail + 16 + 16 * kUnits);
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Item w = find_item(P);
    const bool has_b = w.live > BM;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kK; ++s) {
            mbar_init(bar(kBarKF + s), 128);
            mbar_init(bar(kBarKE + s), 1);
        }
        for (int s = 0; s < kV; ++s) {
            mbar_init(bar(kBarVF + s), 128);
            mbar_init(bar(kBarVE + s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kBarS + i), 1);
            mbar_init(bar(kBarP + i), 128);
        }
        mbar_init(bar(kBarO), 1);
        mbar_init(bar(kBarQ), 256);
        *abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;

    if (warp < 4) {
        load_tiles<D, kCodes>(P, w, threadIdx.x, sK, sV, bars, notes, abort);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        put_queries<D, kCodes>(P, w, warp - 4, lane, sQ, s_rs);
        fence_proxy_async();
        asm volatile("bar.sync 1, 256;" ::: "memory");           // (the row factors, too)
        mbar_arrive(bar(kBarQ));
        const int x = warp >= 8;
        if (x == 0 || has_b) softmax_rows<D, kCodes>(X, w, tmem, bars, x, warp & 3, lane, notes, s_rs, abort);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
        if (warp == 12 && lane == 0 && w.n > 0)
            issue_products<D, kCodes>(tmem, sQ, sK, sV, bars, w.n, has_b, P.err, abort);
    }

    tc_fence_before();
    if (w.R.splits > 1) __threadfence();                         // the partials, before the ticket
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
    if (w.R.splits == 1) return;
    if (threadIdx.x == 0) {
        const uint32_t t = atomicAdd(X.tickets + w.unit, 1u);
        s_last = t == (uint32_t)w.R.splits - 1;
        if (s_last) X.tickets[w.unit] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    // the unit's stretches joined: items of stretch k are hkv apart
    const int G = P.hq / P.hkv, S = w.R.splits;
    const int64_t item0 = (int64_t)blockIdx.x - (int64_t)w.sp * P.hkv;
    for (int i = threadIdx.x; i < w.live * (D / 4); i += kThreads) {
        const int row = i / (D / 4), f = i % (D / 4);
        float top = -CUDART_INF_F, sum = 0.f;
        for (int k = 0; k < S; ++k) top = fmaxf(top, __ldcg(X.part_lse + (item0 + (int64_t)k * P.hkv) * kPair + row));
        const float base = top == -CUDART_INF_F ? 0.f : top;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < S; ++k) {
            const int64_t at = (item0 + (int64_t)k * P.hkv) * kPair + row;
            const float a = ex2(__ldcg(X.part_lse + at) - base);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(X.part_o + at * D + 4 * f));
            sum += a;
            o.x = fmaf(y.x, a, o.x);
            o.y = fmaf(y.y, a, o.y);
            o.z = fmaf(y.z, a, o.z);
            o.w = fmaf(y.w, a, o.w);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t tok = w.R.q0 + (w.row0 + row) / G;
        const int h = w.hk * G + (w.row0 + row) % G;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.out) + (tok * P.hq + h) * D + 4 * f) =
            make_uint2(pack16<false>(o.x * inv, o.y * inv), pack16<false>(o.z * inv, o.w * inv));
        if (f == 0 && P.lse) P.lse[(int64_t)h * P.n_tokens + tok] = sum == 0.f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

template <int D, bool kCodes, int kReq>
cudaError_t launch(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    static PerDevice<cudaError_t> smem_set;
    const auto kernel = paged_tc_kernel<D, kCodes, kReq>;
    cudaError_t e = opt_in_smem(smem_set, (const void*)kernel, Tc<D>::kSmem);
    if (e != cudaSuccess) return e;
    for (int b0 = 0; b0 < n; b0 += kReq) {
        const int nb = std::min(n - b0, kReq);
        TcLaunch<kReq> X;
        fill_paged(X.a, c, D, req + b0, nb);
        const int slots = device_sms(), G = c.hq / c.hkv;
        auto pairs_of = [&](const PagedReq& q) { return (q.nq * G + kPair - 1) / kPair; };
        auto tiles_of = [&](const PagedReq& q) {
            const int keys = c.window ? std::min(q.n_keys, c.window + std::min(q.nq, kPair / G + 1) + BN) : q.n_keys;
            return std::max(1, (keys + BN - 1) / BN);
        };
        // Keys are cut only where whole units would leave SMs without work, into stretches of eight
        // tiles and more (a stretch's partial is written and read again, 128 KB).
        int64_t units = 0, tiles = 0;
        for (int i = 0; i < nb; ++i) {
            units += (int64_t)pairs_of(X.a.req[i]) * c.hkv;
            tiles += (int64_t)pairs_of(X.a.req[i]) * c.hkv * tiles_of(X.a.req[i]);
        }
        int per = units >= slots ? 1 << 30 : std::max(8, (int)((tiles + slots - 1) / slots));
        auto count = [&](int p) {
            int64_t items = 0;
            for (int i = 0; i < nb; ++i) items += (int64_t)pairs_of(X.a.req[i]) * c.hkv * ((tiles_of(X.a.req[i]) + (int64_t)p - 1) / p);
            return items;
        };
        while (per < (1 << 20) && count(per) > slots) per += std::max(1, per / 16);
        int64_t items = 0;
        units = 0;
        bool split = false;
        for (int i = 0; i < nb; ++i) {
            PagedReq& q = X.a.req[i];
            q.splits = (int32_t)((tiles_of(q) + (int64_t)per - 1) / per);
            split = split || q.splits > 1;
            q.item0 = (int32_t)items;
            q.unit0 = (int32_t)units;
            units += (int64_t)pairs_of(q) * c.hkv;
            items += (int64_t)pairs_of(q) * c.hkv * q.splits;
        }
        X.part_o = X.part_lse = nullptr;
        X.tickets = nullptr;
        if (split) {
            void* p = nullptr;
            const size_t o_bytes = (size_t)items * kPair * D * 4;
            e = context_workspace(c.ctx, o_bytes + (size_t)items * kPair * 4, (size_t)units, &p, &X.tickets);
            if (e != cudaSuccess) return e;
            X.part_o = static_cast<float*>(p);
            X.part_lse = reinterpret_cast<float*>(static_cast<char*>(p) + o_bytes);
        }
        kernel<<<(unsigned)items, kThreads, Tc<D>::kSmem, s>>>(X);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool kCodes>
cudaError_t by_count(const PagedAttnCall& c, const PagedReq* req, int n, cudaStream_t s) {
    return n <= kPagedFew ? launch<D, kCodes, kPagedFew>(c, req, n, s) : launch<D, kCodes, kPagedMany>(c, req, n, s);
}

}  // namespace

cudaError_t launch_paged_tc(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    if (d == 128) return codes ? by_count<128, true>(c, req, n, s) : by_count<128, false>(c, req, n, s);
    return codes ? by_count<64, true>(c, req, n, s) : by_count<64, false>(c, req, n, s);
}

}  // namespace c2kv
