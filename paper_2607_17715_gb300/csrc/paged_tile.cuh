// What the tcgen05 kernels of paged attention share (paged_tc.cu, paged_direct.cu): a CTA's work, its queries, which
// keys a row sees, values that are not finite, and the join of cut keys.
#pragma once

#include "paged.cuh"
#include "paged_row.cuh"
#include "per_device.cuh"
#include "ptx.cuh"
#include "rope.cuh"
#include "tcgen05.cuh"

#include <math_constants.h>

#include <type_traits>

namespace c2kv {
namespace {

constexpr int BM = 128;                  // rows of a query tile
constexpr int BN = 128;                  // keys of a tile

template <int D>
struct TileOf {
    static constexpr int kTile = BN * D * 2;               // bytes of a tile
    static constexpr int kHalf = BN * 128;                 // of its 64-channel block
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

// The CTA's work: rows [row0, row0 + live) of request R's KV head hk, at most kUnit of them, key tiles [j0, j0 + n).
struct Item {
    PagedReq R;
    int hk, sp, row0, live, j0, n;
    int k_lo, k_hi;                      // keys that some row sees: [k_lo, k_hi)
};

template <bool kTree, int kUnit, int kReq>
__device__ __forceinline__ Item find_item(const PagedAttn<kReq>& P, int item) {
    Item w;
    int r = 0;
    for (int hi = P.batch; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.req[mid].item0 <= item) r = mid;
        else hi = mid;
    }
    w.R = P.req[r];
    const int G = P.hq / P.hkv, n_rows = w.R.nq * G;
    int i = item - w.R.item0;
    // the last rows first: they see the most keys
    w.hk = i % P.hkv;
    i /= P.hkv;
    w.sp = i % w.R.splits;
    const int pr = w.R.tile0 + w.R.tiles - 1 - i / w.R.splits;
    w.row0 = pr * kUnit;
    w.live = min(kUnit, n_rows - w.row0);
    const int before = w.R.n_keys - w.R.nq;
    w.k_hi = before + (w.row0 + w.live - 1) / G + 1;
    w.k_lo = P.window ? max(0, before + (kTree ? 0 : w.row0 / G) - P.window + 1) : 0;    // (a tree's root has the least depth)
    const int t_lo = w.k_lo / BN, t_n = max(0, (w.k_hi + BN - 1) / BN - t_lo);
    w.j0 = t_lo + (int)((int64_t)t_n * w.sp / w.R.splits);
    w.n = t_lo + (int)((int64_t)t_n * (w.sp + 1) / w.R.splits) - w.j0;
    return w;
}

// The CTA's queries, turned, into their tiles (128-byte swizzle), by as many warps as they need, 32 rows
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

template <int D, int kRows = 32, int kReq>
__device__ __forceinline__ QueryRows<D> fetch_queries(const PagedAttn<kReq>& P, const Item& w, int warp, int lane, uint32_t sQ) {
    using T = __nv_bfloat16;
    using C = TileOf<D>;
    const int G = P.hq / P.hkv;
    const int r0 = warp * kRows, n = max(0, min(kRows, w.live - r0));
    const uint32_t tile = sQ + (r0 / BM) * C::kTile + (r0 % BM) * 128;
    // lane i knows where row i lies; a copy takes whole rows, 16 bytes a lane
    const int row = w.row0 + r0 + min(lane, max(0, n - 1)), tok = row / G;
    const int64_t at = (w.R.q0 + tok) * P.q_stride + ((int64_t)w.hk * G + row - tok * G) * D;
    constexpr int kChunks = D / 8, kStep = 32 / kChunks;
    const int q = lane % kChunks;
    const T* const base = static_cast<const T*>(P.q) + q * 8;
#pragma unroll
    for (int i0 = 0; i0 < kRows; i0 += kStep) {
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

template <int D, int kRows = 32, int kReq>
__device__ __forceinline__ void turn_queries(const PagedAttn<kReq>& P, const QueryRows<D>& k, int warp, int lane, uint32_t sQ, int8_t* s_back) {
    using C = TileOf<D>;
    constexpr int E = QueryRows<D>::E, kBatch = 8;       // rows in flight
    const int r0 = warp * kRows;
    const int c = lane * E, q0 = c >> 3, q1 = (D / 2 + c) >> 3;
    const uint32_t tile = sQ + (r0 / BM) * C::kTile + (r0 % BM) * 128;
    float2 cs[E];
    int pos_cs = __shfl_sync(0xffffffffu, k.pos, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) cs[e] = turn_cs_fast(k.turn[e], pos_cs);
    cp_async_wait<0>();
    __syncwarp();
#pragma unroll 1
    for (int i0 = 0; i0 < kRows; i0 += kBatch) {
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

// The keys that a row sees: up to its last one, in its window.
struct Before {
    int start, end;                      // (start, end]
    template <int kReq>
    __device__ __forceinline__ Before(const PagedAttn<kReq>& P, const Item& w, int tok) {
        end = w.R.n_keys - w.R.nq + tok;
        start = P.window ? end - P.window : -1;
    }
    __device__ __forceinline__ bool sees(int key) const { return key > start && key <= end; }
    // all of 128 keys from key0 on
    __device__ __forceinline__ bool sees_tile(int key0) const { return key0 + BN - 1 <= end && key0 > start; }
    // of 32 keys from key0 on, a bit each
    __device__ __forceinline__ uint32_t of32(int key0) const { return within(0xffffffffu, key0, start, end); }
};
// The same of a tree's node: the rows before the tree, and its way to the root, a bit a node (in local memory:
// few of a CTA's key tiles meet the tree).
struct Through {
    int start, before;
    uint32_t bits[kTreeWords];
    template <int kReq>
    __device__ __forceinline__ Through(const PagedAttn<kReq>& P, const Item& w, int tok) {
        before = w.R.n_keys - w.R.nq;
        start = -1;
#pragma unroll
        for (int i = 0; i < kTreeWords; ++i) bits[i] = 0u;
        if ((w.j0 + w.n) * BN > before || P.window) start = tree_bits(P.parent + w.R.q0, tok, before, P.window, P.err, bits);
    }
    __device__ __forceinline__ bool sees(int key) const { return tree_sees(key, before, start, bits); }
    __device__ __forceinline__ bool sees_tile(int key0) const { return key0 + BN <= before && key0 > start; }
    __device__ __forceinline__ uint32_t of32(int key0) const {
        uint32_t seen = key0 < before ? within(0xffffffffu, key0, start, before - 1) : 0u;
        const int j = key0 - before;                     // the node of the first key
        if (j > -32 && j < 0) seen |= bits[0] << -j;
        else if (j >= 0 && j < kTreeMost) seen |= __funnelshift_r(bits[j >> 5], j + 32 < kTreeMost ? bits[(j >> 5) + 1] : 0u, j & 31);
        return seen;
    }
};
// The same, a node's way walked when it is asked for: nothing is kept but its ends.
template <class Attn>
struct Climb {
    const Attn& P;
    int q0, start, before, tok;
    template <class F>
    __device__ __forceinline__ int way(int window, const F& f) const { return tree_way(P.parent + q0, tok, window, P.err, f); }
    __device__ __forceinline__ Climb(const Attn& P_, const Item& w, int tok_) : P(P_), q0(w.R.q0), start(-1), before(w.R.n_keys - w.R.nq), tok(tok_) {
        if (P.window) start = max(-1, min(before + way(P.window, [](int) {}) - P.window, before - 1));
    }
    __device__ __forceinline__ bool sees_tile(int key0) const { return key0 + BN <= before && key0 > start; }
    __device__ __forceinline__ bool sees(int key) const {
        bool seen = key < before && key > start;
        if (key >= before) way(P.window, [&](int j) { seen = seen || before + j == key; });
        return seen;
    }
    // of 64 keys from key0 on, a bit each
    __device__ __forceinline__ void of64(int key0, uint32_t& lo, uint32_t& hi) const {
        lo = key0 < before ? within(0xffffffffu, key0, start, before - 1) : 0u;
        hi = key0 + 32 < before ? within(0xffffffffu, key0 + 32, start, before - 1) : 0u;
        if (key0 + 64 <= before || key0 > before + tok) return;
        way(P.window, [&](int j) {
            const int at = before + j - key0;
            if (at >= 0 && at < 32) lo |= 1u << at;
            else if (at >= 32 && at < 64) hi |= 1u << (at - 32);
        });
    }
};
template <bool kTree>
using Sight = typename std::conditional<kTree, Through, Before>::type;

// Rows that see values of V which are not finite (bits of `bad`, a lane a row from row0 on): of a channel's
// infinities and NaN nothing is left but which there are, and nothing else matters there.  The warp looks the
// noted keys up once for all its rows.  (Computed again key by key, a chunk of 256 tokens over one such row
// of 8192 took 28 ms for 70 us.)
template <int D, bool kCodes, int kUnit, class S, class Launch>
__device__ __forceinline__ void take_in(const Launch& X, const Item& w, uint32_t bad, const S& sight, int row0, int lane, uint8_t* q_tiles) {
    using T = __nv_bfloat16;
    constexpr int E = D / 32;                                    // channels a lane, a byte each: 1 infinity, 2 minus it, 4 NaN
    constexpr uint32_t kNan = E == 4 ? 0x04040404u : 0x0404u;
    using Word = typename std::conditional<E == 4, uint32_t, uint16_t>::type;
    const auto& P = X.a;
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
                    uint32_t rows = __ballot_sync(0xffffffffu, sight.sees(key)) & bad;
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
        const int64_t at = whole ? ((w.R.q0 + rr / G) * (int64_t)P.hq + w.hk * G + rr % G) * D : ((int64_t)blockIdx.x * kUnit + row0 + i) * D;
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

// The stretches of cut keys joined: a row a thread, 512 / D rows of a unit a CTA, eight stretches' loads a thread on their
// way at once (one request of 8 KV heads has few units: with 32 rows a CTA, eight a thread and a stretch at a time, 32 CTAs took 54 us
// for 64 rows over 30000 where these take 42, attention and all; 32 nodes over 120000 rows took 6 more with 8 rows a CTA).
constexpr int kJoinThreads = 128;
__host__ __device__ constexpr int join_rows(int d) { return kJoinThreads * 4 / d; }

template <int D, int kUnit, bool kTree, class Launch>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const __grid_constant__ Launch X) {
    const auto& P = X.a;
    extern __shared__ float weight[];                            // [stretch][row]
    constexpr int kJoinRows = join_rows(D), kSlices = kUnit / kJoinRows;
    const int u = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
    int r = 0;
    while (r + 1 < P.batch && P.req[r + 1].unit0 <= u) ++r;      // (entries that are not cut have no units)
    asm volatile("griddepcontrol.wait;" ::: "memory");           // the partials are complete and visible
    const PagedReq R = P.req[r];
    const int G = P.hq / P.hkv, S = R.splits, k0 = u - R.unit0, hk = k0 % P.hkv, pr = R.tile0 + k0 / P.hkv;
    const int first = slice * kJoinRows, live = min(kJoinRows, R.nq * G - pr * kUnit - first);
    if (live <= 0) return;
    // items of the unit's stretch k: see find_item
    const int64_t item0 = R.item0 + ((int64_t)(R.tile0 + R.tiles - 1 - pr) * S) * P.hkv + hk;
    for (int i = threadIdx.x; i < S * kJoinRows; i += kJoinThreads) {
        if (i % kJoinRows < live) weight[i] = ld_after_l2(X.part_lse + (item0 + (int64_t)(i / kJoinRows) * P.hkv) * kUnit + first + i % kJoinRows);
    }
    __syncthreads();
    for (int row = threadIdx.x; row < live; row += kJoinThreads) {
        float top = -CUDART_INF_F, sum = 0.f;
        for (int k = 0; k < S; ++k) top = fmaxf(top, weight[k * kJoinRows + row]);
        const float base = top == -CUDART_INF_F ? 0.f : top;
        for (int k = 0; k < S; ++k) sum += ex2(weight[k * kJoinRows + row] - base);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const float none = sum == 0.f ? of_no_weight<kTree>(P, R, (pr * kUnit + first + row) / G) : 0.f;
        for (int k = 0; k < S; ++k) weight[k * kJoinRows + row] = ex2(weight[k * kJoinRows + row] - base) * inv + none;
        if (P.lse) {
            const int all = pr * kUnit + first + row;
            P.lse[(int64_t)(hk * G + all % G) * P.n_tokens + R.q0 + all / G] = sum == 0.f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
        }
    }
    __syncthreads();
    constexpr int kLines = D / 4, kBatch = 8;
    const int f = threadIdx.x % kLines, row = threadIdx.x / kLines;
    if (row >= live) return;
    const float* const from = X.part_o + (item0 * kUnit + first + row) * D + 4 * f;
    const int64_t step = (int64_t)P.hkv * kUnit * D;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < S; k0 += kBatch) {
        float4 y[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) y[b] = ld_after_l2(reinterpret_cast<const float4*>(from + min(k0 + b, S - 1) * step));
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (k0 + b >= S) break;
            const float a = weight[(k0 + b) * kJoinRows + row];
            o.x = fmaf(y[b].x, a, o.x);
            o.y = fmaf(y[b].y, a, o.y);
            o.z = fmaf(y[b].z, a, o.z);
            o.w = fmaf(y[b].w, a, o.w);
        }
    }
    const int all = pr * kUnit + first + row;
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.out) + ((int64_t)(R.q0 + all / G) * P.hq + hk * G + all % G) * D + 4 * f) =
        make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
}

}  // namespace
}  // namespace c2kv
