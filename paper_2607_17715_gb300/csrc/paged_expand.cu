// Pages as key tiles, for the attention of many query rows (paged_tc.cu): 128 keys of a KV head in f16,
// K and V each relative to a power of two of the tile's own.
//
// Why a pass of its own.  Every CTA of a head meets the same keys; converted there, each did the work
// again and its conversions took twice the time of its products.  And why f16: the products take one type
// for both operands, and queries turned by RoPE need more than bf16's 8 bits (a score's error of 2^-9 of
// its terms was two thirds of the output's whole error over long contexts).  f16 keeps 11 bits of queries,
// weights and E4M3 rows, and all 8 of bf16 values down to 2^-25 of their tile's largest (V's, by its common power: 2^-18 of
// a sample's).  What f16 lacks in range the powers of two hold.
//
// V's power of two is one for most tiles of a request's head, since a tile's weights lie that much lower in
// f16 where its own is smaller than others': with one row 2^10 times the others' the others' weights lost 10
// of their bits.  It leaves room for rows 2^12 above the largest of a sample of 32 rows; tiles of larger values,
// or of values too small for it, have their own.
//
// Values of V that are not finite become zero here, and their rows are noted: a query that does not see such a
// row is not touched by it (0 times it is NaN), and one that does takes them in at the end (paged_tc.cu).
//
// Bytes bound it: a page's read once, two written for each value.  Measured: 32768 rows of codes of 8 heads,
// 67 MB to 134 MB, in 39 us (5.2 TB/s).
#include "paged.cuh"
#include "ptx.cuh"
#include "vec16.cuh"

#include <algorithm>
#include <cuda_fp16.h>

namespace c2kv {
namespace {

constexpr int kExpandThreads = 256;

template <int kReq>
struct PagedExpand {
    PageView pg;
    KeyTiles to;
    int32_t* err;
    int32_t hkv;
    int32_t n;
    int32_t item0[kReq];         // tiles of the launch before request i's
    int32_t first;               // the launch's first tile in `to`
    int32_t row[kReq];           // its row of the table
    int32_t tile0[kReq];         // its first key tile
    int32_t key0[kReq];          // the first key that any query sees
    int32_t n_keys[kReq];
};

// The power of two above bits of a finite fp32 magnitude: every value is below 2^u.
__device__ __forceinline__ int above(uint32_t bits) { return max(-100, min(126, (int)(bits >> 23) - 126)); }

__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Binades above the sample's largest value that the common power of two of V leaves room for, and how far
// below it a tile's own may be: its largest value is then 2^-9, 16 bits above what f16 cuts off.
constexpr int kSampleRoom = 12, kSampleDepth = 24;

// K (z = 0) or V (1) of one tile and KV head a CTA, 16 values a thread and pass.
template <int D, bool kCodes, int kReq>
__global__ void __launch_bounds__(kExpandThreads) paged_expand_kernel(const __grid_constant__ PagedExpand<kReq> P) {
    constexpr int kChunks = D / 16, kStep = kExpandThreads / kChunks, kPasses = kTileKeys / kStep;   // rows a pass
    __shared__ uint32_t s_top[kExpandThreads / 32], s_there, s_sample;
    __shared__ uint8_t s_odd[kTileKeys];
    // the attention may be set up and turn its queries meanwhile: it waits for this grid before it reads tiles
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int r = 0;
    for (int hi = P.n; hi - r > 1;) {
        const int mid = (r + hi) >> 1;
        if (P.item0[mid] <= (int)blockIdx.x) r = mid;
        else hi = mid;
    }
    const int h = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const bool v = blockIdx.z != 0;
    const int key0 = (P.tile0[r] + (int)blockIdx.x - P.item0[r]) * kTileKeys;
    const int64_t tile = P.first + (int64_t)blockIdx.x;
    const int shift = P.pg.page_shift, size = 1 << shift;
    // page of 16-key group `lane` (0..7): -1 for none, or without a key that any query sees
    int page = -1;
    {
        const int key = key0 + (lane & 7) * 16;
        // (pages that a window has left behind may be gone from the table)
        if (key < P.n_keys[r] && ((key >> shift) + 1) << shift > P.key0[r]) {
            page = __ldg(P.pg.table + (int64_t)P.row[r] * P.pg.table_stride + (key >> shift));
            if (page < 0 || page >= P.pg.n_pages) {
                if (threadIdx.x < 8 && h == 0 && !v) atomicOr(P.err, 1);
                page = -1;
            }
        }
    }
    const uint32_t there = __ballot_sync(0xffffffffu, page >= 0) & 0xffu;
    const int chunk = threadIdx.x % kChunks;
    const void* const base = v ? P.pg.v : P.pg.k;
    const float* const scales = v ? P.pg.v_scale : P.pg.k_scale;
    uint4 raw[kPasses][kCodes ? 1 : 2];
    float scale[kPasses];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int row = threadIdx.x / kChunks + kStep * i, key = key0 + row;
        const int pg = __shfl_sync(0xffffffffu, page, row >> 4);
        const bool ok = pg >= 0 && key >= P.key0[r] && key < P.n_keys[r];
        const int64_t in_page = (int64_t)h * size + (key & (size - 1));
        const int64_t at = (int64_t)pg * P.pg.page_stride + in_page * D + chunk * 16;
        scale[i] = 0.f;
        if constexpr (kCodes) {
            raw[i][0] = ok ? ld16(static_cast<const uint8_t*>(base) + at) : make_uint4(0u, 0u, 0u, 0u);
            if (ok) scale[i] = __ldg(scales + (int64_t)pg * P.pg.scale_stride + in_page);
        } else {
            const __nv_bfloat16* const p = static_cast<const __nv_bfloat16*>(base) + at;
            raw[i][0] = ok ? ld16(p) : make_uint4(0u, 0u, 0u, 0u);
            raw[i][1] = ok ? ld16(p + 8) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // (V) magnitude bits of row `lane` of 32 spread over what is seen, the same for every tile of the request's head
    uint32_t sample = 0;
    if (v) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            bool odd = false;
            if constexpr (kCodes) {
                uint32_t* const w = reinterpret_cast<uint32_t*>(&raw[i][0]);
                if (!(fabsf(scale[i]) < INFINITY)) {
                    odd = true;
                    scale[i] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {            // codes 0x7f and 0xff are NaN
                    const uint32_t nan = ((w[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                    odd = odd || nan != 0u;
                    w[e] &= ~((nan >> 7) * 0xffu);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t* const w = reinterpret_cast<uint32_t*>(&raw[i][k]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {        // (an exponent of ones carries into the bit above it)
                        const uint32_t out = ((w[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                        odd = odd || out != 0u;
                        w[e] &= ~((out >> 15) * 0xffffu);
                    }
                }
            }
            const uint32_t all = __ballot_sync(0xffffffffu, odd);      // a row's threads lie next to one another
            if (chunk == 0) s_odd[threadIdx.x / kChunks + kStep * i] = (all >> (lane & ~(kChunks - 1)) & ((1u << kChunks) - 1u)) != 0u;
        }
    }
    if (v && warp == 0) {
        const int key = P.key0[r] + (int)((int64_t)(P.n_keys[r] - P.key0[r]) * lane / 32);
        const int pg = __ldg(P.pg.table + (int64_t)P.row[r] * P.pg.table_stride + (key >> shift));
        if (pg >= 0 && pg < P.pg.n_pages) {
            const int64_t in_page = (int64_t)h * size + (key & (size - 1));
            if constexpr (kCodes) {
                const uint32_t b = __float_as_uint(__ldg(scales + (int64_t)pg * P.pg.scale_stride + in_page)) & 0x7fffffffu;
                if (b < 0x7f800000u) sample = b;
            } else {                     // eight of its channels
                const uint4 x = ld16(static_cast<const __nv_bfloat16*>(base) + (int64_t)pg * P.pg.page_stride + in_page * D + lane * 8 % D);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = w[e] << 16 & 0x7fff0000u, hi = w[e] & 0x7fff0000u;
                    sample = max(sample, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                }
            }
        }
    }
    if constexpr (kCodes) {              // a row's values are at most 448 of its scale: the scales decide
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const uint32_t b = __float_as_uint(scale[i]) & 0x7fffffffu;
            top = max(top, b < 0x7f800000u ? b : 0u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t w[4] = {raw[i][k].x, raw[i][k].y, raw[i][k].z, raw[i][k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = w[e] << 16 & 0x7fff0000u, hi = w[e] & 0x7fff0000u;
                    top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                }
            }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s_top[warp] = top;
    if (v && warp == 0) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, sample);
        if (lane == 0) s_sample = m;
    }
    if (threadIdx.x == 0) s_there = there;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int w = 0; w < kExpandThreads / 32; ++w) top = max(top, s_top[w]);
    // 16-bit values to below 2^9, as codes times their relative scales are; V to below 2^15
    constexpr int kBits = kCodes ? 0 : 9;
    int unit = max(-100, above(top) - kBits);
    if (v) {                             // (from -90 on: the sum of weights takes 2^-unit, 2^16 of them a tile)
        unit = max(-90, above(top) - kBits - 6);
        const int common = s_sample == 0u ? 0 : max(-90, min(120, above(s_sample) - kBits - 6 + kSampleRoom));
        if (top == 0u || (s_sample != 0u && unit <= common && unit >= common - kSampleDepth)) unit = common;
    }
    const float inv = pow2i(-unit);
    if (threadIdx.x == 0) {
        float* const u = reinterpret_cast<float*>(P.to.unit + tile * P.hkv + h);
        u[v] = v ? (float)unit : pow2i(unit);
        if (h == 0 && !v) P.to.there[tile] = s_there;
    }
    if (v && warp == 0) {
        uint32_t odd[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) odd[k] = __ballot_sync(0xffffffffu, s_odd[32 * k + lane] != 0);
        if (lane == 0) P.to.odd[tile * P.hkv + h] = make_uint4(odd[0], odd[1], odd[2], odd[3]);
    }
    __half* const out = static_cast<__half*>(v ? P.to.v : P.to.k) + (tile * P.hkv + h) * kTileKeys * D + chunk * 16;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int row = threadIdx.x / kChunks + kStep * i;
        uint32_t y[8];
        if constexpr (kCodes) {
            const uint32_t w[4] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w};
            const float f = scale[i] * inv;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t a, b;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((uint16_t)w[e]));
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((uint16_t)(w[e] >> 16)));
                const float2 x = __half22float2(*reinterpret_cast<__half2*>(&a)), z = __half22float2(*reinterpret_cast<__half2*>(&b));
                y[2 * e] = half2_of(x.x * f, x.y * f);
                y[2 * e + 1] = half2_of(z.x * f, z.y * f);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t w[4] = {raw[i][k].x, raw[i][k].y, raw[i][k].z, raw[i][k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[4 * k + e] = half2_of(__uint_as_float(w[e] << 16) * inv, __uint_as_float(w[e] & 0xffff0000u) * inv);
            }
        }
        st16(out + row * D, make_uint4(y[0], y[1], y[2], y[3]));
        st16(out + row * D + 8, make_uint4(y[4], y[5], y[6], y[7]));
    }
}

template <int D, bool kCodes, int kReq>
cudaError_t launch_expand(const PagedExpandCall& c, cudaStream_t s) {
    int first = 0;
    for (int b0 = 0; b0 < c.n; b0 += kReq) {
        const int nb = std::min(c.n - b0, kReq);
        PagedExpand<kReq> P;
        P.pg = c.pg;
        P.to = c.to;
        P.err = c.err;
        P.hkv = c.hkv;
        P.n = nb;
        P.first = first;
        int items = 0;
        for (int i = 0; i < nb; ++i) {
            P.item0[i] = items;
            P.row[i] = c.req[b0 + i].row;
            P.tile0[i] = c.tile0[b0 + i];
            P.key0[i] = c.key0[b0 + i];
            P.n_keys[i] = c.req[b0 + i].n_keys;
            items += c.tiles[b0 + i];
        }
        first += items;
        if (items == 0) continue;
        paged_expand_kernel<D, kCodes, kReq><<<dim3(items, c.hkv, 2), kExpandThreads, 0, s>>>(P);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D>
cudaError_t by_format(const PagedExpandCall& c, bool codes, cudaStream_t s) {
    if (c.n <= kPagedFew) return codes ? launch_expand<D, true, kPagedFew>(c, s) : launch_expand<D, false, kPagedFew>(c, s);
    return codes ? launch_expand<D, true, kPagedMany>(c, s) : launch_expand<D, false, kPagedMany>(c, s);
}

}  // namespace

cudaError_t launch_paged_expand(const PagedExpandCall& c, int d, bool codes, cudaStream_t s) {
    return d == 128 ? by_format<128>(c, codes, s) : by_format<64>(c, codes, s);
}

}  // namespace c2kv
