// Rows moved within pages, in every layer of a model: the rows of the drafted tokens that a walk kept, moved
// together (c2kv_paged_keep), and the page that a beam writes next, copied where several beams would write it
// (c2kv_paged_reorder).
//
// Both read and write what they move once, and are bound by that where it is much (beams), by the launch and the
// chain table, page, row where it is not (kept rows).  Measured: 16 x 8 beams, 32 layers of 8 heads of 8-bit rows, 158 MB
// read and written in 32 us (4.9 TB/s); the kept rows of 32 trees in 32 layers 10 us, of which the host takes most.
#include "paged.cuh"
#include "per_device.cuh"

#include <algorithm>

namespace c2kv {
namespace {

constexpr int kRowThreads = 256;

template <int kReq, int kLayers>
struct RowsLaunch {
    PageView pg;             // geometry and table
    LayerPages layer[kLayers];
    int32_t* err;
    const int32_t* path;
    const int32_t* n_accepted;
    const int32_t* parent;
    int32_t* table_out;
    int64_t table_out_stride;
    int32_t b0;              // the launch's first request
    int32_t hkv;
    int32_t row_bytes;
    int32_t table_width;
    int32_t width;
    int32_t first_layers;    // its layers are the call's first: the tables are its to write
    int32_t ptr[kReq + 1];   // (kept rows) tokens of request b0 + r
    int32_t rows[kReq];      // their first row, or (beams) the requests' rows
};

__device__ __forceinline__ bool page_there(const PageView& pg, int page) { return page >= 0 && page < pg.n_pages; }

// Kept rows.  CTA: a request and a layer.  A thread owns 16 bytes of every row (or a head's scale) and moves them in the
// path's order, eight rows at a time: a row is read before any thread of its column writes it, since path[i] >= i rises.
template <int kReq, int kLayers>
__global__ void __launch_bounds__(kRowThreads) paged_keep_kernel(const __grid_constant__ RowsLaunch<kReq, kLayers> P) {
    __shared__ int2 s_from[kTreeMost], s_to[kTreeMost];   // page and row in it; page -1: not moved
    __shared__ int s_bad;
    const int r = blockIdx.x, lo = P.ptr[r], n = P.ptr[r + 1] - lo;
    after_kernels_before();
    if (n == 0) return;
    if (threadIdx.x == 0) s_bad = n;
    __syncthreads();
    int kept = ld_after(P.n_accepted + P.b0 + r) + 1;
    if (kept < 1 || kept > n) {
        if (threadIdx.x == 0) atomicOr(P.err, 1);
        return;
    }
    const int size = 1 << P.pg.page_shift;
    const int32_t* const table = P.pg.table + (int64_t)(P.b0 + r) * P.pg.table_stride;
    for (int i = threadIdx.x; i < kept; i += kRowThreads) {
        const int at = ld_after(P.path + lo + i), last = i ? ld_after(P.path + lo + i - 1) : -1;
        if (at <= last || at >= n) {
            atomicOr(P.err, 1);
            atomicMin(&s_bad, i);
            continue;
        }
        const int a = P.rows[r] + at, b = P.rows[r] + i;
        int from = -1, to = -1;
        if (at != i) {
            from = ld_after(table + (a >> P.pg.page_shift));
            to = ld_after(table + (b >> P.pg.page_shift));
            if (!page_there(P.pg, from) || !page_there(P.pg, to)) {
                atomicOr(P.err, 1);
                from = -1;
            }
        }
        s_from[i] = make_int2(from, a & (size - 1));
        s_to[i] = make_int2(to, b & (size - 1));
    }
    __syncthreads();
    kept = min(kept, s_bad);
    const LayerPages L = P.layer[blockIdx.y];
    const int chunks = P.row_bytes / 16, columns = P.hkv * chunks;
    auto move = [&](auto* base, int64_t stride, int head, int per_row, int in_row) {   // elements of one column
        using E = typename std::remove_reference<decltype(*base)>::type;
        constexpr int kBatch = 8;
        for (int i0 = 0; i0 < kept; i0 += kBatch) {
            E x[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k >= kept) break;
                const int2 f = s_from[i0 + k];
                if (f.x >= 0) x[k] = base[f.x * stride + ((int64_t)(head << P.pg.page_shift) + f.y) * per_row + in_row];
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k >= kept) break;
                const int2 t = s_to[i0 + k];
                if (s_from[i0 + k].x >= 0) base[t.x * stride + ((int64_t)(head << P.pg.page_shift) + t.y) * per_row + in_row] = x[k];
            }
        }
    };
    const int64_t stride16 = P.pg.page_stride;               // in 16-byte lines (see the launch)
    for (int i = threadIdx.x; i < 2 * columns; i += kRowThreads) {
        const int c = i % columns;
        move(static_cast<uint4*>(i < columns ? L.k : L.v), stride16, c / chunks, chunks, c % chunks);
    }
    if (L.k_scale)
        for (int i = threadIdx.x; i < 2 * P.hkv; i += kRowThreads)
            move(i < P.hkv ? L.k_scale : L.v_scale, P.pg.scale_stride, i % P.hkv, 1, 0);
}

// Beams.  CTA: a beam and a layer.  A beam's last page, where it is not full, goes to the first beam that descends from
// it; the others copy it into the pages of beams from which none descends, in order: as many as there are copies.
template <int kReq, int kLayers>
__global__ void __launch_bounds__(kRowThreads) paged_reorder_kernel(const __grid_constant__ RowsLaunch<kReq, kLayers> P) {
    __shared__ int s_parent[kBeamsMost];
    __shared__ unsigned long long s_copies, s_free;
    const int beam = blockIdx.x, W = P.width, r = beam / W, w = beam - r * W;
    const int full = P.rows[r] >> P.pg.page_shift, part = P.rows[r] & ((1 << P.pg.page_shift) - 1);
    after_kernels_before();
    const int64_t beam0 = (int64_t)(P.b0 + r) * W;           // the request's first beam
    if (threadIdx.x == 0) s_copies = s_free = 0ull;
    if ((int)threadIdx.x < W) {
        int p = ld_after(P.parent + beam0 + threadIdx.x);
        if (p < -1 || p >= W) {
            if (blockIdx.y == 0 && w == 0) atomicOr(P.err, 1);
            p = -1;
        }
        s_parent[threadIdx.x] = p < 0 ? threadIdx.x : p;     // (-1: the beam goes on as it is)
    }
    __syncthreads();
    if ((int)threadIdx.x < W) {
        const int mine = s_parent[threadIdx.x];
        bool first = true, childless = true;
        for (int i = 0; i < W; ++i) {
            const int p = s_parent[i];
            first = first && (i >= (int)threadIdx.x || p != mine);
            childless = childless && p != (int)threadIdx.x;
        }
        if (!first) atomicOr(&s_copies, 1ull << threadIdx.x);
        if (childless) atomicOr(&s_free, 1ull << threadIdx.x);
    }
    __syncthreads();
    const int from_beam = s_parent[w];
    const bool copies = s_copies >> w & 1ull;
    int to_beam = from_beam;                                 // whose page the beam takes
    if (copies) {
        unsigned long long f = s_free;
        for (int i = __popcll(s_copies & ((1ull << w) - 1)); i > 0; --i) f &= f - 1;
        to_beam = __ffsll((long long)f) - 1;
    }
    auto row_of = [&](int b) { return P.pg.table + (beam0 + b) * P.pg.table_stride; };
    if (blockIdx.y == 0 && P.first_layers) {
        const int32_t *const from = row_of(from_beam), *const own = row_of(w), *const to = row_of(to_beam);
        int32_t* const out = P.table_out + (beam0 + w) * P.table_out_stride;
        for (int j = threadIdx.x; j < P.table_width; j += kRowThreads)
            out[j] = ld_after(j < full ? from + j : j == full && part ? to + j : own + j);
    }
    if (!copies || !part) return;
    const int from = ld_after(row_of(from_beam) + full), to = ld_after(row_of(to_beam) + full);
    if (!page_there(P.pg, from) || !page_there(P.pg, to)) {
        if (threadIdx.x == 0) atomicOr(P.err, 1);
        return;
    }
    const LayerPages L = P.layer[blockIdx.y];
    // a head's rows of a page are one run
    const int chunks = P.row_bytes / 16, run = part * chunks, all = P.hkv * run;
    const int64_t stride16 = P.pg.page_stride;
    constexpr int kBatch = 4;
    for (int side = 0; side < 2; ++side) {
        const uint4* const a = static_cast<const uint4*>(side ? L.v : L.k) + from * stride16;
        uint4* const b = static_cast<uint4*>(side ? L.v : L.k) + to * stride16;
        for (int i0 = threadIdx.x; i0 < all; i0 += kBatch * kRowThreads) {
            uint4 x[kBatch];
            int at[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int i = i0 + k * kRowThreads, h = i / run;
                at[k] = i < all ? ((h << P.pg.page_shift) * chunks) + i - h * run : -1;
                if (at[k] >= 0) x[k] = ld_after(a + at[k]);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (at[k] >= 0) b[at[k]] = x[k];
        }
        if (L.k_scale) {
            const float* const sa = (side ? L.v_scale : L.k_scale) + from * P.pg.scale_stride;
            float* const sb = (side ? L.v_scale : L.k_scale) + to * P.pg.scale_stride;
            for (int i = threadIdx.x; i < P.hkv * part; i += kRowThreads) {
                const int h = i / part, at = (h << P.pg.page_shift) + i - h * part;
                sb[at] = ld_after(sa + at);
            }
        }
    }
}

template <int kReq, int kLayers, bool kBeams>
cudaError_t launch(const PagedRowsCall& c, cudaStream_t s) {
    for (int l0 = 0; l0 < c.n_layers; l0 += kLayers)
        for (int b0 = 0; b0 < c.batch; b0 += kReq) {
            const int nb = std::min(c.batch - b0, kReq), nl = std::min(c.n_layers - l0, kLayers);
            RowsLaunch<kReq, kLayers> P;
            P.pg = c.pg;
            // (pages are whole 16-byte lines)
            P.pg.page_stride = c.pg.page_stride / 16;
            for (int i = 0; i < nl; ++i) P.layer[i] = c.layers[l0 + i];
            P.err = c.err;
            P.path = c.path;
            P.n_accepted = c.n_accepted;
            P.parent = c.parent;
            P.table_out = c.table_out;
            P.table_out_stride = c.table_out_stride;
            P.b0 = b0;
            P.hkv = c.hkv;
            P.row_bytes = c.row_bytes;
            P.table_width = c.table_width;
            P.width = c.width;
            P.first_layers = l0 == 0;
            for (int i = 0; i < nb; ++i) P.rows[i] = kBeams ? c.n_rows[b0 + i] : c.start[b0 + i];
            if (!kBeams)
                for (int i = 0; i <= nb; ++i) P.ptr[i] = c.ptr[b0 + i];
            const dim3 grid((unsigned)(kBeams ? nb * c.width : nb), (unsigned)nl);
            const cudaError_t e = launch_overlapped(kBeams ? paged_reorder_kernel<kReq, kLayers> : paged_keep_kernel<kReq, kLayers>, grid,
                                                    kRowThreads, 0, s, P);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

template <bool kBeams>
cudaError_t by_size(const PagedRowsCall& c, cudaStream_t s) {
    if (c.batch > kPagedFew) return launch<kPagedMany, 48, kBeams>(c, s);
    return c.n_layers <= 4 ? launch<kPagedFew, 4, kBeams>(c, s) : launch<kPagedFew, 48, kBeams>(c, s);
}

}  // namespace

cudaError_t launch_paged_keep(const PagedRowsCall& c, cudaStream_t s) { return by_size<false>(c, s); }
cudaError_t launch_paged_reorder(const PagedRowsCall& c, cudaStream_t s) { return by_size<true>(c, s); }

}  // namespace c2kv
