// Attention of each request's new tokens over its paged cache (c2kv_paged_attend).
#include "paged.cuh"

#include <algorithm>
#include <vector>

namespace c2kv {
namespace {

// Query rows of a KV head up to which mma.sync takes a request.  tcgen05 works on 128 rows whatever they
// are and pays for its key tiles first; mma.sync reads and converts the keys again for every 32 rows.
// Measured (us, mma.sync / tcgen05; 32 / 8 heads, 64 and 80 rows; 1 request of 30000 rows, 8 of 4000, 16 of
// 500): 8-bit pages of 128 channels 60 / 92 and 74 / 92, 62 / 78 and 96 / 78, 23 / 34 and 39 / 33; 16-bit
// ones 91 / 100 and 126 / 100, 97 / 90 and 185 / 90, 44 / 37 and 62 / 38; 16-bit of 64 channels 44 / 65 and
// 56 / 66, 47 / 60 and 75 / 61, 19 / 27 and 30 / 27.  One limit for all of them: it is right for 8-bit pages and
// for heads of 64 channels, and late for 16-bit pages of 128 channels, where 64 rows of eight and of sixteen
// requests take 8 and 19 % longer than on tcgen05.
constexpr int kMmaRows = 64;

// The same of fp32 contexts, and the keys that some request has to see for it: the lanes' kernel reads keys
// again for every 4 rows, the register-tiled loop works on 16 rows or, below that, leaves most of its lanes
// to wait.  Measured (us, lanes / tiles; 16-bit pages as good as 8-bit ones).  32 / 8 heads of 128 channels, 4
// and 16 rows: 27 requests of 1381 keys 66 / 94 and 186 / 241, one of 30000 49 / 247 and 145 / 368, 16 of 9000
// 191 / 403 and 703 / 909; 24 rows of 8 requests of 700 keys 75 / 63.  8 / 8 heads of 64, 4 and 8 rows: 42 / 54
// and 67 / 77, 38 / 151 and 59 / 191, 135 / 182 and 295 / 277.  One request of 200 keys, any: 13 / 12, and four
// of 300: 14 / 15.  The limits go by a request's rows alone, so as to lose nowhere; heads of 64 channels with
// eight rows over one long context would gain most from another (59 where the tiles take 191).
constexpr int lane_rows(int d) { return d == 128 ? 16 : 4; }
constexpr int kLaneKeys = 256;

// Requests of many rows on tcgen05: what they see of their pages becomes key tiles first, in scratch that
// the stream hands back; requests go in groups so that the scratch stays small beside the cache.
constexpr int64_t kTileBytes = (int64_t)512 << 20;

cudaError_t launch_many(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s) {
    const int64_t tile_bytes = (int64_t)c.hkv * kTileKeys * d * 2;
    for (int b0 = 0; b0 < n;) {
        std::vector<PagedReq> part;
        std::vector<int32_t> tile0, tiles, key0;
        int64_t total = 0;
        for (; b0 < n; ++b0) {
            PagedReq q = req[b0];
            const int64_t first = c.window ? std::max<int64_t>(0, (int64_t)q.n_keys - q.nq + 1 - c.window) : 0;   // the first row that a query sees
            const int32_t lo = (int32_t)(first / kTileKeys), hi = (int32_t)(((int64_t)q.n_keys + kTileKeys - 1) / kTileKeys);
            if (!part.empty() && (total + hi - lo) * tile_bytes * 2 > kTileBytes) break;
            tile0.push_back(lo);
            tiles.push_back(std::max(0, hi - lo));
            key0.push_back((int32_t)first);
            q.scratch = (int32_t)(total - lo);
            total += tiles.back();
            part.push_back(q);
        }
        const int m = (int)part.size();
        const size_t most = (size_t)std::max<int64_t>(1, total), half = most * tile_bytes, odd = most * c.hkv * 16, units = most * c.hkv * 8;
        void* p = nullptr;
        cudaError_t e = context_alloc(c.ctx, &p, 2 * half + odd + units + most * 4);
        if (e == cudaErrorMemoryAllocation) {           // no room: key by key, slower
            (void)cudaGetLastError();
            e = launch_paged_mma(c, part.data(), m, d, codes, s);
            if (e != cudaSuccess) return e;
            continue;
        }
        if (e != cudaSuccess) return e;
        char* const base = static_cast<char*>(p);
        PagedExpandCall x{};
        x.pg = c.pg;
        x.to = KeyTiles{base, base + half, reinterpret_cast<uint4*>(base + 2 * half), reinterpret_cast<float2*>(base + 2 * half + odd),
                        reinterpret_cast<uint32_t*>(base + 2 * half + odd + units), (int32_t)total};
        x.err = c.err;
        x.hkv = c.hkv;
        x.n = m;
        x.req = part.data();
        x.tile0 = tile0.data();
        x.tiles = tiles.data();
        x.key0 = key0.data();
        e = launch_paged_expand(x, d, codes, s);
        if (e == cudaSuccess) e = launch_paged_tc(c, x.to, part.data(), m, d, codes, s);
        context_free(c.ctx, p);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_paged_attn(const PagedAttnCall& c, int dtype, int d, bool codes, cudaStream_t s) {
    std::vector<PagedReq> req;
    req.reserve(c.batch);
    for (int r = 0; r < c.batch; ++r)
        if (c.ptr[r + 1] > c.ptr[r]) req.push_back(PagedReq{c.ptr[r], c.ptr[r + 1] - c.ptr[r], c.n_keys[r], r, 0, 1, 0, 0, 0, 0});
    std::vector<PagedReq> few, many;
    auto part = [&](int64_t rows) {
        for (const PagedReq& q : req) ((int64_t)q.nq * (c.hq / c.hkv) > rows ? many : few).push_back(q);
    };
    cudaError_t e = cudaSuccess;
    if (dtype == kDtypeF32) {    // CUDA cores: a register-tiled loop, or lanes that share a key
        part(lane_rows(d));
        const bool seen = std::any_of(few.begin(), few.end(), [&](const PagedReq& q) {
            return q.n_keys > kLaneKeys && (!c.window || (int64_t)c.window + q.nq > kLaneKeys);
        });
        if (!seen) {
            many = req;
            few.clear();
        }
        if (!many.empty()) e = launch_paged_simt(c, many.data(), (int)many.size(), d, codes, s);
        if (e == cudaSuccess && !few.empty()) e = launch_paged_lane(c, few.data(), (int)few.size(), d, codes, s);
        return e;
    }
    part(kMmaRows);
    // requests of many rows on tcgen05, those of few on mma.sync
    if (!many.empty()) e = launch_many(c, many.data(), (int)many.size(), d, codes, s);
    if (e == cudaSuccess && !few.empty()) e = launch_paged_mma(c, few.data(), (int)few.size(), d, codes, s);
    return e;
}

}  // namespace c2kv
