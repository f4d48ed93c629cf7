// Attention of each request's new tokens over its paged cache (c2kv_paged_attend).
#include "paged.cuh"
#include "per_device.cuh"

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

// The same of trees, and the rows up to which tcgen05 takes them straight from the pages instead of making key
// tiles first.  Measured (us, mma.sync / straight from the pages; one request of 30000 rows, 8 of 4000, 16 of 500): 8-bit
// pages of 128 channels, 16 rows 33 / 39, 29 / 39, 16 / 16, 32 rows 53 / 39, 44 / 40, 26 / 17; 16-bit ones, 16 rows 39 / 43, 40 / 43,
// 14 / 17, 32 rows 65 / 43, 66 / 44, 24 / 18; 8-bit ones of 64 channels, 32 rows 33 / 34, 30 / 34, 19 / 15.  24 rows of eight requests
// of 4000: 35 / 39 from 8-bit pages, 49 / 44 from 16-bit ones.  Straight from the pages / with key tiles: 256 rows 63 / 86, 60 / 91,
// 36 / 38, 384 rows 77 / 107, 113 / 106, 56 / 56, 512 rows 104 / 109, 116 / 112, 74 / 58, of 16-bit pages 116 / 121, 130 / 126, 78 / 62.
constexpr int tree_mma_rows(int d, bool codes) { return d * (codes ? 1 : 2) == 64 ? 32 : d * (codes ? 1 : 2) == 128 ? 24 : 16; }
constexpr int kDirectRows = 512;

// ... and trees over few keys, which many rows a CTA would leave SMs idle for: mma.sync takes them eight rows a CTA,
// or 16, where that is one wave of CTAs that read at most so many values of K, counted for eight rows.  Measured (us, eight /
// 16 / the routes above; 128 channels): 8-bit pages, one request of 1500 rows, 64 rows of queries (13 million values) 13.2 / 16.5 / 17.1,
// 128 rows (26) 17.3 / 18.5 / 17.5, of 6000, 32 rows (25) 16.6 / 21.1 / 22.0, 64 rows (50) 22.7 / 22.3 / 22.2; four of 500, 64
// rows (17) 13.2 / 16.6 / 17.9, 16 of 100, 32 rows (8; eight are more than a wave) - / 10.6 / 13.3; 16-bit pages, 64 rows over 1500
// 15.6 / 16.8 / 18.1, 96 rows (19) 19.5 / 18.4 / 18.3, 24 rows over 6000 (19) 17.3 / 19.9 / 22.4, 32 (25) 22.1 / 19.9 / 22.6.
constexpr int64_t short_values(bool codes) { return codes ? 26000000 : 18000000; }

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

// Trees whose (four rows, KV head, key)s are no more than this go to the lanes' kernel, whatever their rows: a CTA a stretch for
// every four rows fills the SMs where tiles leave most of them without one.  Measured (us, lanes / tiles): 16 / 4 heads of 64
// channels, one request of 700 keys, 104 rows (75 thousand) 18.7 / 20.7, 256 rows (196) 34 / 27, one of 3000, 64 rows (193) 31 / 37,
// three of 700, 64 rows (137) 25 / 27, eight of 1500, 16 rows (193) 31 / 35, 32 rows (386) 61 / 40; 32 / 8 heads of 128, one of 700,
// 64 rows (92) 25 / 37, 256 rows (391) 78 / 61, three of 700, 32 rows (136) 40 / 50, 64 rows (275) 76 / 56, one of 3000, 32 rows (193) 42 / 70.
constexpr int64_t kLaneTrees = 190000;

// The keys that any of a request's queries sees, at most.
int64_t keys_of(const PagedAttnCall& c, const PagedReq& q) { return c.window ? std::min<int64_t>(q.n_keys, (int64_t)c.window + q.nq) : q.n_keys; }

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

// Eights of query rows a CTA for trees that short rows of keys leave SMs free for, 0 for others.
int short_eights(const PagedAttnCall& c, const std::vector<PagedReq>& req, int d, bool codes) {
    const int64_t G = c.hq / c.hkv;
    int64_t units[2] = {0, 0}, values = 0;
    for (const PagedReq& q : req) {
        values += (q.nq * G + 7) / 8 * c.hkv * keys_of(c, q) * d;
        if (values > short_values(codes)) return 0;
        units[0] += (q.nq * G + 7) / 8 * c.hkv;
        units[1] += (q.nq * G + 15) / 16 * c.hkv;
    }
    for (int eights = 1; eights <= 2; ++eights)
        if (units[eights - 1] <= (int64_t)device_sms() * paged_mma_tree_ctas(d, codes, eights)) return eights;
    return 0;
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
        int64_t met = 0;
        for (const PagedReq& q : req)
            if (met <= kLaneTrees) met += ((int64_t)q.nq * (c.hq / c.hkv) + 3) / 4 * c.hkv * keys_of(c, q);
        if (c.parent && met <= kLaneTrees) return launch_paged_lane(c, req.data(), (int)req.size(), d, codes, s);
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
    if (c.parent) {
        if (const int eights = short_eights(c, req, d, codes)) {
            PagedAttnCall by_eights = c;
            by_eights.eights = eights;
            return launch_paged_mma(by_eights, req.data(), (int)req.size(), d, codes, s);
        }
        // those of middling size straight from the pages
        std::vector<PagedReq> middling, rest;
        for (const PagedReq& q : req) {
            const int64_t rows = (int64_t)q.nq * (c.hq / c.hkv);
            (rows > tree_mma_rows(d, codes) && rows <= kDirectRows ? middling : rest).push_back(q);
        }
        if (!middling.empty()) e = launch_paged_direct(c, middling.data(), (int)middling.size(), d, codes, s);
        if (e != cudaSuccess || rest.empty()) return e;
        req.swap(rest);
    }
    part(c.parent ? tree_mma_rows(d, codes) : kMmaRows);
    // requests of many rows on tcgen05, those of few on mma.sync
    if (!many.empty()) e = launch_many(c, many.data(), (int)many.size(), d, codes, s);
    if (e == cudaSuccess && !few.empty()) e = launch_paged_mma(c, few.data(), (int)few.size(), d, codes, s);
    return e;
}

}  // namespace c2kv
