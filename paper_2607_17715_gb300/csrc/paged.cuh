// Paged caches: parameters and launchers shared by the paged calls' translation units.
//
// A page holds page_size rows of every KV head, head-major ([Hkv][page_size][d]), so that one
// head's rows of a page are one contiguous run: what an attention CTA, which works on one KV
// head, reads.  Row j of request r lives in page table[r][j / page_size].
#pragma once

#include "internal.cuh"

namespace c2kv {

// Requests a launch carries in its parameter block: a launch's latency grows by about 0.4 us for
// each KB of parameters, so calls of few requests take the small block.
constexpr int kPagedFew = 32;
constexpr int kPagedMany = 256;

struct PageView {
    void* k;                 // [n_pages][Hkv][page_size][d]: the context's type, or E4M3 codes
    void* v;
    float* k_scale;          // [n_pages][Hkv][page_size] (E4M3)
    float* v_scale;
    const int32_t* table;    // [batch][table_stride]: page of rows j * page_size ..
    int64_t page_stride;     // elements between pages
    int64_t scale_stride;    // scales between pages
    int64_t table_stride;
    int32_t n_pages;
    int32_t page_shift;      // log2(page_size)
};

// Rows of new (or old) tokens moved between a dense block [T][Hkv][d] and pages.
template <int kReq>
struct PagedMove {
    PageView pg;
    void* k;                 // dense [T] rows, stride elements apart
    void* v;
    int64_t stride;
    const int32_t* turn;     // [T] positions that K turns by, or null
    int32_t* err;            // device error word: bit 0 = index refused
    int32_t batch;
    int32_t b0;              // table row of the launch's first request
    int32_t hkv;
    float per_hkv;           // 1 / hkv
    int32_t tokens_per_cta;
    int32_t t0;              // first token of this launch
    int32_t t1;              // one past its last
    RopeTurns rope;
    int32_t ptr[kReq + 1];   // tokens [ptr[r], ptr[r + 1]) are request r's ...
    int32_t start[kReq];     // ... rows start[r] ..
};

// Moves tokens [ptr[0], ptr[batch]) of the call's `batch` requests, kPagedMany requests a launch.
struct PagedMoveCall {
    PageView pg;
    void* k;
    void* v;
    int64_t stride;
    const int32_t* turn;
    int32_t* err;
    int32_t hkv;
    int32_t batch;
    const int32_t* ptr;      // host [batch + 1]
    const int32_t* start;    // host [batch]
    const RopeTurns* rope;
};
cudaError_t launch_paged_append(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s);
cudaError_t launch_paged_gather(const PagedMoveCall& c, int dtype, int d, bool codes, cudaStream_t s);

// One request of an attention launch: queries [q0, q0 + nq) are the last nq of its n_keys rows.
struct PagedReq {
    int32_t q0;
    int32_t nq;              // at least 1
    int32_t n_keys;
    int32_t row;             // its row of the table
    int32_t item0;           // first work item of the request
    int32_t splits;          // stretches that its keys are cut into
    int32_t unit0;           // first unit (row tile of a KV head)
    int32_t scratch;         // (paged_tc.cu) its key tile 0 among the launch's key tiles
    int32_t tile0;           // its row tiles of this entry: [tile0, tile0 + tiles)
    int32_t tiles;
};

template <int kReq>
struct PagedAttn {
    PageView pg;
    const void* q;           // [T] rows of [Hq][d], q_stride elements apart, before RoPE
    void* out;               // [T][Hq][d]
    float* lse;              // [Hq][T] natural log, or null
    const int32_t* turn;     // [T] positions that the queries turn by, or null
    int32_t* err;
    int64_t q_stride;
    int64_t n_tokens;        // T
    int32_t batch;
    int32_t hq;
    int32_t hkv;
    int32_t group;           // hq / hkv
    int32_t window;          // a query sees at most the last `window` rows up to its own (0: all)
    float scale_log2;        // log2(e) / sqrt(d)
    RopeTurns rope;
    PagedReq req[kReq];
};

struct PagedAttnCall {
    c2kv_ctx* ctx;           // whose workspace holds the partials of split keys
    PageView pg;
    const void* q;
    void* out;
    float* lse;
    const int32_t* turn;
    int32_t* err;
    int64_t q_stride;
    int32_t hq;
    int32_t hkv;
    int32_t window;
    int32_t batch;
    const int32_t* ptr;      // host [batch + 1]
    const int32_t* n_keys;   // host [batch]
    const RopeTurns* rope;
};
cudaError_t launch_paged_attn(const PagedAttnCall& c, int dtype, int d, bool codes, cudaStream_t s);
// fp32 queries of n requests on the CUDA cores (paged_simt.cu).
cudaError_t launch_paged_simt(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// The same of few rows a request (paged_lane.cu).
cudaError_t launch_paged_lane(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// bf16 queries of n requests on mma.sync (paged_mma.cu).
cudaError_t launch_paged_mma(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);

// Tensor map of pages [n_pages][Hkv][page_size][d], elements of 16 bits or codes of 8.
bool encode_page_map(CUtensorMap* tm, const void* base, const PageView& pg, int hkv, int d, bool codes, int box_channels,
                     int box_rows, CUtensorMapSwizzle swizzle);
// Key tiles: what requests see of their pages, 128 keys of a KV head at a time, as f16 relative to a power
// of two of the tile's own (paged_expand.cu).  Key tile t of a request is tile `scratch` + t.
constexpr int kTileKeys = 128;
struct KeyTiles {
    void* k;                 // [n][Hkv][128][d] f16; rows that no query sees, or of no page, are zero
    void* v;                 // (and values of V that are not finite)
    uint4* odd;              // [n][Hkv]: rows of V with values that are not finite (128 bits)
    float2* unit;            // [n][Hkv]: the factor that K's values lack, and the exponent of V's
    uint32_t* there;         // [n]: which groups of 16 keys lie in pages (bits 0 .. 7)
    int32_t n;               // may be 0: no query sees a row
};
struct PagedExpandCall {
    PageView pg;
    KeyTiles to;
    int32_t* err;
    int32_t hkv;
    int32_t n;
    const PagedReq* req;
    const int32_t* tile0;    // first key tile of each request that any query sees ...
    const int32_t* tiles;    // ... how many from there on; they follow one another in `to`
    const int32_t* key0;     // ... and the first key
};
cudaError_t launch_paged_expand(const PagedExpandCall& c, int d, bool codes, cudaStream_t s);
// bf16 queries of n requests over their key tiles on tcgen05 (paged_tc.cu).
cudaError_t launch_paged_tc(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);

template <int kReq>
void fill_paged(PagedAttn<kReq>& P, const PagedAttnCall& c, int d, const PagedReq* req, int n) {
    P.pg = c.pg;
    P.q = c.q;
    P.out = c.out;
    P.lse = c.lse;
    P.turn = c.turn;
    P.err = c.err;
    P.q_stride = c.q_stride;
    P.n_tokens = c.ptr[c.batch];
    P.batch = n;
    P.hq = c.hq;
    P.hkv = c.hkv;
    P.group = c.hq / c.hkv;
    P.window = c.window;
    P.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)d));
    P.rope = *c.rope;
    for (int i = 0; i < n; ++i) P.req[i] = req[i];
}

// Whether any row lo .. hi - 1 of the request at row `r` of the table lies in a page.
__device__ __forceinline__ bool any_page(const PageView& pg, int r, int lo, int hi) {
    if (hi <= lo) return false;
    for (int j = lo >> pg.page_shift; j <= (hi - 1) >> pg.page_shift; ++j) {
        const int page = pg.table[(int64_t)r * pg.table_stride + j];
        if (page >= 0 && page < pg.n_pages) return true;
    }
    return false;
}
// The output of a row whose weights' sum is zero, its last key being `end`: zero where it sees no key, and no
// number where every score that it sees is -inf.
template <int kReq>
__device__ __forceinline__ float of_no_weight(const PagedAttn<kReq>& P, int r, int end) {
    return any_page(P.pg, r, P.window ? max(0, end - P.window + 1) : 0, end + 1) ? __uint_as_float(0x7fc00000u) : 0.f;
}

// Drafted tokens against the target's probabilities (verify.cu).
template <int kReq>
struct VerifyParams {
    const int32_t* tokens;   // [T] drafted tokens
    const float* p;          // target's probabilities, p_stride apart: request r's rows ptr[r] + r ..
    const float* q;          // draft's, q_stride apart, or null (a draft that is sure of its tokens)
    const float* u_accept;   // [T]
    const float* u_next;     // [B]
    int32_t* n_accepted;     // [B]
    int32_t* next_token;     // [B]
    int32_t* err;
    int64_t p_stride;
    int64_t q_stride;
    int32_t vocab;
    int32_t b0;
    int32_t ptr[kReq + 1];
};
struct VerifyCall {
    const int32_t* tokens;
    const float* p;
    const float* q;
    const float* u_accept;
    const float* u_next;
    int32_t* n_accepted;
    int32_t* next_token;
    int32_t* err;
    int64_t p_stride;
    int64_t q_stride;
    int32_t vocab;
    int32_t batch;
    const int32_t* ptr;      // host [batch + 1]
};
cudaError_t launch_verify(const VerifyCall& c, cudaStream_t s);

}  // namespace c2kv
