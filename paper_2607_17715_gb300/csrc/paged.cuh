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
    const int32_t* parent;   // [T] (trees) the queries' parents among their request's, -1 for a root
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
    const int32_t* parent;   // null: each request's queries follow one another
    int32_t* err;
    int64_t q_stride;
    int32_t hq;
    int32_t hkv;
    int32_t window;
    int32_t batch;
    const int32_t* ptr;      // host [batch + 1]
    const int32_t* n_keys;   // host [batch]
    const RopeTurns* rope;
    int32_t eights;          // most eights of query rows a CTA of paged_mma.cu, 0: as many as it holds
};
cudaError_t launch_paged_attn(const PagedAttnCall& c, int dtype, int d, bool codes, cudaStream_t s);
// fp32 queries of n requests on the CUDA cores (paged_simt.cu).
cudaError_t launch_paged_simt(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// The same of few rows a request (paged_lane.cu).
cudaError_t launch_paged_lane(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// bf16 queries of n requests on mma.sync (paged_mma.cu).
cudaError_t launch_paged_mma(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// The same of trees (paged_*_tree.cu): what the three launchers call where there are parents.
cudaError_t launch_paged_simt_tree(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
cudaError_t launch_paged_lane_tree(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
cudaError_t launch_paged_mma_tree(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);
// CTAs of that many eights of query rows which an SM holds.
int paged_mma_tree_ctas(int d, bool codes, int eights);

// bf16 trees of n requests on tcgen05, straight from the pages (paged_direct.cu).
cudaError_t launch_paged_direct(const PagedAttnCall& c, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);

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
cudaError_t launch_paged_tc_tree(const PagedAttnCall& c, const KeyTiles& tiles, const PagedReq* req, int n, int d, bool codes, cudaStream_t s);

template <int kReq>
void fill_paged(PagedAttn<kReq>& P, const PagedAttnCall& c, int d, const PagedReq* req, int n) {
    P.pg = c.pg;
    P.q = c.q;
    P.out = c.out;
    P.lse = c.lse;
    P.turn = c.turn;
    P.parent = c.parent;
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
// Trees (c2kv_paged_attend_tree): the queries of a request are the nodes of trees, parents before children, and
// node i's key is row `before` + i.  A node sees the rows before the tree, the nodes on its way to its root and
// itself; with a window, the last `window` rows of that path.
constexpr int kTreeMost = 512;           // nodes of a request: a bit a node in shared memory for every query row
constexpr int kTreeWords = kTreeMost / 32;

// f(node) for node i and those above it that it sees, by the parents of its request; returns i's depth.  A parent
// that is none of the nodes before its child is refused, and the child a root: the way always ends.
template <class F>
__device__ __forceinline__ int tree_way(const int32_t* parent, int i, int window, int32_t* err, const F& f) {
    int depth = 0;
    for (;; ++depth) {
        if (!window || depth < window) f(i);
        const int p = parent[i];
        if (p < -1 || p >= i) atomicOr(err, 1);
        if (p < 0 || p >= i) return depth;
        i = p;
    }
}
// What a node sees as a bit a node (bits[kTreeWords], zero before), and the last row before the tree that it does
// not see (-1: it sees all of them).
__device__ __forceinline__ int tree_bits(const int32_t* parent, int i, int before, int window, int32_t* err, uint32_t* bits) {
    const int depth = tree_way(parent, i, window, err, [&](int j) { bits[j >> 5] |= 1u << (j & 31); });
    return window ? max(-1, min(before + depth - window, before - 1)) : -1;
}
__device__ __forceinline__ bool tree_sees(int key, int before, int start, const uint32_t* bits) {
    if (key < before) return key > start;
    const int j = key - before;
    return j < kTreeMost && (bits[j >> 5] >> (j & 31) & 1u);
}

// The output of a row whose weights' sum is zero, of query `tok` of the request: zero where it sees no key, and no
// number where every score that it sees is -inf.
template <bool kTree, int kReq>
__device__ __forceinline__ float of_no_weight(const PagedAttn<kReq>& P, const PagedReq& R, int tok) {
    const int before = R.n_keys - R.nq, end = before + tok;
    bool any = false;
    if constexpr (kTree) {
        const int depth = tree_way(P.parent + R.q0, tok, P.window, P.err, [&](int j) { any = any || any_page(P.pg, R.row, before + j, before + j + 1); });
        any = any || any_page(P.pg, R.row, P.window ? max(0, before + depth - P.window + 1) : 0, before);
    } else {
        any = any_page(P.pg, R.row, P.window ? max(0, end - P.window + 1) : 0, end + 1);
    }
    return any ? __uint_as_float(0x7fc00000u) : 0.f;
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

// The walk down a tree of drafted tokens (verify_tree.cu).
template <int kReq>
struct VerifyTreeParams {
    const int32_t* tokens;   // [T] drafted tokens (the root's is not read)
    const int32_t* parent;   // [T] among the request's nodes, -1 for a root
    const float* p;          // [T] target's probabilities after each node, p_stride apart
    const float* u;          // [T]
    int32_t* n_accepted;     // [B]
    int32_t* path;           // [T]
    int32_t* next_token;     // [B]
    int32_t* err;
    int64_t p_stride;
    int32_t vocab;
    int32_t b0;
    int32_t ptr[kReq + 1];
};
struct VerifyTreeCall {
    const int32_t* tokens;
    const int32_t* parent;
    const float* p;
    const float* u;
    int32_t* n_accepted;
    int32_t* path;
    int32_t* next_token;
    int32_t* err;
    int64_t p_stride;
    int32_t vocab;
    int32_t batch;
    const int32_t* ptr;      // host [batch + 1]
};
cudaError_t launch_verify_tree(const VerifyTreeCall& c, cudaStream_t s);

// Rows moved within the pages of several layers, which share a table and their pages' geometry (paged_rows.cu).
struct LayerPages {
    void* k;
    void* v;
    float* k_scale;
    float* v_scale;
};
struct PagedRowsCall {
    PageView pg;             // geometry and table; its pages are layer 0's
    const LayerPages* layers;     // host [n_layers]
    int32_t n_layers;
    int32_t hkv;
    int32_t row_bytes;       // of one KV head's row of K or V
    int32_t* err;
    int32_t batch;
    // rows of the tokens that a walk kept
    const int32_t* ptr;      // host [batch + 1]
    const int32_t* start;    // host [batch]
    const int32_t* path;     // [T]
    const int32_t* n_accepted;    // [batch]
    // beams
    const int32_t* n_rows;   // host [batch]
    const int32_t* parent;   // [batch][width]
    int32_t* table_out;      // [batch * width], table_out_stride apart
    int64_t table_out_stride;
    int32_t table_width;
    int32_t width;
};
cudaError_t launch_paged_keep(const PagedRowsCall& c, cudaStream_t s);
cudaError_t launch_paged_reorder(const PagedRowsCall& c, cudaStream_t s);
constexpr int kBeamsMost = 64;           // beams of a request, and candidates that a choice leaves

// The best continuations of beams over the vocabulary (beam_select.cu).
struct BeamParams {
    const void* x;           // [batch * width][vocab], x_stride elements apart
    const float* norm;       // [batch * width] or null
    const float* score;      // [batch * width]
    const int32_t* done;     // [batch * width] or null
    int32_t* parent;         // [batch][best]
    int32_t* token;
    float* score_out;
    int32_t* done_out;       // or null
    int64_t x_stride;
    uint2* part;             // [batch][parts][best]: keys and places of each part's best
    uint32_t* tickets;       // [batch], zero between launches
    int32_t batch, width, vocab, best, end_token;
    int32_t b0;              // the launch's first request
    int32_t parts;           // CTAs (stretches) of a request
};
struct BeamCall {
    c2kv_ctx* ctx;
    BeamParams p;            // (all but the partials)
    bool bf16;
};
cudaError_t launch_beam_select(const BeamCall& c, cudaStream_t s);

}  // namespace c2kv
