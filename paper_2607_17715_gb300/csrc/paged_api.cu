// Host side of the paged calls and of draft verification: every argument is checked before anything
// is enqueued; the launches carry the per-request tables in their parameter blocks.
#include "c2kv.h"
#include "paged.cuh"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <exception>

namespace {

using c2kv::ContextView;

c2kv_status refuse(c2kv_ctx* c, c2kv_status code, const char* fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return c2kv::set_last_error(c, code, buf);
}

c2kv_status launched(c2kv_ctx* c, cudaError_t e, const char* what) {
    if (e == cudaSuccess) return C2KV_OK;
    (void)cudaGetLastError();   // a non-sticky failure must not leak into later calls
    return refuse(c, e == cudaErrorMemoryAllocation ? C2KV_ERR_NOMEM : C2KV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// What the three paged calls share: the pages and their table, and the requests' token ranges.
c2kv_status check_pages(c2kv_ctx* c, const ContextView& v, const char* what, const c2kv_pages* p, const int32_t* table,
                        int32_t table_width, int64_t table_stride, int32_t batch, const int32_t* ptr, c2kv::PageView* out) {
    if (!p || !table || !ptr) return refuse(c, C2KV_ERR_ARG, "%s: null pages, table or token ranges", what);
    if (!p->k || !p->v) return refuse(c, C2KV_ERR_ARG, "%s: null pages", what);
    if (p->format != C2KV_PAGES_NATIVE && p->format != C2KV_PAGES_E4M3)
        return refuse(c, C2KV_ERR_DTYPE, "%s: bad page format %d", what, p->format);
    const bool codes = p->format == C2KV_PAGES_E4M3;
    if (codes && (!p->k_scale || !p->v_scale)) return refuse(c, C2KV_ERR_ARG, "%s: E4M3 pages need scales", what);
    int shift = 4;
    while (shift < 7 && (1 << shift) != p->page_size) ++shift;
    if ((1 << shift) != p->page_size) return refuse(c, C2KV_ERR_ARG, "%s: page_size must be 16, 32, 64 or 128", what);
    if (p->n_pages < 1) return refuse(c, C2KV_ERR_ARG, "%s: n_pages < 1", what);
    const int eb = codes ? 1 : v.dtype == C2KV_DTYPE_BF16 ? 2 : 4;
    const int64_t rows = (int64_t)v.n_kv_heads * p->page_size;
    const int64_t stride = p->page_stride ? p->page_stride : rows * v.head_dim;
    const int64_t sstride = p->scale_stride ? p->scale_stride : rows;
    if (stride < rows * v.head_dim || stride * eb % 16 || (codes && (sstride < rows || sstride % 4)))
        return refuse(c, C2KV_ERR_ARG, "%s: page strides shorter than a page or not whole 16-byte lines", what);
    if (misaligned(p->k, 16) || misaligned(p->v, 16) || misaligned(table, 4) ||
        (codes && (misaligned(p->k_scale, 16) || misaligned(p->v_scale, 16))))
        return refuse(c, C2KV_ERR_ARG, "%s: pages and scales must be 16-byte aligned", what);
    if (table_width < 1 || table_stride < table_width) return refuse(c, C2KV_ERR_ARG, "%s: bad table shape", what);
    if (batch < 1) return refuse(c, C2KV_ERR_ARG, "%s: batch < 1", what);
    if (ptr[0] != 0) return refuse(c, C2KV_ERR_ARG, "%s: token ranges must start at 0", what);
    for (int32_t r = 0; r < batch; ++r)
        if (ptr[r + 1] < ptr[r]) return refuse(c, C2KV_ERR_ARG, "%s: token ranges decrease at request %d", what, r);
    *out = c2kv::PageView{p->k, p->v, codes ? p->k_scale : nullptr, codes ? p->v_scale : nullptr, table, stride, sstride,
                          table_stride, p->n_pages, shift};
    return C2KV_OK;
}

c2kv_status check_device(c2kv_ctx* c, const char* what, std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (c2kv::mem_kind(p) != c2kv::MemKind::kDevice)
            return refuse(c, C2KV_ERR_ARG, "%s: tensors must be device memory (a pointer is host memory or memory the "
                                           "GPU cannot address)", what);
    return C2KV_OK;
}

// Rows [0, rows) of every request must be named by its table.  The kernels count rows in 32 bits and
// round them up to whole tiles: 2^30 leave room.
constexpr int64_t kMostRows = (int64_t)1 << 30;

bool in_table(int64_t rows, int32_t table_width, const c2kv::PageView& pg) {
    return rows <= std::min((int64_t)table_width << pg.page_shift, kMostRows);
}

c2kv_status move(c2kv_ctx* c, const char* what, bool append, const c2kv_pages* pages, int32_t batch, const int32_t* table,
                 int32_t table_width, int64_t table_stride, const int32_t* ptr, const int32_t* start, void* k, void* v,
                 int64_t stride, const int32_t* turn) {
    ContextView x{};
    if (!c2kv::context_view(c, &x)) return C2KV_ERR_ARG;
    c2kv::PagedMoveCall m{};
    c2kv_status st = check_pages(c, x, what, pages, table, table_width, table_stride, batch, ptr, &m.pg);
    if (st != C2KV_OK) return st;
    if (!start) return refuse(c, C2KV_ERR_ARG, "%s: null start rows", what);
    for (int32_t r = 0; r < batch; ++r)
        if (start[r] < 0 || (ptr[r + 1] > ptr[r] && !in_table((int64_t)start[r] + ptr[r + 1] - ptr[r], table_width, m.pg)))
            return refuse(c, C2KV_ERR_ARG, "%s: rows of request %d are outside its table", what, r);
    if (ptr[batch] == 0) return c2kv::set_last_error(c, C2KV_OK, "");
    if (!k || !v) return refuse(c, C2KV_ERR_ARG, "%s: null k or v", what);
    const int64_t row = (int64_t)x.n_kv_heads * x.head_dim;
    m.stride = stride ? stride : row;
    const int eb = x.dtype == C2KV_DTYPE_BF16 ? 2 : 4;
    if (m.stride < row || m.stride * eb % 16)
        return refuse(c, C2KV_ERR_ARG, "%s: token stride shorter than a row or not whole 16-byte lines", what);
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(turn, 4))
        return refuse(c, C2KV_ERR_ARG, "%s: k, v must be 16-byte aligned", what);
    st = check_device(c, what, {pages->k, pages->v, m.pg.k_scale, m.pg.v_scale, table, k, v, turn});
    if (st != C2KV_OK) return st;
    m.k = k;
    m.v = v;
    m.turn = turn;
    m.err = x.err;
    m.hkv = x.n_kv_heads;
    m.batch = batch;
    m.ptr = ptr;
    m.start = start;
    m.rope = x.turns;
    const bool codes = pages->format == C2KV_PAGES_E4M3;
    c2kv::TraceScope trace(c, append ? C2KV_PROF_SUFFIX : C2KV_PROF_COMPOSE);
    const cudaError_t e = append ? c2kv::launch_paged_append(m, x.dtype, x.head_dim, codes, x.stream)
                                 : c2kv::launch_paged_gather(m, x.dtype, x.head_dim, codes, x.stream);
    if (e != cudaSuccess) return launched(c, e, what);
    return c2kv::set_last_error(c, C2KV_OK, "");
}

}  // namespace

extern "C" {

c2kv_status c2kv_paged_append(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t batch, const int32_t* table,
                              int32_t table_width, int64_t table_stride, const int32_t* new_ptr, const int32_t* start,
                              const void* k, const void* v, int64_t kv_stride, const int32_t* turn) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return move(ctx, "paged_append", true, pages, batch, table, table_width, table_stride, new_ptr, start,
                    const_cast<void*>(k), const_cast<void*>(v), kv_stride, turn);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "paged_append: host allocation failed");
    }
}

c2kv_status c2kv_paged_gather(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t batch, const int32_t* table,
                              int32_t table_width, int64_t table_stride, const int32_t* row_ptr, const int32_t* start,
                              void* k_out, void* v_out, int64_t out_stride, const int32_t* turn) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return move(ctx, "paged_gather", false, pages, batch, table, table_width, table_stride, row_ptr, start, k_out, v_out,
                    out_stride, turn);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "paged_gather: host allocation failed");
    }
}

c2kv_status c2kv_paged_attend(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t batch, const int32_t* table,
                              int32_t table_width, int64_t table_stride, const int32_t* q_ptr, const int32_t* n_keys,
                              int32_t window, const void* q, int64_t q_stride, const int32_t* turn, void* out, float* lse) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        const char* const what = "paged_attend";
        ContextView x{};
        if (!c2kv::context_view(ctx, &x)) return C2KV_ERR_ARG;
        c2kv::PagedAttnCall a{};
        c2kv_status st = check_pages(ctx, x, what, pages, table, table_width, table_stride, batch, q_ptr, &a.pg);
        if (st != C2KV_OK) return st;
        if (!n_keys) return refuse(ctx, C2KV_ERR_ARG, "%s: null n_keys", what);
        if (window < 0) return refuse(ctx, C2KV_ERR_ARG, "%s: window < 0", what);
        int32_t most = 0;
        for (int32_t r = 0; r < batch; ++r) {
            if (n_keys[r] < 0 || !in_table(n_keys[r], table_width, a.pg))
                return refuse(ctx, C2KV_ERR_ARG, "%s: rows of request %d are outside its table", what, r);
            most = std::max(most, n_keys[r]);
        }
        if (q_ptr[batch] == 0) return c2kv::set_last_error(ctx, C2KV_OK, "");
        if (!q || !out) return refuse(ctx, C2KV_ERR_ARG, "%s: null q or out", what);
        const int64_t row = (int64_t)x.n_q_heads * x.head_dim;
        a.q_stride = q_stride ? q_stride : row;
        const int eb = x.dtype == C2KV_DTYPE_BF16 ? 2 : 4;
        if (a.q_stride < row || a.q_stride * eb % 16)
            return refuse(ctx, C2KV_ERR_ARG, "%s: token stride shorter than a row or not whole 16-byte lines", what);
        if ((int64_t)q_ptr[batch] * x.n_q_heads > INT32_MAX)
            return refuse(ctx, C2KV_ERR_ARG, "%s: tokens * Hq above 2^31", what);
        if (misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4) || misaligned(turn, 4))
            return refuse(ctx, C2KV_ERR_ARG, "%s: q, out must be 16-byte aligned", what);
        st = check_device(ctx, what, {pages->k, pages->v, a.pg.k_scale, a.pg.v_scale, table, q, out, lse, turn});
        if (st != C2KV_OK) return st;
        a.ctx = ctx;
        a.q = q;
        a.out = out;
        a.lse = lse;
        a.turn = turn;
        a.err = x.err;
        a.hq = x.n_q_heads;
        a.hkv = x.n_kv_heads;
        a.window = window < most ? window : 0;   // (one that leaves nothing out is none)
        a.batch = batch;
        a.ptr = q_ptr;
        a.n_keys = n_keys;
        a.rope = x.turns;
        c2kv::TraceScope trace(ctx, C2KV_PROF_ATTN);
        const cudaError_t e = c2kv::launch_paged_attn(a, x.dtype, x.head_dim, pages->format == C2KV_PAGES_E4M3, x.stream);
        if (e != cudaSuccess) return launched(ctx, e, what);
        return c2kv::set_last_error(ctx, C2KV_OK, "");
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "paged_attend: host allocation failed");
    }
}

c2kv_status c2kv_verify_drafts(c2kv_ctx* ctx, int32_t batch, const int32_t* draft_ptr, int32_t vocab, const int32_t* tokens,
                               const float* p, int64_t p_stride, const float* q, int64_t q_stride, const float* u_accept,
                               const float* u_next, int32_t* n_accepted, int32_t* next_token) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        const char* const what = "verify_drafts";
        ContextView x{};
        if (!c2kv::context_view(ctx, &x)) return C2KV_ERR_ARG;
        if (batch < 1 || !draft_ptr) return refuse(ctx, C2KV_ERR_ARG, "%s: batch < 1 or null draft ranges", what);
        if (vocab < 1 || vocab > (1 << 19)) return refuse(ctx, C2KV_ERR_ARG, "%s: vocab outside [1, 2^19]", what);
        if (draft_ptr[0] != 0) return refuse(ctx, C2KV_ERR_ARG, "%s: draft ranges must start at 0", what);
        for (int32_t r = 0; r < batch; ++r)
            if (draft_ptr[r + 1] < draft_ptr[r])
                return refuse(ctx, C2KV_ERR_ARG, "%s: draft ranges decrease at request %d", what, r);
        const bool drafts = draft_ptr[batch] > 0;
        if (!p || !u_next || !n_accepted || !next_token || (drafts && (!tokens || !u_accept)))
            return refuse(ctx, C2KV_ERR_ARG, "%s: null pointer", what);
        c2kv::VerifyCall v{};
        v.p_stride = p_stride ? p_stride : vocab;
        v.q_stride = q_stride ? q_stride : vocab;
        if (v.p_stride < vocab || v.q_stride < vocab)
            return refuse(ctx, C2KV_ERR_ARG, "%s: row stride shorter than the vocabulary", what);
        for (const void* t : {(const void*)tokens, (const void*)p, (const void*)q, (const void*)u_accept, (const void*)u_next,
                              (const void*)n_accepted, (const void*)next_token})
            if (misaligned(t, 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
        const c2kv_status st = check_device(ctx, what, {tokens, p, q, u_accept, u_next, n_accepted, next_token});
        if (st != C2KV_OK) return st;
        v.tokens = tokens;
        v.p = p;
        v.q = q;
        v.u_accept = u_accept;
        v.u_next = u_next;
        v.n_accepted = n_accepted;
        v.next_token = next_token;
        v.err = x.err;
        v.vocab = vocab;
        v.batch = batch;
        v.ptr = draft_ptr;
        const cudaError_t e = c2kv::launch_verify(v, x.stream);
        if (e != cudaSuccess) return launched(ctx, e, what);
        return c2kv::set_last_error(ctx, C2KV_OK, "");
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "verify_drafts: host allocation failed");
    }
}

}  // extern "C"
