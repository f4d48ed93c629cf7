// Host side of generation that branches: the walk down a tree, the rows that it kept, beams and their pages.  As in the
// other paged calls, every argument is checked before anything is enqueued.
#include "paged_check.cuh"

#include <vector>

namespace {

// The pages of the layers: each fits, and all have one geometry.
c2kv_status check_layers(c2kv_ctx* c, const ContextView& v, const char* what, const c2kv_pages* pages, int32_t n_layers, int32_t batch,
                         int32_t beams, const int32_t* table, int32_t table_width, int64_t table_stride, std::vector<c2kv::LayerPages>* layers,
                         c2kv::PagedRowsCall* m) {
    if (n_layers < 1 || !pages) return refuse(c, C2KV_ERR_ARG, "%s: n_layers < 1 or null pages", what);
    const int32_t none[2] = {0, 0};
    c2kv::DeviceMemory device;
    for (int32_t i = 0; i < n_layers; ++i) {
        c2kv::PageView pg{};
        c2kv_status st = check_pages(c, v, what, pages + i, table, table_width, table_stride, 1, none, &pg);
        if (st != C2KV_OK) return st;
        if (i == 0) m->pg = pg;
        else if (pg.page_stride != m->pg.page_stride || pg.n_pages != m->pg.n_pages || pg.page_shift != m->pg.page_shift ||
                 pages[i].format != pages[0].format || (pg.k_scale && pg.scale_stride != m->pg.scale_stride))
            return refuse(c, C2KV_ERR_ARG, "%s: the pages of layer %d differ from the first's in number, size, format or stride", what, i);
        for (const void* p : {(const void*)pg.k, (const void*)pg.v, (const void*)pg.k_scale, (const void*)pg.v_scale})
            if (!device.holds(p)) return refuse(c, C2KV_ERR_ARG, "%s: pages must be device memory (those of layer %d are not)", what, i);
        layers->push_back(c2kv::LayerPages{pg.k, pg.v, pg.k_scale, pg.v_scale});
    }
    if ((int64_t)batch * beams > INT32_MAX) return refuse(c, C2KV_ERR_ARG, "%s: too many table rows", what);
    const int eb = pages[0].format == C2KV_PAGES_E4M3 ? 1 : v.dtype == C2KV_DTYPE_BF16 ? 2 : 4;
    m->pg.page_stride *= eb;                     // bytes
    m->layers = layers->data();
    m->n_layers = n_layers;
    m->hkv = v.n_kv_heads;
    m->row_bytes = v.head_dim * eb;
    m->err = v.err;
    m->batch = batch;
    m->table_width = table_width;
    return C2KV_OK;
}

c2kv_status check_trees(c2kv_ctx* c, const char* what, int32_t batch, const int32_t* ptr) {
    if (batch < 1 || !ptr) return refuse(c, C2KV_ERR_ARG, "%s: batch < 1 or null token ranges", what);
    if (ptr[0] != 0) return refuse(c, C2KV_ERR_ARG, "%s: token ranges must start at 0", what);
    for (int32_t r = 0; r < batch; ++r) {
        if (ptr[r + 1] < ptr[r]) return refuse(c, C2KV_ERR_ARG, "%s: token ranges decrease at request %d", what, r);
        if (ptr[r + 1] - ptr[r] > c2kv::kTreeMost)
            return refuse(c, C2KV_ERR_UNSUPPORTED, "%s: more than %d nodes of request %d", what, c2kv::kTreeMost, r);
    }
    return C2KV_OK;
}

c2kv_status verify_tree(c2kv_ctx* ctx, int32_t batch, const int32_t* tree_ptr, int32_t vocab, const int32_t* tokens, const int32_t* parent,
                        const float* p, int64_t p_stride, const float* u, int32_t* n_accepted, int32_t* path, int32_t* next_token) {
    const char* const what = "verify_tree";
    ContextView x{};
    if (!c2kv::context_view(ctx, &x)) return C2KV_ERR_ARG;
    c2kv_status st = check_trees(ctx, what, batch, tree_ptr);
    if (st != C2KV_OK) return st;
    if (vocab < 1 || vocab > (1 << 19)) return refuse(ctx, C2KV_ERR_ARG, "%s: vocab outside [1, 2^19]", what);
    if (!n_accepted || !next_token || (tree_ptr[batch] > 0 && (!tokens || !parent || !p || !u || !path)))
        return refuse(ctx, C2KV_ERR_ARG, "%s: null pointer", what);
    c2kv::VerifyTreeCall v{};
    v.p_stride = p_stride ? p_stride : vocab;
    if (v.p_stride < vocab) return refuse(ctx, C2KV_ERR_ARG, "%s: row stride shorter than the vocabulary", what);
    for (const void* t : {(const void*)tokens, (const void*)parent, (const void*)p, (const void*)u, (const void*)n_accepted, (const void*)path,
                          (const void*)next_token})
        if (misaligned(t, 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
    st = check_device(ctx, what, {tokens, parent, p, u, n_accepted, path, next_token});
    if (st != C2KV_OK) return st;
    v.tokens = tokens;
    v.parent = parent;
    v.p = p;
    v.u = u;
    v.n_accepted = n_accepted;
    v.path = path;
    v.next_token = next_token;
    v.err = x.err;
    v.vocab = vocab;
    v.batch = batch;
    v.ptr = tree_ptr;
    const cudaError_t e = c2kv::launch_verify_tree(v, x.stream);
    if (e != cudaSuccess) return launched(ctx, e, what);
    return c2kv::set_last_error(ctx, C2KV_OK, "");
}

c2kv_status keep(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t n_layers, int32_t batch, const int32_t* table, int32_t table_width,
                 int64_t table_stride, const int32_t* tree_ptr, const int32_t* start, const int32_t* path, const int32_t* n_accepted) {
    const char* const what = "paged_keep";
    ContextView x{};
    if (!c2kv::context_view(ctx, &x)) return C2KV_ERR_ARG;
    c2kv_status st = check_trees(ctx, what, batch, tree_ptr);
    if (st != C2KV_OK) return st;
    c2kv::PagedRowsCall m{};
    std::vector<c2kv::LayerPages> layers;
    st = check_layers(ctx, x, what, pages, n_layers, batch, 1, table, table_width, table_stride, &layers, &m);
    if (st != C2KV_OK) return st;
    if (!start) return refuse(ctx, C2KV_ERR_ARG, "%s: null start rows", what);
    for (int32_t r = 0; r < batch; ++r)
        if (start[r] < 0 || (tree_ptr[r + 1] > tree_ptr[r] && !in_table((int64_t)start[r] + tree_ptr[r + 1] - tree_ptr[r], table_width, m.pg)))
            return refuse(ctx, C2KV_ERR_ARG, "%s: rows of request %d are outside its table", what, r);
    if (tree_ptr[batch] == 0) return c2kv::set_last_error(ctx, C2KV_OK, "");
    if (!path || !n_accepted) return refuse(ctx, C2KV_ERR_ARG, "%s: null path or n_accepted", what);
    if (misaligned(path, 4) || misaligned(n_accepted, 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
    st = check_device(ctx, what, {table, path, n_accepted});
    if (st != C2KV_OK) return st;
    m.ptr = tree_ptr;
    m.start = start;
    m.path = path;
    m.n_accepted = n_accepted;
    c2kv::TraceScope trace(ctx, C2KV_PROF_SUFFIX);
    const cudaError_t e = c2kv::launch_paged_keep(m, x.stream);
    if (e != cudaSuccess) return launched(ctx, e, what);
    return c2kv::set_last_error(ctx, C2KV_OK, "");
}

c2kv_status reorder(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t n_layers, int32_t batch, int32_t width, const int32_t* table,
                    int32_t table_width, int64_t table_stride, const int32_t* n_rows, const int32_t* parent, int32_t* table_out,
                    int64_t table_out_stride) {
    const char* const what = "paged_reorder";
    ContextView x{};
    if (!c2kv::context_view(ctx, &x)) return C2KV_ERR_ARG;
    if (batch < 1) return refuse(ctx, C2KV_ERR_ARG, "%s: batch < 1", what);
    if (width < 1 || width > c2kv::kBeamsMost) return refuse(ctx, C2KV_ERR_ARG, "%s: width outside [1, %d]", what, c2kv::kBeamsMost);
    c2kv::PagedRowsCall m{};
    std::vector<c2kv::LayerPages> layers;
    c2kv_status st = check_layers(ctx, x, what, pages, n_layers, batch, width, table, table_width, table_stride, &layers, &m);
    if (st != C2KV_OK) return st;
    if (!n_rows || !parent || !table_out) return refuse(ctx, C2KV_ERR_ARG, "%s: null rows, parents or new table", what);
    if (table_out_stride < table_width) return refuse(ctx, C2KV_ERR_ARG, "%s: bad shape of the new table", what);
    for (int32_t r = 0; r < batch; ++r)
        if (n_rows[r] < 0 || !in_table(n_rows[r], table_width, m.pg))
            return refuse(ctx, C2KV_ERR_ARG, "%s: rows of request %d are outside its table", what, r);
    if (misaligned(parent, 4) || misaligned(table_out, 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
    // beams read one another's rows of the old table while the new one is written
    const int64_t rows = (int64_t)batch * width - 1;
    const uintptr_t a = reinterpret_cast<uintptr_t>(table), b = reinterpret_cast<uintptr_t>(table_out);
    if (a < b + 4 * (uintptr_t)(rows * table_out_stride + table_width) && b < a + 4 * (uintptr_t)(rows * table_stride + table_width))
        return refuse(ctx, C2KV_ERR_ARG, "%s: the new table must not lie over the old one", what);
    st = check_device(ctx, what, {table, parent, table_out});
    if (st != C2KV_OK) return st;
    m.n_rows = n_rows;
    m.parent = parent;
    m.table_out = table_out;
    m.table_out_stride = table_out_stride;
    m.width = width;
    c2kv::TraceScope trace(ctx, C2KV_PROF_COMPOSE);
    const cudaError_t e = c2kv::launch_paged_reorder(m, x.stream);
    if (e != cudaSuccess) return launched(ctx, e, what);
    return c2kv::set_last_error(ctx, C2KV_OK, "");
}

c2kv_status select(c2kv_ctx* ctx, int32_t batch, int32_t width, int32_t vocab, int32_t best, int32_t dtype, const void* x, int64_t x_stride,
                   const float* norm, const float* score, const int32_t* done, int32_t end_token, int32_t* parent, int32_t* token,
                   float* score_out, int32_t* done_out) {
    const char* const what = "beam_select";
    ContextView v{};
    if (!c2kv::context_view(ctx, &v)) return C2KV_ERR_ARG;
    if (batch < 1) return refuse(ctx, C2KV_ERR_ARG, "%s: batch < 1", what);
    if (width < 1 || width > c2kv::kBeamsMost || best < 1 || best > c2kv::kBeamsMost)
        return refuse(ctx, C2KV_ERR_ARG, "%s: width or n_best outside [1, %d]", what, c2kv::kBeamsMost);
    if (vocab < 1 || vocab > (1 << 19)) return refuse(ctx, C2KV_ERR_ARG, "%s: vocab outside [1, 2^19]", what);
    if (dtype != C2KV_DTYPE_BF16 && dtype != C2KV_DTYPE_F32) return refuse(ctx, C2KV_ERR_DTYPE, "%s: bad type %d", what, dtype);
    if (end_token < -1 || end_token >= vocab || (done && end_token < 0))
        return refuse(ctx, C2KV_ERR_ARG, "%s: end_token outside the vocabulary, or none beside done", what);
    if ((int64_t)batch * width > (1 << 22)) return refuse(ctx, C2KV_ERR_ARG, "%s: more than 2^22 beams", what);
    if (!x || !score || !parent || !token || !score_out) return refuse(ctx, C2KV_ERR_ARG, "%s: null pointer", what);
    c2kv::BeamCall c{};
    c.p.x_stride = x_stride ? x_stride : vocab;
    if (c.p.x_stride < vocab) return refuse(ctx, C2KV_ERR_ARG, "%s: row stride shorter than the vocabulary", what);
    if (misaligned(x, dtype == C2KV_DTYPE_BF16 ? 2 : 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
    for (const void* t : {(const void*)norm, (const void*)score, (const void*)done, (const void*)parent, (const void*)token,
                          (const void*)score_out, (const void*)done_out})
        if (misaligned(t, 4)) return refuse(ctx, C2KV_ERR_ARG, "%s: misaligned pointer", what);
    const c2kv_status st = check_device(ctx, what, {x, norm, score, done, parent, token, score_out, done_out});
    if (st != C2KV_OK) return st;
    c.ctx = ctx;
    c.bf16 = dtype == C2KV_DTYPE_BF16;
    c.p.x = x;
    c.p.norm = norm;
    c.p.score = score;
    c.p.done = done;
    c.p.parent = parent;
    c.p.token = token;
    c.p.score_out = score_out;
    c.p.done_out = done_out;
    c.p.batch = batch;
    c.p.width = width;
    c.p.vocab = vocab;
    c.p.best = best;
    c.p.end_token = end_token;
    const cudaError_t e = c2kv::launch_beam_select(c, v.stream);
    if (e != cudaSuccess) return launched(ctx, e, what);
    return c2kv::set_last_error(ctx, C2KV_OK, "");
}

}  // namespace

extern "C" {

c2kv_status c2kv_verify_tree(c2kv_ctx* ctx, int32_t batch, const int32_t* tree_ptr, int32_t vocab, const int32_t* tokens,
                             const int32_t* parent, const float* p, int64_t p_stride, const float* u, int32_t* n_accepted, int32_t* path,
                             int32_t* next_token) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return verify_tree(ctx, batch, tree_ptr, vocab, tokens, parent, p, p_stride, u, n_accepted, path, next_token);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "verify_tree: host allocation failed");
    }
}

c2kv_status c2kv_paged_keep(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t n_layers, int32_t batch, const int32_t* table,
                            int32_t table_width, int64_t table_stride, const int32_t* tree_ptr, const int32_t* start, const int32_t* path,
                            const int32_t* n_accepted) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return keep(ctx, pages, n_layers, batch, table, table_width, table_stride, tree_ptr, start, path, n_accepted);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "paged_keep: host allocation failed");
    }
}

c2kv_status c2kv_beam_select(c2kv_ctx* ctx, int32_t batch, int32_t width, int32_t vocab, int32_t n_best, int32_t dtype, const void* x,
                             int64_t x_stride, const float* norm, const float* score, const int32_t* done, int32_t end_token,
                             int32_t* parent, int32_t* token, float* score_out, int32_t* done_out) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return select(ctx, batch, width, vocab, n_best, dtype, x, x_stride, norm, score, done, end_token, parent, token, score_out, done_out);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "beam_select: host allocation failed");
    }
}

c2kv_status c2kv_paged_reorder(c2kv_ctx* ctx, const c2kv_pages* pages, int32_t n_layers, int32_t batch, int32_t width, const int32_t* table,
                               int32_t table_width, int64_t table_stride, const int32_t* n_rows, const int32_t* parent, int32_t* table_out,
                               int64_t table_out_stride) {
    if (!ctx) return C2KV_ERR_ARG;
    try {
        return reorder(ctx, pages, n_layers, batch, width, table, table_width, table_stride, n_rows, parent, table_out, table_out_stride);
    } catch (const std::exception&) {
        return refuse(ctx, C2KV_ERR_NOMEM, "paged_reorder: host allocation failed");
    }
}

}  // extern "C"
