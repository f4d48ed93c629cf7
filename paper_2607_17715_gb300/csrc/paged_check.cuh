// Argument checks that the paged calls' entry points share.
#pragma once

#include "c2kv.h"
#include "paged.cuh"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <initializer_list>

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

}  // namespace
