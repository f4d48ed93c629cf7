// Host code of generation that branches over the stand-in runtime: one scenario a run (its name is the argument).
#include <c2kv.h>

#include <cstdio>
#include <cstdlib>
#include <string>
#include <utility>
#include <vector>

#include "fake_cudart.h"

namespace {

#define CHECK(cond, ...)                                                \
    do {                                                                \
        if (!(cond)) {                                                  \
            std::printf("%s:%d: %s: ", __FILE__, __LINE__, #cond);      \
            std::printf(__VA_ARGS__);                                   \
            std::printf("\n");                                          \
            std::exit(1);                                               \
        }                                                               \
    } while (0)

alignas(256) char buffer[256];          // every tensor: its address is checked, nothing is read
int32_t* const ints = reinterpret_cast<int32_t*>(buffer);
float* const floats = reinterpret_cast<float*>(buffer);
constexpr int kBf16 = C2KV_DTYPE_BF16, kF32 = C2KV_DTYPE_F32;

struct Context {
    c2kv_ctx* ctx = nullptr;
    Context(int dtype, int hq, int hkv, int d) {
        c2kv_config cfg{};
        cfg.layers = 1;
        cfg.n_q_heads = hq;
        cfg.n_kv_heads = hkv;
        cfg.head_dim = d;
        cfg.rope_theta = 1e4;
        cfg.dtype = dtype;
        cfg.pool_slots = 64;
        CHECK(c2kv_create(&cfg, nullptr, &ctx) == C2KV_OK, "create: %s", c2kv_last_error(nullptr));
    }
    ~Context() { c2kv_destroy(ctx); }
    static c2kv_pages pages(bool codes) {
        c2kv_pages p{};
        p.k = p.v = buffer;
        p.k_scale = p.v_scale = floats;
        p.n_pages = 1 << 20;
        p.page_size = 64;
        p.format = codes ? C2KV_PAGES_E4M3 : C2KV_PAGES_NATIVE;
        return p;
    }
    // trees of `nodes` nodes after `rows` rows each
    c2kv_status tree(int batch, int nodes, int rows, bool codes) {
        const c2kv_pages p = pages(codes);
        std::vector<int32_t> ptr(batch + 1), keys(batch, rows + nodes);
        for (int r = 0; r <= batch; ++r) ptr[r] = r * nodes;
        const int32_t width = (rows + nodes + 63) / 64;
        return c2kv_paged_attend_tree(ctx, &p, batch, ints, width, width, ptr.data(), keys.data(), ints, 0, buffer, 0, nullptr, buffer, nullptr);
    }
    c2kv_status select(int batch, int width, int vocab) {
        return c2kv_beam_select(ctx, batch, width, vocab, width, kF32, buffer, 0, nullptr, floats, nullptr, -1, ints, ints, floats, nullptr);
    }
};

int grid(const char* kernel) {
    for (const fake::Launch& l : fake::launches)
        if (l.kernel.find(kernel) != std::string::npos) return (int)l.grid.x;
    return 0;
}

// The kernel that a call goes to: by its keys first, then by its rows.
void tree_routes() {
    const struct {
        int dtype, hq, hkv, d, batch, nodes, rows;
        bool codes;
        const char* kernel;
    } kinds[] = {
        {kBf16, 32, 8, 128, 1, 16, 1500, true, "paged_mma_kernel"},     {kBf16, 32, 8, 128, 1, 64, 100, false, "paged_mma_kernel"},
        {kBf16, 32, 8, 128, 1, 4, 60000, true, "paged_mma_kernel"},     {kBf16, 32, 8, 128, 1, 32, 60000, true, "paged_direct_kernel"},
        {kBf16, 32, 8, 128, 1, 5, 60000, false, "paged_direct_kernel"}, {kBf16, 32, 8, 64, 1, 8, 60000, true, "paged_mma_kernel"},
        {kBf16, 8, 8, 64, 1, 512, 60000, true, "paged_direct_kernel"},  {kBf16, 32, 8, 128, 1, 129, 9000, false, "paged_tc_kernel"},
        {kBf16, 32, 8, 128, 200, 32, 10, true, "paged_direct_kernel"},  {kF32, 16, 4, 64, 3, 26, 300, false, "paged_lane_kernel"},
        {kF32, 16, 4, 64, 3, 64, 9000, false, "paged_simt_kernel"},     {kF32, 16, 4, 64, 3, 1, 9000, true, "paged_lane_kernel"}};
    for (const auto& k : kinds) {
        Context one(k.dtype, k.hq, k.hkv, k.d);
        fake::launches.clear();
        CHECK(one.tree(k.batch, k.nodes, k.rows, k.codes) == C2KV_OK, "%s: %s", k.kernel, c2kv_last_error(one.ctx));
        for (const char* other : {"paged_mma_kernel", "paged_direct_kernel", "paged_tc_kernel", "paged_lane_kernel", "paged_simt_kernel"})
            CHECK(fake::launched(other) == (std::string(other) == k.kernel), "%s for %s: %d nodes after %d rows", other, k.kernel, k.nodes, k.rows);
    }
    // 64 rows of each of 8 heads: eight a CTA, 16 where eights are more than one wave of CTAs, else another kernel
    Context few(kBf16, 32, 8, 128);
    for (const auto& [batch, ctas] : {std::pair{1, 64}, std::pair{8, 8 * 32}, std::pair{16, 0}}) {
        fake::launches.clear();
        CHECK(few.tree(batch, 16, 0, true) == C2KV_OK, "%s", c2kv_last_error(few.ctx));
        CHECK(grid("paged_mma_kernel") == ctas, "%d requests: %d CTAs", batch, grid("paged_mma_kernel"));
    }
}

// A captured call leaves its scratch to the graph, warm or not, and later calls alone.
void tree_capture() {
    for (const int nodes : {16, 64, 300})
        for (int warm = 0; warm < 2; ++warm) {
            Context one(kBf16, 32, 8, 128);
            if (warm) CHECK(one.tree(1, nodes, 9000, true) == C2KV_OK, "%s", c2kv_last_error(one.ctx));
            fake::pool_allocations.clear();
            fake::capturing = true;
            const c2kv_status st = one.tree(1, nodes, 9000, true);
            fake::capturing = false;
            CHECK(st == C2KV_OK, "%d nodes captured, warm %d: %s", nodes, warm, c2kv_last_error(one.ctx));
            // its partials (and notes), and the key tiles of many rows
            CHECK(fake::pool_allocations.size() == (nodes == 300 ? 2u : 1u), "%d nodes: %zu allocations", nodes, fake::pool_allocations.size());
            CHECK(one.tree(8, nodes, 60000, true) == C2KV_OK, "%s", c2kv_last_error(one.ctx));
        }
    Context beams(kBf16, 32, 8, 128);
    fake::pool_allocations.clear();
    fake::capturing = true;
    const c2kv_status st = beams.select(4, 4, 100000);
    fake::capturing = false;
    CHECK(st == C2KV_OK && fake::pool_allocations.size() == 1, "%zu", fake::pool_allocations.size());
}

// Without memory for partials keys are not cut; without any, rows go key by key.  A choice among beams needs its own.
void tree_no_memory() {
    const size_t least = 4 << 20;                                // a context's scratch: notes of tiles fit, ten megabytes of partials do not
    Context one(kBf16, 32, 8, 128), none(kBf16, 32, 8, 128), less(kBf16, 32, 8, 128);
    fake::launches.clear();
    CHECK(one.tree(1, 64, 30000, false) == C2KV_OK, "%s", c2kv_last_error(one.ctx));
    CHECK(grid("paged_direct_kernel") > 16 && fake::launched("paged_join_kernel"), "keys are cut when there is memory");
    fake::alloc_fails = [=](size_t bytes) { return bytes > least; };
    fake::launches.clear();
    CHECK(less.tree(1, 64, 30000, false) == C2KV_OK, "%s", c2kv_last_error(less.ctx));
    CHECK(grid("paged_direct_kernel") == 16 && !fake::launched("paged_join_kernel"), "%d CTAs", grid("paged_direct_kernel"));
    fake::alloc_fails = [](size_t) { return true; };
    fake::launches.clear();
    CHECK(none.tree(1, 64, 30000, false) == C2KV_OK, "%s", c2kv_last_error(none.ctx));
    CHECK(fake::launched("paged_mma_kernel") && !fake::launched("paged_direct_kernel"), "no memory at all");
    fake::launches.clear();
    CHECK(none.select(4, 4, 100000) == C2KV_ERR_NOMEM && fake::launches.empty(), "%s", c2kv_last_error(none.ctx));
    CHECK(cudaGetLastError() == cudaSuccess, "the refusal of memory stays behind");
    fake::alloc_fails = [](size_t) { return false; };
    CHECK(none.select(4, 4, 100000) == C2KV_OK, "%s", c2kv_last_error(none.ctx));
}

// The walk, kept rows and reordered beams ask for no memory, and cover every request and layer.
void moves() {
    Context one(kBf16, 32, 8, 128);
    fake::alloc_fails = [](size_t) { return true; };
    fake::pool_allocations.clear();
    for (const int batch : {1, 300})
        for (const int layers : {1, 4, 32, 100}) {
            const std::vector<c2kv_pages> pages(layers, Context::pages(true));
            std::vector<int32_t> ptr(batch + 1), rows(batch, 40);
            for (int r = 0; r <= batch; ++r) ptr[r] = r * 7;
            auto ctas = [&](const char* kernel) {
                size_t n = 0;
                for (const fake::Launch& l : fake::launches) n += l.kernel.find(kernel) != std::string::npos ? (size_t)l.grid.x * l.grid.y : 0;
                return n;
            };
            fake::launches.clear();
            CHECK(c2kv_paged_keep(one.ctx, pages.data(), layers, batch, ints, 4, 4, ptr.data(), rows.data(), ints, ints) == C2KV_OK, "%s",
                  c2kv_last_error(one.ctx));
            CHECK(ctas("paged_keep_kernel") == (size_t)batch * layers, "%zu", ctas("paged_keep_kernel"));
            CHECK(c2kv_paged_reorder(one.ctx, pages.data(), layers, batch, 5, ints, 4, 4, rows.data(), ints, ints + (1 << 20), 4) == C2KV_OK, "%s",
                  c2kv_last_error(one.ctx));
            CHECK(ctas("paged_reorder_kernel") == (size_t)batch * 5 * layers, "%zu", ctas("paged_reorder_kernel"));
            CHECK(c2kv_verify_tree(one.ctx, batch, ptr.data(), 1000, ints, ints, floats, 0, floats, ints, ints, ints) == C2KV_OK, "%s",
                  c2kv_last_error(one.ctx));
            CHECK(ctas("verify_tree_kernel") >= (size_t)batch, "%zu", ctas("verify_tree_kernel"));
        }
    CHECK(fake::pool_allocations.empty(), "%zu allocations", fake::pool_allocations.size());
    fake::alloc_fails = [](size_t) { return false; };
}

}  // namespace

int main(int argc, char** argv) {
    const std::string name = argc > 1 ? argv[1] : "";
    if (name == "tree_routes") tree_routes();
    else if (name == "tree_capture") tree_capture();
    else if (name == "tree_no_memory") tree_no_memory();
    else if (name == "moves") moves();
    else CHECK(false, "unknown scenario '%s'", name.c_str());
    std::printf("ok\n");
}
