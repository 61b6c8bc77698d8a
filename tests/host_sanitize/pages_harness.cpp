// The host code of pages, copies of blocks and joins through a stand-in for the HIP runtime (fake_hip.h): tables and counts after random calls, which bytes the
// launches of a copy name, and what a join enqueues.  Built and run by tests/test_pages_host.py under AddressSanitizer and UBSan, one check (named on
// the command line) to a process.
#include <cstdio>

#include "fake_hip.h"
#include "kvl_plan.hip"
#include "kvl_kernels.hip"
#include "kvl_attn_plan.hip"
#include "kvl_attn_join.hip"
#include "kvl_copy_blocks.hip"
#include "kvl_pages.cpp"

using fake::launches;
using namespace kvl;

#define REQUIRE(c) do { if (!(c)) { std::printf("%s failed at line %d\n", #c, __LINE__); return 1; } } while (0)

static uint64_t rng_state = 0x9E3779B97F4A7C15ull;
static uint32_t rnd(uint32_t n) {
    rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17;
    return (uint32_t)((rng_state >> 11) % n);
}

// Every block is as often in use as tables name it, and free where none does; arrays are of exact sizes.
static int check_pages() {
    for (int it = 0; it < 60; ++it) {
        const uint32_t bs = 1 + rnd(20), blocks = 1 + rnd(it % 3 ? 200 : 5000);
        kvl_pages_t *p = nullptr;
        REQUIRE(kvl_pages(bs, blocks, &p) == KVL_OK);
        std::vector<uint64_t> all;
        for (int step = 0; step < 150; ++step) {
            std::vector<uint64_t> some;
            for (uint64_t s : all)
                if (rnd(3) == 0) some.push_back(s);
            const uint32_t n = (uint32_t)some.size();
            const uint32_t what = rnd(7);
            if (what == 0) {
                std::vector<kvl_request_t> req(1 + rnd(3), kvl_request_t{});
                std::vector<uint64_t> got(req.size());
                REQUIRE(kvl_pages_adopt(p, req.data(), (uint32_t)req.size(), got.data()) == KVL_OK);
                all.insert(all.end(), got.begin(), got.end());
            } else if (what == 1 && all.size() < 60) {
                std::vector<uint64_t> got(n);
                REQUIRE(kvl_pages_fork(p, some.data(), n, got.data()) == KVL_OK);
                all.insert(all.end(), got.begin(), got.end());
            } else if (what <= 3) {
                std::vector<uint32_t> tokens(n);
                for (uint32_t &t : tokens) t = rnd(3 * bs);
                std::vector<kvl_block_copy_t> copies(n);
                uint32_t made = 0;
                const int rc = kvl_pages_extend(p, some.data(), tokens.data(), n, copies.data(), &made);
                REQUIRE(rc == KVL_OK || (rc == KVL_ESPACE && made == 0));
            } else if (what == 4) {
                std::vector<uint32_t> tokens(n);
                REQUIRE(kvl_pages_tokens(p, some.data(), n, tokens.data()) == KVL_OK);
                for (uint32_t &t : tokens) t = rnd(t + 1);
                REQUIRE(kvl_pages_truncate(p, some.data(), tokens.data(), n) == KVL_OK);
            } else if (what == 5) {
                REQUIRE(kvl_pages_free(p, some.data(), n) == KVL_OK);
                std::vector<uint64_t> rest;
                for (uint64_t s : all)
                    if (std::find(some.begin(), some.end(), s) == some.end()) rest.push_back(s);
                all = rest;
            } else {
                kvl_pages_stats_t st{};
                REQUIRE(kvl_pages_stats(p, &st) == KVL_OK);
                std::vector<kvl_block_copy_t> copies(rnd((uint32_t)st.moves + 1));
                uint32_t made = 0;
                REQUIRE(kvl_pages_compact(p, (uint32_t)copies.size(), copies.data(), &made) == KVL_OK && made == copies.size());
            }
            std::vector<uint64_t> first(all.size() + 1);
            const int rc = kvl_pages_tables(p, all.data(), (uint32_t)all.size(), nullptr, 0, first.data());
            std::vector<int32_t> table(first.back());
            REQUIRE(rc == (table.empty() ? KVL_OK : KVL_ESPACE));
            REQUIRE(kvl_pages_tables(p, all.data(), (uint32_t)all.size(), table.data(), table.size(), first.data()) == KVL_OK);
            std::vector<uint32_t> users(blocks, 0), tokens(all.size());
            REQUIRE(kvl_pages_tokens(p, all.data(), (uint32_t)all.size(), tokens.data()) == KVL_OK);
            for (size_t i = 0; i < all.size(); ++i) REQUIRE(first[i + 1] - first[i] == (tokens[i] + bs - 1) / bs);
            for (int32_t b : table) ++users[(size_t)b];
            REQUIRE(users == p->users);
            uint64_t free = 0;
            for (uint32_t b = 0; b < blocks; ++b) {
                REQUIRE(p->free.has(b) == (users[b] == 0));
                free += users[b] == 0;
            }
            REQUIRE(p->free.count() == free);
        }
        kvl_pages_destroy(p);
    }
    return 0;
}

// What the lanes of a launch would do, on the host's memory.
static int wrong = 0;
static uint64_t pool_blocks;
template <uint32_t N>
static void run_copies(const BlockCopies<N> &a, dim3 grid, bool shared) {
    for (uint32_t z = 0; z < grid.z; ++z)
        for (uint32_t y = 0; y < grid.y; ++y)
            for (uint32_t x = 0; x < grid.x; ++x) {
                uint32_t p = 0;
                while (x >= a.plane[p].tiles_end) ++p;
                if (p >= a.n_planes) { wrong = 1; return; }
                const uint32_t tile = x - (p ? a.plane[p - 1].tiles_end : 0), run = shared ? a.runs[y] : 1u << 16 | y;
                char *base = reinterpret_cast<char *>(a.planes[z * a.n_planes + p]);
                for (uint32_t i = run & 0xffffu, end = i + (run >> 16); i < end; ++i) {
                    const kvl_block_copy_t c = a.copies[i];
                    if (c.from != a.copies[run & 0xffffu].from) { wrong = 2; return; }
                    for (uint64_t lane = 0; lane < kCopyThreads; ++lane) {
                        const uint64_t at = ((uint64_t)tile * kCopyThreads + lane) << a.plane[p].width_log2;
                        if (at >= a.plane[p].block_bytes) break;
                        std::memcpy(base + (uint64_t)c.to * a.plane[p].block_bytes + at, base + (uint64_t)c.from * a.plane[p].block_bytes + at,
                                    (size_t)1 << a.plane[p].width_log2);
                    }
                }
            }
}
static void on_copy(const fake::Launch &l, void **args) {
    if (l.kernel.find("kvl_copy_blocks_kernel") == std::string::npos) return;
    const bool shared = l.kernel.find("true") != std::string::npos;
    if (l.block.x != kCopyThreads || (uint64_t)l.grid.x * l.grid.y * l.grid.z * kCopyThreads >> 32) wrong = 3;
    if (l.kernel.find("<24u") != std::string::npos) run_copies(*static_cast<const BlockCopies<kFewCopies> *>(args[0]), l.grid, shared);
    else run_copies(*static_cast<const BlockCopies<kMostCopies> *>(args[0]), l.grid, shared);
}

static int check_copies() {
    static fake::Stream s;
    fake::watch = on_copy;
    for (int it = 0; it < 60; ++it) {
        kvl_page_layout_t lay{};
        lay.n_layers = 1 + rnd(3);
        lay.n_planes = 1 + rnd(KVL_MAX_PLANES);
        lay.pool_blocks = pool_blocks = it % 5 ? 2 + rnd(60) : 1200;
        for (uint32_t i = 0; i < lay.n_planes; ++i) lay.block_bytes[i] = it % 5 ? 1 + rnd(rnd(2) ? 60 : 9000) : 16 * (1 + rnd(8));
        if (it % 3 == 0) for (uint32_t i = 0; i < lay.n_planes; ++i) lay.block_bytes[i] = (lay.block_bytes[i] + 15) / 16 * 16;
        std::vector<std::vector<uint8_t>> planes;
        std::vector<void *> at;
        for (uint32_t i = 0; i < lay.n_layers * lay.n_planes; ++i) {
            planes.emplace_back(lay.block_bytes[i % lay.n_planes] * lay.pool_blocks);
            for (uint8_t &x : planes.back()) x = (uint8_t)rnd(256);
        }
        for (auto &x : planes) at.push_back(x.data());
        kvl_page_pools_t *pools = nullptr;
        REQUIRE(kvl_page_pools(&lay, at.data(), KVL_NO_POINTER_CHECKS, &pools) == KVL_OK);
        // sources in one half of the pool's blocks, in no order
        std::vector<int32_t> order(lay.pool_blocks);
        for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
        for (size_t i = order.size(); i > 1; --i) std::swap(order[i - 1], order[rnd((uint32_t)i)]);
        std::vector<kvl_block_copy_t> copies;
        const size_t half = order.size() / 2;
        for (size_t i = half; i < order.size(); ++i)
            copies.push_back({it % 2 && !copies.empty() && rnd(4) ? copies.back().from : order[rnd((uint32_t)half)], order[i]});
        auto want = planes;
        for (size_t i = 0; i < want.size(); ++i) {
            const uint64_t b = lay.block_bytes[i % lay.n_planes];
            for (const kvl_block_copy_t &c : copies) std::memcpy(want[i].data() + (uint64_t)c.to * b, planes[i].data() + (uint64_t)c.from * b, b);
        }
        launches.clear();
        REQUIRE(kvl_copy_blocks(pools, copies.data(), copies.size(), fake::handle(s)) == KVL_OK);
        REQUIRE(wrong == 0 && planes == want && !launches.empty());
        REQUIRE(launches.back().event);
        // a block twice, or on both sides
        launches.clear();
        auto bad = copies;
        bad.push_back(copies[0]);
        REQUIRE(kvl_copy_blocks(pools, bad.data(), bad.size(), fake::handle(s)) == KVL_EALIAS);
        bad.back() = {copies[0].to, copies[0].from};
        REQUIRE(kvl_copy_blocks(pools, bad.data(), bad.size(), fake::handle(s)) == KVL_EALIAS);
        for (int32_t b : {-1, (int32_t)lay.pool_blocks}) {
            bad.back() = {b, copies[0].from};
            REQUIRE(kvl_copy_blocks(pools, bad.data(), bad.size(), fake::handle(s)) == KVL_ERANGE);
        }
        REQUIRE(launches.empty() && kvl_copy_blocks(pools, nullptr, 0, fake::handle(s)) == KVL_OK && launches.empty());
        kvl_page_pools_destroy(pools);
    }
    // more lanes than a launch has for one copy
    kvl_page_layout_t lay{};
    lay.n_layers = 4096;
    lay.n_planes = 1;
    lay.pool_blocks = 2;
    lay.block_bytes[0] = 1u << 20;
    for (uintptr_t odd : {0u, 1u}) {
        std::vector<void *> at(4096, reinterpret_cast<void *>((uintptr_t)1 << 40 | odd));
        kvl_page_pools_t *pools = nullptr;
        REQUIRE(kvl_page_pools(&lay, at.data(), KVL_NO_POINTER_CHECKS, &pools) == KVL_OK);
        const kvl_block_copy_t one{0, 1};
        fake::watch = nullptr;
        REQUIRE(kvl_copy_blocks(pools, &one, 1, fake::handle(s)) == (odd ? KVL_ERANGE : KVL_OK));
        kvl_page_pools_destroy(pools);
    }
    return 0;
}

static int check_joins() {
    static fake::Stream s;
    for (int it = 0; it < 200; ++it) {
        kvl_attn_layout_t lay{};
        lay.block_tokens = 16;
        lay.q_heads = lay.kv_heads = 1 + rnd(40);
        lay.head_dim = rnd(2) ? 64 : 128;
        lay.dtype = lay.cache_dtype = rnd(2) ? KVL_F16 : KVL_BF16;
        const uint32_t tokens = rnd(it % 4 ? 50 : 5000);
        std::vector<int32_t> table(tokens / 16 + 1);
        for (size_t i = 0; i < table.size(); ++i) table[i] = (int32_t)i;
        lay.pool_blocks = table.size();
        kvl_request_t r{};
        r.append_tokens = tokens;
        r.block_table = table.data();
        r.n_blocks = (uint32_t)table.size();
        kvl_attn_plan_t *p = nullptr;
        REQUIRE(kvl_attn_plan(&lay, &r, 1, KVL_GATHER | KVL_NO_POINTER_CHECKS, &p) == KVL_OK);
        const uint32_t n = 1 + rnd(KVL_JOIN_MOST);
        std::vector<const void *> parts(n);
        std::vector<const float *> lses(n);
        std::vector<uint64_t> strides(n, (uint64_t)lay.q_heads * lay.head_dim + 8 * rnd(3));
        for (uint32_t i = 0; i < n; ++i) {
            parts[i] = reinterpret_cast<const void *>((uintptr_t)(i + 1) << 40);
            lses[i] = reinterpret_cast<const float *>((uintptr_t)(i + 100) << 40);
        }
        kvl_attn_join_t t{};
        t.n_parts = n;
        t.parts = parts.data();
        t.part_strides = strides.data();
        t.lses = lses.data();
        t.out = reinterpret_cast<void *>((uintptr_t)99 << 40);
        launches.clear();
        REQUIRE(kvl_attn_join(p, &t, fake::handle(s)) == KVL_OK);
        const uint64_t pieces = (uint64_t)tokens * lay.q_heads * lay.head_dim / 8;
        REQUIRE(launches.size() == (tokens ? 1 : 0));
        if (tokens) REQUIRE((uint64_t)launches[0].grid.x * launches[0].block.x >= pieces && (uint64_t)(launches[0].grid.x - 1) * launches[0].block.x < pieces);
        launches.clear();
        if (tokens) {
            for (int what = 0; what < 5; ++what) {
                kvl_attn_join_t u = t;
                auto other = strides;
                u.part_strides = other.data();
                if (what == 0) u.n_parts = 0;
                if (what == 1) u.n_parts = KVL_JOIN_MOST + 1;
                if (what == 2) u.out = reinterpret_cast<void *>(((uintptr_t)99 << 40) + 8);
                if (what == 3) other[n - 1] += 1;
                if (what == 4) { u.out = const_cast<void *>(parts[0]); u.out_stride = strides[0] + 8; }
                REQUIRE(kvl_attn_join(p, &u, fake::handle(s)) == KVL_EINVAL && launches.empty());
            }
        }
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

int main(int argc, char **argv) {
    const std::map<std::string, int (*)()> checks = {{"copies", check_copies}, {"joins", check_joins}, {"pages", check_pages}};
    if (argc != 2 || !checks.count(argv[1])) {
        for (const auto &c : checks) std::printf("%s\n", c.first.c_str());
        return argc == 1 ? 0 : 2;
    }
    const int rc = checks.at(argv[1])();
    if (rc == 0) std::printf("ok\n");
    return rc;
}
