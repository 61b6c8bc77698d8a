// The attention operators' host code through a stand-in for the HIP runtime (fake_hip.h): what the plans' lists name, which kernel takes which
// rows, and what the two calls enqueue.  Built and run by tests/test_attn_host.py under AddressSanitizer and UBSan, one check (named on the
// command line) to a process.
#include <cstdio>

#include "fake_hip.h"
#include "kvl_plan.hip"
#include "kvl_kernels.hip"
#include "kvl_attn_plan.hip"
#include "kvl_append.hip"
#include "kvl_attn.hip"

using fake::launches;
using namespace kvl;

#define REQUIRE(c) do { if (!(c)) { std::printf("%s failed at line %d\n", #c, __LINE__); return 1; } } while (0)

static uint64_t rng_state = 0x9E3779B97F4A7C15ull;
static uint32_t rnd(uint32_t n) {
    rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17;
    return (uint32_t)((rng_state >> 11) % n);
}

// A batch with tables of its own blocks, in no order.
struct Batch {
    kvl_attn_layout_t lay{};
    std::vector<kvl_request_t> req;
    std::vector<std::vector<int32_t>> tables;
    Batch(uint32_t bs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t cache) {
        lay.block_tokens = bs;
        lay.q_heads = q_heads;
        lay.kv_heads = kv_heads;
        lay.head_dim = dim;
        lay.dtype = KVL_BF16;
        lay.cache_dtype = cache;
    }
    void add(uint32_t hit, uint32_t app) {
        kvl_request_t r{};
        r.hit_tokens = hit;
        r.append_tokens = app;
        r.n_blocks = (hit + app + lay.block_tokens - 1) / lay.block_tokens;
        req.push_back(r);
    }
    kvl_attn_plan_t *plan(uint32_t flags) {
        uint32_t next = 0;
        tables.clear();
        for (kvl_request_t &r : req) {
            tables.emplace_back(r.n_blocks);
            for (int32_t &b : tables.back()) b = (int32_t)next++;
        }
        for (uint32_t i = 0; i < next; ++i) {           // blocks change places
            const uint32_t a = rnd((uint32_t)req.size()), b = rnd((uint32_t)req.size());
            if (req[a].n_blocks && req[b].n_blocks) std::swap(tables[a][rnd(req[a].n_blocks)], tables[b][rnd(req[b].n_blocks)]);
        }
        for (size_t i = 0; i < req.size(); ++i) req[i].block_table = tables[i].data();
        lay.pool_blocks = next + 1;
        kvl_attn_plan_t *p = nullptr;
        return kvl_attn_plan(&lay, req.data(), (uint32_t)req.size(), flags | KVL_NO_POINTER_CHECKS, &p) == KVL_OK ? p : nullptr;
    }
};

template <typename X>
static const X *list(const kvl_attn_plan_t *p, uint64_t at) { return reinterpret_cast<const X *>(reinterpret_cast<const char *>(p->base.d_units) + at); }

static int check_lists() {
    for (int it = 0; it < 200; ++it) {
        const uint32_t group = 1 + rnd(8), kv = 1u << rnd(4);
        Batch b(1 + rnd(it % 4 ? 40 : 300), group * kv, kv, rnd(2) ? 64 : 128, rnd(2) ? KVL_E4M3 : KVL_BF16);
        if (rnd(2)) {
            b.lay.window = 1 + rnd(600);
            b.lay.sinks = rnd(3) ? rnd(8) : rnd(1000);
        }
        for (uint32_t n = 1 + rnd(6); n--;) b.add(rnd(it % 5 ? 900 : 20000), rnd(rnd(2) ? 4 : 300));
        const uint32_t range[] = {0, KVL_TOKENS_APPEND, KVL_TOKENS_ALL};
        const uint32_t r = range[rnd(3)];
        kvl_attn_plan_t *p = b.plan(KVL_GATHER | KVL_SCATTER | r);
        REQUIRE(p);
        uint64_t tokens = 0, entries = 0;
        std::vector<uint64_t> token0, table0;
        for (const kvl_request_t &q : b.req) {
            token0.push_back(tokens);
            table0.push_back(entries);
            tokens += q.append_tokens;
            entries += q.n_blocks;
        }
        REQUIRE(p->new_tokens == tokens);
        // every place of every item is a token of its request's range, found in the table as the kernels find it
        const AttnItem *items = list<AttnItem>(p, p->off_items);
        const int32_t *tables = list<int32_t>(p, p->off_tables);
        const uint64_t floats = p->workspace_bytes / 4;
        std::vector<uint8_t> written(floats, 0);
        std::vector<uint32_t> rows_done(tokens * group, 0);
        REQUIRE(p->items.size() == p->class_first[kAttnClasses]);
        for (uint32_t c = 0; c < kAttnClasses; ++c)
            for (uint32_t i = p->class_first[c]; i < p->class_first[c + 1]; ++i) {
                const AttnItem &x = items[i];
                const uint32_t q = p->items[i].request;
                REQUIRE(x.token0 == token0[q] && x.table == table0[q] && x.hit == b.req[q].hit_tokens);
                REQUIRE(x.n_rows >= 1 && x.n_rows <= kClassRows[c] && x.first_row + x.n_rows <= b.req[q].append_tokens * group);
                REQUIRE(x.begin <= x.end);
                const uint64_t first = r == KVL_TOKENS_APPEND ? x.hit : 0, last = r ? x.hit + b.req[q].append_tokens : x.hit;
                for (uint32_t v = x.begin; v < x.end; ++v) {
                    const uint32_t t = v < x.sinks ? v : v + x.gap;
                    REQUIRE(t >= first && t < last);
                    const uint32_t block = (uint32_t)(((uint64_t)(2 * t) * p->div_mul) >> 32) >> p->div_shift;
                    REQUIRE(block == t / b.lay.block_tokens && block < b.req[q].n_blocks);
                    REQUIRE(tables[x.table + block] == b.tables[q][block]);
                }
                if (x.pieces > 1) {                     // its part of the workspace is in nobody else's use
                    const uint64_t size = partial_floats(kClassRows[c], b.lay.head_dim) * b.lay.kv_heads;
                    REQUIRE(x.partial % 2 == 0 && x.partial + size <= floats);
                    for (uint64_t f = x.partial; f < x.partial + size; ++f) REQUIRE(!written[f]++);
                } else {
                    for (uint32_t row = 0; row < x.n_rows; ++row) ++rows_done[x.token0 * group + x.first_row + row];
                }
            }
        const JoinItem *joins = list<JoinItem>(p, p->off_join);
        uint64_t joined = 0;
        for (uint32_t i = 0; i < p->n_join; ++i) {
            const JoinItem &j = joins[i];
            const uint64_t size = partial_floats(j.tile_rows, b.lay.head_dim) * b.lay.kv_heads;
            REQUIRE(j.pieces > 1 && j.partial + j.pieces * size <= floats && j.n_rows <= j.tile_rows);
            REQUIRE(p->join_groups() * (4 / p->join_waves()) >= j.n_rows && j.pieces <= p->most_pieces);
            joined += j.pieces * size;
            for (uint32_t row = 0; row < j.n_rows; ++row) ++rows_done[j.token0 * group + j.first_row + row];
        }
        REQUIRE(joined == floats);
        for (uint32_t n : rows_done) REQUIRE(n == 1);
        // new tokens: a row of the pool each, and every receiving block once
        const AppendToken *places = list<AppendToken>(p, p->off_tokens);
        const AppendBlock *blocks = list<AppendBlock>(p, p->off_blocks);
        std::vector<uint8_t> row_taken(b.lay.pool_blocks * b.lay.block_tokens, 0);
        for (size_t q = 0; q < b.req.size(); ++q)
            for (uint32_t n = 0; n < b.req[q].append_tokens; ++n) {
                const AppendToken &a = places[token0[q] + n];
                const uint32_t t = b.req[q].hit_tokens + n;
                REQUIRE(a.position == t && a.position <= p->last_position);
                REQUIRE(a.pool_row == (uint32_t)b.tables[q][t / b.lay.block_tokens] * b.lay.block_tokens + t % b.lay.block_tokens && !row_taken[a.pool_row]++);
            }
        uint64_t in_blocks = 0;
        for (uint32_t i = 0; i < p->n_append_blocks; ++i) {
            const AppendBlock &a = blocks[i];
            REQUIRE(a.n >= 1 && a.n <= p->most_append_rows && a.row + a.n <= b.lay.block_tokens);
            for (uint32_t n = 0; n < a.n; ++n)
                REQUIRE(places[a.token + n].pool_row == a.block * b.lay.block_tokens + a.row + n && places[a.token + n].position == a.position + n);
            in_blocks += a.n;
        }
        REQUIRE(in_blocks == (b.lay.cache_dtype == KVL_E4M3 ? tokens : 0));
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

// A token's block by one product, for all block sizes.
static int check_division() {
    for (uint64_t bs : {1ull, 2ull, 3ull, 5ull, 7ull, 16ull, 24ull, 100ull, 65535ull, 65537ull, 1000003ull, (1ull << 30) - 1, (1ull << 30) + 1, (1ull << 31) - 1, 1ull << 31, (1ull << 31) + 1, (1ull << 32) - 1}) {
        Batch b((uint32_t)bs, 1, 1, 64, KVL_BF16);
        b.add(0, 1);
        b.req[0].n_blocks = 1;
        std::vector<int32_t> one(1, 0);
        b.req[0].block_table = one.data();
        b.lay.pool_blocks = 1;
        kvl_attn_plan_t *p = nullptr;
        REQUIRE(kvl_attn_plan(&b.lay, b.req.data(), 1, KVL_GATHER | KVL_HOST_ONLY, &p) == KVL_OK);
        auto found = [&](uint32_t t) { return (uint32_t)(((uint64_t)(2 * t) * p->div_mul) >> 32) >> p->div_shift; };
        for (uint64_t k = 0; k < 40000; ++k) {          // both sides of blocks' edges, and anywhere
            const uint64_t edge = (k % 2 ? k / 2 : ((1ull << 31) / bs) - std::min<uint64_t>(k / 2, (1ull << 31) / bs)) * bs;
            for (uint64_t t : {edge, edge ? edge - 1 : 0, (uint64_t)rnd(1u << 31)})
                if (t < 1ull << 31) REQUIRE(found((uint32_t)t) == t / bs);
        }
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

static uint32_t in_class(const kvl_attn_plan_t *p, uint32_t c) { return p->class_first[c + 1] - p->class_first[c]; }

// Few rows: one launch, of the widest kernel among them, where keys times heads are at most 2^21; else each in its own.
static int check_classes() {
    Batch b(16, 32, 4, 128, KVL_E4M3);          // 8 rows a token
    b.add(100, 1);                              // 8 rows
    b.add(200, 3);                              // 24
    b.add(300, 6);                              // 48
    b.add(50, 40);                              // 320: three tiles
    kvl_attn_plan_t *p = b.plan(KVL_GATHER | KVL_TOKENS_ALL);
    REQUIRE(p && in_class(p, kRows16) == 0 && in_class(p, kRows32) == 0 && in_class(p, kRows64) == 3 && in_class(p, kRows128) == 3);
    kvl_attn_plan_destroy(p);
    b.req.pop_back();
    b.req.pop_back();
    p = b.plan(KVL_GATHER | KVL_TOKENS_ALL);
    REQUIRE(p && in_class(p, kRows16) == 0 && in_class(p, kRows32) == 2 && in_class(p, kRows64) == 0 && in_class(p, kRows128) == 0);
    kvl_attn_plan_destroy(p);
    // 4 heads: up to 2^19 keys
    const uint32_t all = 1u << 19;
    for (uint32_t more : {0u, 1u}) {
        b.req.clear();
        b.add(all - 1000 - 1 - 3 + more, 1);
        b.add(1000, 3);
        p = b.plan(KVL_GATHER | KVL_TOKENS_ALL);
        REQUIRE(p && (in_class(p, kRows16) != 0) == (more != 0) && in_class(p, kRows32) != 0);
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

static std::vector<AppendArgs> append_calls;
static bool is(const fake::Launch &l, const char *kernel) { return l.kernel.find(kernel) != std::string::npos; }
static fake::Stream s;                          // (outlives the plans' events)
static void *somewhere(uint64_t n) { return (void *)(n << 40); }

// Launches: the widest rows first, the join last, the plan's event on the last one alone, and none where the caller synchronises.
static int check_attn_launches() {
    for (uint32_t flags : {0u, (uint32_t)KVL_CALLER_SYNCS}) {
        Batch b(16, 32, 4, 128, KVL_E4M3);
        b.add(600000, 1);
        b.add(1000, 3);
        b.add(0, 40);
        kvl_attn_plan_t *p = b.plan(KVL_GATHER | KVL_TOKENS_ALL | flags);
        REQUIRE(p && p->n_join && p->workspace_bytes);
        kvl_attn_t a{};
        a.q = somewhere(1);
        a.out = somewhere(2);
        a.scale = 1;
        a.workspace = somewhere(3);
        a.workspace_bytes = p->workspace_bytes - 1;
        const void *planes[4] = {somewhere(4), somewhere(5), somewhere(6), somewhere(7)};
        launches.clear();
        REQUIRE(kvl_attn_layer(p, &a, planes, fake::handle(s)) == KVL_ESPACE && launches.empty());
        ++a.workspace_bytes;
        REQUIRE(kvl_attn_layer(p, &a, planes, fake::handle(s)) == KVL_OK);
        REQUIRE(launches.size() == 4);
        REQUIRE(is(launches[0], "kvl_attn_many_kernel") && is(launches[3], "kvl_attn_join_kernel"));
        for (int i = 0; i < 4; ++i) {
            REQUIRE(launches[i].stream == &s && launches[i].event == (i == 3 && !flags));
            if (i < 3) REQUIRE(launches[i].block.x == 256 && launches[i].grid.x == in_class(p, i == 0 ? kRows128 : i == 1 ? kRows32 : kRows16) * 4);
        }
        REQUIRE(launches[3].grid.x == p->n_join * 4 * p->join_groups());
        a.out = const_cast<void *>(a.q);                // in place: at one stride
        a.q_stride = a.out_stride = 8192;
        REQUIRE(kvl_attn_layer(p, &a, planes, fake::handle(s)) == KVL_OK);
        a.out_stride = 0;
        REQUIRE(kvl_attn_layer(p, &a, planes, fake::handle(s)) == KVL_EINVAL);
        fake::finish(&s);
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

// Appends: one launch, or queries in their own from 5 * 2^20 tasks on, and several beyond 2^30.
static int check_append_launches() {
    struct { uint32_t heads, tokens, cache; size_t want; } cases[] = {
        {64, 10240, KVL_E4M3, 1}, {64, 10241, KVL_E4M3, 2}, {64, 10241, KVL_BF16, 1}, {65536, 2047, KVL_BF16, 1}, {65536, 4100, KVL_BF16, 3}, {65536, 4100, KVL_E4M3, 4}};
    for (const auto &c : cases) {
        Batch b(64, c.heads, 1, 128, c.cache);
        b.lay.rope_dim = 128;
        b.add(70, c.tokens);
        kvl_attn_plan_t *p = b.plan(KVL_SCATTER);
        REQUIRE(p);
        kvl_append_t a{};
        a.k = somewhere(1);
        a.v = somewhere(2);
        a.q = somewhere(3);
        a.q_out = somewhere(4);
        a.rope = (const float *)somewhere(5);
        a.rope_positions = 70 + c.tokens;
        void *planes[4] = {somewhere(6), somewhere(7), somewhere(8), somewhere(9)};
        append_calls.clear();
        launches.clear();
        fake::watch = [](const fake::Launch &, void **args) { append_calls.push_back(*static_cast<AppendArgs *>(args[0])); };
        REQUIRE(kvl_append_layer(p, &a, planes, fake::handle(s)) == KVL_OK);
        fake::watch = nullptr;
        REQUIRE(launches.size() == c.want);
        const uint64_t per_token = c.heads * 8 + (c.cache == KVL_E4M3 ? 0 : 16);
        uint64_t tokens = 0;
        for (size_t i = 0; i < launches.size(); ++i) {
            const uint64_t lanes = (uint64_t)launches[i].grid.x * launches[i].block.x;
            REQUIRE(launches[i].event == (i + 1 == launches.size()) && lanes < 1ull << 32);
            const bool codes = is(launches[i], "codes");
            REQUIRE(codes == (c.cache == KVL_E4M3 && i == 0));
            if (codes) {
                const uint64_t work = (uint64_t)p->n_append_blocks * launches[i].block.x;
                REQUIRE(p->n_append_blocks && lanes >= work + (c.want == 1 ? c.tokens * per_token : 0));
                if (c.want == 1) tokens = c.tokens;
                continue;
            }
            REQUIRE(append_calls[i].token_first == tokens && append_calls[i].tasks % per_token == 0 && append_calls[i].tasks <= 1ull << 30);
            REQUIRE(lanes >= append_calls[i].tasks && lanes < append_calls[i].tasks + 256);
            tokens += append_calls[i].tasks / per_token;
        }
        REQUIRE(tokens == c.tokens);
        a.rope_positions = 70 + c.tokens - 1;
        REQUIRE(kvl_append_layer(p, &a, planes, fake::handle(s)) == KVL_ESPACE);
        fake::finish(&s);
        kvl_attn_plan_destroy(p);
    }
    return 0;
}

// A stride with which the last token would lie beyond what 64 bits number is refused, and does not come out as a small extent.
static int check_strides() {
    const uint32_t n = (1u << 23) + 1;
    Batch b(1u << 24, 1, 1, 64, KVL_BF16);
    b.add(0, n);
    kvl_attn_plan_t *p = b.plan(KVL_SCATTER | KVL_GATHER | KVL_TOKENS_APPEND);
    REQUIRE(p);
    void *planes[2] = {somewhere(6), somewhere(7)};
    const void *from[2] = {planes[0], planes[1]};
    for (uint64_t stride : {1ull << 40, (1ull << 37) + 8, 1ull << 62, ~7ull}) {
        uint64_t kvl_append_t::*strides[] = {&kvl_append_t::k_stride, &kvl_append_t::v_stride, &kvl_append_t::q_stride, &kvl_append_t::q_out_stride};
        for (auto field : strides) {
            kvl_append_t a{};
            a.k = somewhere(1);
            a.v = somewhere(2);
            a.q = somewhere(3);
            a.q_out = somewhere(4);
            launches.clear();
            REQUIRE(kvl_append_layer(p, &a, planes, fake::handle(s)) == KVL_OK && !launches.empty());
            a.*field = stride;
            launches.clear();
            REQUIRE(kvl_append_layer(p, &a, planes, fake::handle(s)) == KVL_EINVAL && launches.empty());
        }
        for (bool out : {false, true}) {
            kvl_attn_t a{};
            a.q = somewhere(1);
            a.out = somewhere(2);
            a.scale = 1;
            a.workspace = somewhere(3);
            a.workspace_bytes = p->workspace_bytes;
            (out ? a.out_stride : a.q_stride) = stride;
            launches.clear();
            REQUIRE(kvl_attn_layer(p, &a, from, fake::handle(s)) == KVL_EINVAL && launches.empty());
        }
    }
    fake::finish(&s);
    kvl_attn_plan_destroy(p);
    return 0;
}

int main(int argc, char **argv) {
    const std::map<std::string, int (*)()> checks = {
        {"lists", check_lists}, {"division", check_division}, {"classes", check_classes}, {"attn_launches", check_attn_launches}, {"append_launches", check_append_launches}, {"strides", check_strides}};
    if (argc != 2 || !checks.count(argv[1])) {
        for (const auto &c : checks) std::printf("%s\n", c.first.c_str());
        return argc == 1 ? 0 : 2;
    }
    const int rc = checks.at(argv[1])();
    if (rc == 0) std::printf("ok\n");
    return rc;
}
