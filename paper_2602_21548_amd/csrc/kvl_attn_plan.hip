// Plans of the attention operators: from a batch to the lists of work of the append and attention kernels (host).
#include <algorithm>
#include <cstring>
#include <new>

#include "kvl_attn_internal.h"

namespace kvl {

namespace {
// The visible keys of some rows of one request, and the way they are numbered.
struct Places {
    uint32_t begin, end, sinks, gap;
};
struct Tile {
    uint32_t request, first_row, n_rows, cls;       // (cls: AttnClass)
    Places at;
};
}  // namespace

// Keys [first, last) of the plan, queries at positions [p0, p1]: what at least one of them sees.
static Places places_of(const kvl_attn_layout_t &l, uint64_t first, uint64_t last, uint64_t p0, uint64_t p1) {
    const uint64_t end = std::max(first, std::min(last, p1 + 1));
    uint64_t lo = first;
    if (l.window) lo = std::min(end, std::max(first, p0 + 1 > l.window ? p0 + 1 - l.window : 0));
    const uint64_t sinks = std::max(first, std::min<uint64_t>(l.sinks, lo));
    return {(uint32_t)first, (uint32_t)(sinks + end - lo), (uint32_t)sinks, (uint32_t)(lo - sinks)};
}

// How long the pieces are that the keys of a class's tiles are cut into, each one workgroup a cache head.
//
// A workgroup costs what `more` keys cost beside its own (finding its work, the first keys' way from memory, joining); the machine has room
// for `slots` of them at once.  Up to that many run side by side, and the longest counts; more of them come in rounds, the last of
// which is half empty on average; where anything is cut, the results have to be joined: written and read in 32 bits, `join` keys' time for each
// workgroup at the rate at which all of them together take keys.  The length is the one, of a row of them, for which this
// is least.  Whole steps are tiles for every wavefront.
struct Machine {
    uint32_t step, more, slots;
    double join;
};
constexpr uint32_t kJoinKeys = 256;
static Machine machine_of(const kvl_attn_layout_t &l, uint32_t c) {
    // (Heads of 64 have room for 768 tiles of 128 rows and not 512, which is as good for most batches: tails of 256-1024 tokens over 8-32 K
    // keys 450 us with 512 and 453 with 768, but one of 1024 over 8192 121 and 115.)
    // (128 rows: 133 KB of results go by at 4.5 TB/s in 30 ns, a key of 512 workgroups takes 40.  Few rows: the bytes of a result's twice over those of a key)
    if (c == kRows128) return {kManyRowsTile, 256, 512, 0.75};
    const uint32_t slots = l.cache_dtype == KVL_E4M3 && c == kRows16 ? 768 : 512;
    return {(c == kRows64 ? 2 : 4) * few_rows_tile(l.head_dim), 512, slots, 4.0 * kClassRows[c] / (element_bytes(l.cache_dtype) * slots)};
}
static uint64_t piece_of(const kvl_attn_layout_t &l, uint32_t c, const std::vector<Tile> &tiles) {
    const Machine m = machine_of(l, c);
    uint64_t longest = 0, keys = 0, n_tiles = 0;
    for (const Tile &t : tiles) {
        if (t.cls != c) continue;
        const uint64_t n = t.at.end - t.at.begin;
        longest = std::max(longest, n);
        keys += n;
        ++n_tiles;
    }
    const uint64_t whole = std::max<uint64_t>(1, (longest + m.step - 1) / m.step) * m.step;
    uint64_t best = whole;
    double least = 0;
    // (with tiles enough for many rounds only those that are long beside the others are worth a cut)
    const uint64_t from = n_tiles * l.kv_heads > 8ull * m.slots ? std::max<uint64_t>(m.step, keys / n_tiles / m.step * m.step) : m.step;
    for (uint64_t piece = whole; piece >= from; piece = piece > m.step ? std::max<uint64_t>(m.step, piece * 7 / 8 / m.step * m.step) : 0) {
        uint64_t count = 0, most = 0, cut = 0;
        for (const Tile &t : tiles) {
            if (t.cls != c) continue;
            const uint64_t n = t.at.end - t.at.begin, k = std::max<uint64_t>(1, (n + piece - 1) / piece);
            count += k;
            if (k > 1) cut += k;
            most = std::max(most, (n + k - 1) / k);
        }
        const double rounds = (double)(count * l.kv_heads) / m.slots, mean = (double)keys / (double)count + m.more;
        const double time = std::max((double)(most + m.more), rounds > 1 ? (rounds + 0.5) * mean : 0.0) +
                            (cut ? kJoinKeys + m.join * (double)(cut * l.kv_heads) : 0.0);
        if (piece == whole || time < least) {
            least = time;
            best = piece;
        }
    }
    return best;
}

// Requests of unlike numbers of rows, few each, go in one launch where their work is small beside a launch's own time (32 requests of 0.7-9 K
// tokens, 4 heads, rows of 21 to 42: 48 us in one launch, 57 in two).
static void merge_classes(const kvl_attn_layout_t &l, std::vector<Tile> &tiles) {
    uint64_t keys = 0;
    uint32_t most = 0;
    for (const Tile &t : tiles) {
        if (t.cls == kRows128) continue;
        keys += t.at.end - t.at.begin;
        most = std::max(most, t.cls);
    }
    if (keys * l.kv_heads > (1u << 21)) return;
    for (Tile &t : tiles)
        if (t.cls != kRows128) t.cls = most;
}

// Rows of an 8-bit block up to its last new token: the append numbers them times 8 in 32 bits, with room for a step beyond the end.
constexpr uint64_t kMostBlockRows = 1ull << 28;

static int check_attn_layout(const kvl_attn_layout_t *l) {
    if (l->block_tokens == 0 || l->kv_heads == 0 || l->q_heads == 0 || l->q_heads % l->kv_heads) return KVL_EINVAL;
    if (l->q_heads > 65536) return KVL_EINVAL;
    if (l->head_dim != 64 && l->head_dim != 128) return KVL_EINVAL;
    if (l->dtype != KVL_BF16 && l->dtype != KVL_F16) return KVL_EINVAL;
    if (l->cache_dtype != l->dtype && l->cache_dtype != KVL_E4M3) return KVL_EINVAL;
    if (l->rope_dim % 16 || l->rope_dim > l->head_dim || l->rope_pairs > KVL_ROPE_NEIGHBOURS) return KVL_EINVAL;
    if (l->pool_blocks > UINT32_MAX / l->block_tokens) return KVL_ERANGE;
    return KVL_OK;
}

static void put(std::vector<kvl_unit_t> &blob, uint64_t at, const void *from, size_t bytes) {
    if (bytes) std::memcpy(reinterpret_cast<char *>(blob.data()) + at, from, bytes);
}

static int build_attn(const kvl_attn_layout_t *layout, const kvl_request_t *req, uint32_t n_req, uint32_t flags,
                      kvl_attn_plan_t *plan) {
    const kvl_attn_layout_t &l = *layout;
    const uint64_t bs = l.block_tokens;
    const uint32_t group = l.q_heads / l.kv_heads;
    plan->layout = l;
    plan->flags = flags;
    // (neither KVL_GATHER nor KVL_SCATTER: the array is not one of copy descriptors)
    plan->base.flags = flags & (KVL_HOST_ONLY | KVL_NO_POINTER_CHECKS | KVL_CALLER_SYNCS);
    plan->base.layout.block_tokens = l.block_tokens;
    plan->base.layout.n_planes = 2;
    plan->base.layout.row_bytes[0] = plan->base.layout.row_bytes[1] = l.kv_heads * l.head_dim * element_bytes(l.cache_dtype);
    plan->base.layout.pool_blocks = l.pool_blocks;
    while ((1ull << plan->div_shift) < bs) ++plan->div_shift;
    // ((2^(31 + shift) + bs - 1) / bs is at least 2^31, and below 2^32 as bs is above 2^(shift - 1))
    plan->div_mul = (uint32_t)(((1ull << (31 + plan->div_shift)) + bs - 1) / bs);
    if (plan->div_shift == 32) plan->div_mul = plan->div_shift = 0;     // (a block holds every token: 0)

    std::vector<uint64_t> token0(n_req), table0(n_req);
    uint64_t tokens = 0, entries = 0;
    for (uint32_t r = 0; r < n_req; ++r) {
        const uint64_t n = req[r].append_tokens, all = req[r].hit_tokens + n, blocks = (all + bs - 1) / bs;
        if (all >= (1ull << 31) || n * group > UINT32_MAX) return KVL_ERANGE;
        if (req[r].n_blocks < blocks) return KVL_ERANGE;
        if (blocks && !req[r].block_table) return KVL_EINVAL;
        for (uint64_t b = 0; b < blocks; ++b)
            if (req[r].block_table[b] < 0 || (uint64_t)req[r].block_table[b] >= l.pool_blocks) return KVL_ERANGE;
        token0[r] = tokens;
        table0[r] = entries;
        tokens += n;
        entries += blocks;
        if (n) plan->last_position = std::max(plan->last_position, all - 1);
    }
    if (tokens * l.q_heads > UINT32_MAX * 64ull || tokens > UINT32_MAX || entries > UINT32_MAX) return KVL_ERANGE;
    plan->new_tokens = tokens;

    // attention: tiles of rows, then the pieces that their keys are cut into
    std::vector<AttnItem> items;
    std::vector<JoinItem> joins;
    uint64_t floats = 0;
    if (flags & KVL_GATHER) {
        std::vector<Tile> tiles;
        for (uint32_t r = 0; r < n_req; ++r) {
            const uint64_t hit = req[r].hit_tokens, n = req[r].append_tokens, rows = n * group;
            const uint64_t first = flags & KVL_TOKENS_APPEND ? hit : 0, last = flags & (KVL_TOKENS_APPEND | KVL_TOKENS_ALL) ? hit + n : hit;
            const uint32_t c = rows <= 16 ? kRows16 : rows <= 32 ? kRows32 : rows <= 64 ? kRows64 : kRows128;
            for (uint64_t r0 = 0; r0 < rows; r0 += kClassRows[c]) {
                const uint64_t r1 = std::min<uint64_t>(rows, r0 + kClassRows[c]);
                const Places at = places_of(l, first, last, hit + r0 / group, hit + (r1 - 1) / group);
                tiles.push_back({r, (uint32_t)r0, (uint32_t)(r1 - r0), c, at});
            }
        }
        merge_classes(l, tiles);
        for (uint32_t c = 0; c < kAttnClasses; ++c) {
            const uint64_t piece = piece_of(l, c, tiles), step = machine_of(l, c).step;
            const size_t from = items.size();
            for (const Tile &t : tiles) {
                if (t.cls != c) continue;
                const uint64_t n = t.at.end - t.at.begin, pieces = std::max<uint64_t>(1, (n + piece - 1) / piece);
                const uint64_t span = ((n + pieces - 1) / pieces + step - 1) / step * step;
                const uint64_t used = std::max<uint64_t>(1, span ? (n + span - 1) / span : 1);
                AttnItem it{(uint32_t)token0[t.request], req[t.request].hit_tokens, (uint32_t)table0[t.request], t.first_row, t.n_rows,
                            0, 0, t.at.sinks, t.at.gap, (uint32_t)used, floats};
                const uint64_t size = partial_floats(kClassRows[c], l.head_dim) * l.kv_heads;
                for (uint64_t i = 0; i < used; ++i) {
                    it.begin = (uint32_t)(t.at.begin + i * span);
                    it.end = (uint32_t)std::min<uint64_t>(t.at.end, it.begin + span);
                    it.partial = floats + i * size;
                    items.push_back(it);
                    plan->items.push_back({t.request, it.first_row, it.n_rows, it.begin, it.end, it.sinks, it.gap, it.pieces});
                }
                if (used > 1) {
                    joins.push_back({it.token0, it.first_row, it.n_rows, it.pieces, kClassRows[c], 0, floats});
                    plan->most_join_rows = std::max(plan->most_join_rows, it.n_rows);
                    plan->most_pieces = std::max(plan->most_pieces, it.pieces);
                    floats += used * size;
                }
            }
            // the longest first
            std::vector<uint32_t> order(items.size() - from);
            for (size_t i = 0; i < order.size(); ++i) order[i] = (uint32_t)(from + i);
            std::stable_sort(order.begin(), order.end(), [&](uint32_t a, uint32_t b) {
                return items[a].end - items[a].begin > items[b].end - items[b].begin;
            });
            std::vector<AttnItem> sorted;
            std::vector<kvl_attn_item_t> sorted_public;
            for (uint32_t i : order) {
                sorted.push_back(items[i]);
                sorted_public.push_back(plan->items[i]);
            }
            std::copy(sorted.begin(), sorted.end(), items.begin() + (long)from);
            std::copy(sorted_public.begin(), sorted_public.end(), plan->items.begin() + (long)from);
            if (items.size() * l.kv_heads >= (1u << 24)) return KVL_ERANGE;     // fewer than 2^32 lanes
            plan->class_first[c + 1] = (uint32_t)items.size();
        }
        plan->workspace_bytes = floats * sizeof(float);
        plan->n_join = (uint32_t)joins.size();
        if ((uint64_t)plan->n_join * l.kv_heads * plan->join_groups() >= (1u << 24)) return KVL_ERANGE;
    }

    // append: the new tokens' places, and the blocks that receive them
    std::vector<AppendBlock> blocks;
    std::vector<AppendToken> places;
    if (flags & KVL_SCATTER) {
        // (as in kvl_plan: an entry counts only with this plan's stamp)
        static thread_local std::vector<uint32_t> taken;
        static thread_local uint32_t stamp = 0;
        if (taken.size() < l.pool_blocks) taken.resize((size_t)l.pool_blocks, 0);
        if (++stamp == 0) {
            std::fill(taken.begin(), taken.end(), 0u);
            stamp = 1;
        }
        places.reserve(tokens);
        for (uint32_t r = 0; r < n_req; ++r) {
            const uint64_t hit = req[r].hit_tokens, all = hit + req[r].append_tokens;
            for (uint64_t t = hit; t < all;) {
                const uint64_t b = t / bs, upto = std::min(all, (b + 1) * bs);
                const uint32_t id = (uint32_t)req[r].block_table[b], n = (uint32_t)(upto - t);
                if (taken[id] == stamp) return KVL_EALIAS;
                taken[id] = stamp;
                if (l.cache_dtype == KVL_E4M3) {        // (16-bit rows go by their tokens' places alone)
                    if (upto - b * bs > kMostBlockRows) return KVL_ERANGE;
                    blocks.push_back({id, (uint32_t)(token0[r] + t - hit), (uint32_t)(t - b * bs), n, (uint32_t)t, {}});
                    plan->most_append_rows = std::max(plan->most_append_rows, n);
                }
                for (; t < upto; ++t) places.push_back({(uint32_t)t, (uint32_t)(id * bs + t - b * bs)});
            }
        }
        plan->n_append_blocks = (uint32_t)blocks.size();
        if (blocks.size() * l.kv_heads > (1u << 23)) return KVL_ERANGE;      // (fewer than 2^32 lanes, those of the queries with them)
    }

    std::vector<int32_t> tables;
    if (flags & KVL_GATHER) {
        tables.reserve(entries);
        for (uint32_t r = 0; r < n_req; ++r) {
            const uint64_t n = ((uint64_t)req[r].hit_tokens + req[r].append_tokens + bs - 1) / bs;
            tables.insert(tables.end(), req[r].block_table, req[r].block_table + n);
        }
    }
    uint64_t at = 0;
    auto room = [&at](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    plan->off_items = room(items.size() * sizeof(AttnItem));
    plan->off_join = room(joins.size() * sizeof(JoinItem));
    plan->off_tables = room(tables.size() * sizeof(int32_t));
    plan->off_blocks = room(blocks.size() * sizeof(AppendBlock));
    plan->off_tokens = room(places.size() * sizeof(AppendToken));
    if (flags & KVL_HOST_ONLY) return KVL_OK;
    plan->base.units.resize(at / 16);
    put(plan->base.units, plan->off_items, items.data(), items.size() * sizeof(AttnItem));
    put(plan->base.units, plan->off_join, joins.data(), joins.size() * sizeof(JoinItem));
    put(plan->base.units, plan->off_tables, tables.data(), tables.size() * sizeof(int32_t));
    put(plan->base.units, plan->off_blocks, blocks.data(), blocks.size() * sizeof(AppendBlock));
    put(plan->base.units, plan->off_tokens, places.data(), places.size() * sizeof(AppendToken));
    const int rc = upload_units(&plan->base);
    std::vector<kvl_unit_t>().swap(plan->base.units);       // (it is on the device now)
    return rc;
}

int check_attn_pool(const kvl_attn_plan_t *plan, const void *const *planes) {
    const int rc = check_device(&plan->base);
    if (rc != KVL_OK) return rc;
    const kvl_attn_layout_t &l = plan->layout;
    const uint32_t n = l.cache_dtype == KVL_E4M3 ? 4 : 2;
    for (uint32_t p = 0; p < n; ++p) {
        if (!planes[p] || reinterpret_cast<uintptr_t>(planes[p]) % (p < 2 ? 16 : 4)) return KVL_EINVAL;
        const uint64_t bytes = p < 2 ? l.pool_blocks * l.block_tokens * (uint64_t)plan->base.layout.row_bytes[p] : l.pool_blocks * l.kv_heads * 4ull;
        const int found = check_buffer(&plan->base, planes[p], bytes, false);
        if (found != KVL_OK) return found;
    }
    return KVL_OK;
}

int check_rows(const kvl_attn_plan_t *plan, const void *ptr, uint64_t n, uint64_t row, uint64_t *stride, bool half) {
    if (*stride == 0) *stride = row;
    if (!ptr || *stride < row) return KVL_EINVAL;
    if (half && (reinterpret_cast<uintptr_t>(ptr) % 16 || *stride % 8)) return KVL_EINVAL;
    if (*stride > std::min<uint64_t>(1ull << 40, (1ull << 60) / n)) return KVL_EINVAL;     // (the extent is computed in 64 bits)
    return check_buffer(&plan->base, ptr, ((n - 1) * *stride + row) * (half ? 2 : 4), false);
}

}  // namespace kvl

extern "C" {

int kvl_attn_plan(const kvl_attn_layout_t *layout, const kvl_request_t *requests, uint32_t n_req, uint32_t flags, kvl_attn_plan_t **out) {
    if (!layout || !out || (n_req && !requests)) return KVL_EINVAL;
    *out = nullptr;
    if (!(flags & (KVL_GATHER | KVL_SCATTER))) return KVL_EINVAL;
    if (flags & ~(KVL_GATHER | KVL_SCATTER | KVL_HOST_ONLY | KVL_TOKENS_APPEND | KVL_TOKENS_ALL | KVL_NO_POINTER_CHECKS | KVL_CALLER_SYNCS))
        return KVL_EINVAL;
    if ((flags & KVL_TOKENS_APPEND) && (flags & KVL_TOKENS_ALL)) return KVL_EINVAL;
    int rc = kvl::check_attn_layout(layout);
    if (rc != KVL_OK) return rc;
    kvl_attn_plan_t *plan = new (std::nothrow) kvl_attn_plan_t;
    if (!plan) return KVL_ENOMEM;
    try {
        rc = kvl::build_attn(layout, requests, n_req, flags, plan);
    } catch (const std::exception &) {                      // (bad_alloc, length_error)
        rc = KVL_ENOMEM;
    }
    if (rc != KVL_OK) {
        kvl_attn_plan_destroy(plan);
        return rc;
    }
    *out = plan;
    return KVL_OK;
}

void kvl_attn_plan_destroy(kvl_attn_plan_t *plan) {
    if (!plan) return;
    kvl::release_plan(&plan->base);
    delete plan;
}

int kvl_attn_plan_tokens(const kvl_attn_plan_t *plan, uint64_t *new_tokens) {
    if (!plan || !new_tokens) return KVL_EINVAL;
    *new_tokens = plan->new_tokens;
    return KVL_OK;
}

int kvl_attn_plan_workspace(const kvl_attn_plan_t *plan, uint64_t *bytes) {
    if (!plan || !bytes) return KVL_EINVAL;
    *bytes = plan->workspace_bytes;
    return KVL_OK;
}

int kvl_attn_plan_items(const kvl_attn_plan_t *plan, kvl_attn_item_t *out, uint64_t capacity, uint64_t *n_items) {
    if (!plan || !n_items || (capacity && !out)) return KVL_EINVAL;
    *n_items = plan->items.size();
    const uint64_t k = std::min<uint64_t>(capacity, plan->items.size());
    if (k) std::memcpy(out, plan->items.data(), k * sizeof(kvl_attn_item_t));
    return KVL_OK;
}

}  // extern "C"
