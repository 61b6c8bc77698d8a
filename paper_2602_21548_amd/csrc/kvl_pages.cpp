// Whose the blocks of a paged cache are (host only).
#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "kvl_pages.h"

namespace kvl {
namespace {

// The free blocks, as bits; a word of a level says which words of the level below have any, so that the lowest is found in a step a level.
class FreeBlocks {
public:
    explicit FreeBlocks(uint64_t n) : free_(n) {
        do {
            const uint64_t words = (n + 63) / 64;
            levels_.emplace_back(words, ~0ull);
            if (n % 64) levels_.back().back() = (1ull << n % 64) - 1;
            n = words;
        } while (n > 1);
    }
    uint64_t count() const { return free_; }
    bool has(uint32_t b) const { return levels_[0][b / 64] >> b % 64 & 1; }
    uint32_t lowest() const {                   // (there is one)
        uint64_t at = 0;
        for (size_t l = levels_.size(); l-- > 0;) at = at * 64 + (uint64_t)__builtin_ctzll(levels_[l][at]);
        return (uint32_t)at;
    }
    void take(uint32_t b) {
        --free_;
        uint64_t at = b;
        for (auto &level : levels_) {
            level[at / 64] &= ~(1ull << at % 64);
            if (level[at / 64]) break;
            at /= 64;
        }
    }
    void give(uint32_t b) {
        ++free_;
        uint64_t at = b;
        for (auto &level : levels_) {
            const bool empty = level[at / 64] == 0;
            level[at / 64] |= 1ull << at % 64;
            if (!empty) break;
            at /= 64;
        }
    }

private:
    uint64_t free_;
    std::vector<std::vector<uint64_t>> levels_;
};

struct Sequence {
    std::vector<int32_t> table;
    uint32_t tokens = 0;
    uint32_t generation = 0;
    uint32_t stamp = 0;                         // of the list that named it last
    bool there = false;
};

constexpr uint64_t kMostTokens = 1ull << 31;

}  // namespace
}  // namespace kvl

struct kvl_pages_s {
    uint32_t block_tokens;
    uint64_t pool_blocks;
    kvl::FreeBlocks free;
    std::vector<uint32_t> users;                // of each block
    std::vector<kvl::Sequence> sequences;       // by the number's lower half
    std::vector<uint32_t> slots;                // of those that have ended, with room for all
    uint32_t stamp = 0;
    std::vector<uint32_t> named;                // of each block, once a table was adopted: by which one last
    uint32_t naming = 0;

    kvl_pages_s(uint32_t bs, uint64_t n) : block_tokens(bs), pool_blocks(n), free(n), users(n, 0) {}

    uint64_t blocks_of(uint64_t tokens) const { return (tokens + block_tokens - 1) / block_tokens; }
    kvl::Sequence *find(uint64_t number) {
        const uint64_t slot = number & UINT32_MAX;
        if (slot == 0 || slot > sequences.size()) return nullptr;
        kvl::Sequence &s = sequences[slot - 1];
        return s.there && s.generation == number >> 32 ? &s : nullptr;
    }
    const kvl::Sequence *find(uint64_t number) const { return const_cast<kvl_pages_s *>(this)->find(number); }
    // Whether all are there, and none twice.
    bool each_once(const uint64_t *numbers, uint32_t n) {
        if (++stamp == 0) {
            for (kvl::Sequence &s : sequences) s.stamp = 0;
            stamp = 1;
        }
        for (uint32_t i = 0; i < n; ++i) {
            kvl::Sequence *s = find(numbers[i]);
            if (!s || s->stamp == stamp) return false;
            s->stamp = stamp;
        }
        return true;
    }
    // Whether these are blocks of the pool (KVL_ERANGE), and none is there twice (KVL_EALIAS).
    int check_table(const int32_t *table, uint64_t n) {
        if (n && named.empty()) named.resize(pool_blocks, 0);
        if (++naming == 0) {
            std::fill(named.begin(), named.end(), 0u);
            naming = 1;
        }
        for (uint64_t i = 0; i < n; ++i) {
            if (table[i] < 0 || (uint64_t)table[i] >= pool_blocks) return KVL_ERANGE;
            if (named[(size_t)table[i]] == naming) return KVL_EALIAS;
            named[(size_t)table[i]] = naming;
        }
        return KVL_OK;
    }
    // Room for n new sequences: nothing is allocated by their making, or by their end.
    void make_room(uint32_t n) {
        const size_t want = sequences.size() + (n > slots.size() ? n - slots.size() : 0);
        if (want > sequences.capacity()) sequences.reserve(std::max(want, 2 * sequences.capacity()));
        if (slots.capacity() < sequences.capacity()) slots.reserve(sequences.capacity());
    }
    uint64_t add(std::vector<int32_t> &&table, uint32_t tokens) {
        uint32_t slot;
        if (slots.empty()) {
            slot = (uint32_t)sequences.size();
            sequences.emplace_back();
        } else {
            slot = slots.back();
            slots.pop_back();
        }
        kvl::Sequence &s = sequences[slot];
        s.table = std::move(table);
        s.tokens = tokens;
        s.there = true;
        for (int32_t b : s.table) use((uint32_t)b);
        return (uint64_t)s.generation << 32 | (slot + 1);
    }
    void use(uint32_t b) {
        if (users[b]++ == 0) free.take(b);
    }
    void leave(uint32_t b) {
        if (--users[b] == 0) free.give(b);
    }
    void keep(kvl::Sequence &s, uint32_t tokens) {
        const size_t n = (size_t)blocks_of(tokens);
        while (s.table.size() > n) {
            leave((uint32_t)s.table.back());
            s.table.pop_back();
        }
        s.tokens = tokens;
    }
    // Blocks in use from `used` on, where that many are in use: each moves to a free one before.
    uint64_t moves() const {
        uint64_t n = 0;
        for (uint64_t b = pool_blocks - free.count(); b < pool_blocks; ++b) n += users[b] != 0;
        return n;
    }
};

namespace kvl {
namespace {

template <typename F>
int guarded(F &&f) {
    try {
        return f();
    } catch (const std::exception &) {          // (bad_alloc, length_error)
        return KVL_ENOMEM;
    }
}

int adopt(kvl_pages_t *pages, const kvl_request_t *req, uint32_t n, uint64_t *out) {
    std::vector<std::vector<int32_t>> tables(n);
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t tokens = (uint64_t)req[i].hit_tokens + req[i].append_tokens, blocks = pages->blocks_of(tokens);
        if (tokens >= kMostTokens || req[i].n_blocks < blocks) return KVL_ERANGE;
        if (blocks && !req[i].block_table) return KVL_EINVAL;
        const int rc = pages->check_table(req[i].block_table, blocks);
        if (rc != KVL_OK) return rc;
        if (blocks) tables[i].assign(req[i].block_table, req[i].block_table + blocks);
    }
    pages->make_room(n);
    for (uint32_t i = 0; i < n; ++i) out[i] = pages->add(std::move(tables[i]), req[i].hit_tokens + req[i].append_tokens);
    return KVL_OK;
}

int fork(kvl_pages_t *pages, const uint64_t *from, uint32_t n, uint64_t *out) {
    std::vector<std::vector<int32_t>> tables(n);
    std::vector<uint32_t> tokens(n);
    for (uint32_t i = 0; i < n; ++i) {
        const Sequence *s = pages->find(from[i]);
        if (!s) return KVL_EINVAL;
        tables[i] = s->table;
        tokens[i] = s->tokens;
    }
    pages->make_room(n);
    for (uint32_t i = 0; i < n; ++i) out[i] = pages->add(std::move(tables[i]), tokens[i]);
    return KVL_OK;
}

int extend(kvl_pages_t *pages, const uint64_t *numbers, const uint32_t *tokens, uint32_t n, kvl_block_copy_t *copies, uint32_t *n_copies) {
    if (!pages->each_once(numbers, n)) return KVL_EINVAL;
    // what it takes: a shared last block is left by all of its users but the last one, if they are all here
    const uint32_t bs = pages->block_tokens;
    auto writes_shared = [&](const Sequence &s, uint32_t more) { return more && s.tokens % bs && pages->users[(size_t)s.table.back()] > 1; };
    uint64_t need = 0;
    uint32_t done = 0;
    int rc = KVL_OK;
    for (; done < n; ++done) {
        Sequence &s = *pages->find(numbers[done]);
        const uint64_t all = (uint64_t)s.tokens + tokens[done], blocks = pages->blocks_of(all);
        if (all >= kMostTokens) {
            rc = KVL_ERANGE;
            break;
        }
        need += blocks - s.table.size();
        if (need > pages->free.count()) {       // (before tables get room for blocks that are not there)
            rc = KVL_ESPACE;
            break;
        }
        if (blocks > s.table.capacity()) s.table.reserve(std::max<size_t>((size_t)blocks, 2 * s.table.capacity()));
    }
    if (rc != KVL_OK) return rc;
    uint64_t own = 0;
    std::vector<uint32_t> left;                 // blocks whose count of users was lowered to see who is the last one
    left.reserve(n);
    for (uint32_t i = 0; i < n; ++i) {
        const Sequence &s = *pages->find(numbers[i]);
        if (!writes_shared(s, tokens[i])) continue;
        const uint32_t b = (uint32_t)s.table.back();
        --pages->users[b];
        left.push_back(b);
        ++own;
    }
    for (uint32_t b : left) ++pages->users[b];
    if (need + own > pages->free.count()) return KVL_ESPACE;
    uint32_t made = 0;
    for (uint32_t i = 0; i < n; ++i) {
        Sequence &s = *pages->find(numbers[i]);
        if (writes_shared(s, tokens[i])) {
            const uint32_t b = pages->free.lowest();
            pages->use(b);
            copies[made++] = {s.table.back(), (int32_t)b};
            pages->leave((uint32_t)s.table.back());
            s.table.back() = (int32_t)b;
        }
        s.tokens += tokens[i];
        for (size_t blocks = (size_t)pages->blocks_of(s.tokens); s.table.size() < blocks;) {
            const uint32_t b = pages->free.lowest();
            pages->use(b);
            s.table.push_back((int32_t)b);
        }
    }
    *n_copies = made;
    return KVL_OK;
}

int compact(kvl_pages_t *pages, uint32_t most, kvl_block_copy_t *copies, uint32_t *n_copies) {
    const uint64_t used = pages->pool_blocks - pages->free.count();
    std::vector<int32_t> to(pages->pool_blocks - used, -1);       // of blocks from `used` on
    uint32_t n = 0;
    for (uint64_t b = pages->pool_blocks; b-- > used && n < most;) {
        if (!pages->users[b]) continue;
        const uint32_t at = pages->free.lowest();           // (below `used`: fewer than `used` blocks are in use there as long as one is here)
        pages->free.take(at);
        pages->free.give((uint32_t)b);
        pages->users[at] = pages->users[b];
        pages->users[b] = 0;
        to[b - used] = (int32_t)at;
        copies[n++] = {(int32_t)b, (int32_t)at};
    }
    if (n)
        for (Sequence &s : pages->sequences)
            for (int32_t &b : s.table)
                if ((uint64_t)b >= used && to[(uint64_t)b - used] >= 0) b = to[(uint64_t)b - used];
    *n_copies = n;
    return KVL_OK;
}

}  // namespace
}  // namespace kvl

extern "C" {

int kvl_pages(uint32_t block_tokens, uint64_t pool_blocks, kvl_pages_t **out) {
    if (!out) return KVL_EINVAL;
    *out = nullptr;
    if (block_tokens == 0 || pool_blocks == 0) return KVL_EINVAL;
    if (pool_blocks > INT32_MAX) return KVL_ERANGE;
    return kvl::guarded([&] {
        *out = new kvl_pages_t(block_tokens, pool_blocks);
        return KVL_OK;
    });
}

void kvl_pages_destroy(kvl_pages_t *pages) { delete pages; }

int kvl_pages_adopt(kvl_pages_t *pages, const kvl_request_t *requests, uint32_t n_req, uint64_t *sequences) {
    if (!pages || (n_req && (!requests || !sequences))) return KVL_EINVAL;
    return kvl::guarded([&] { return kvl::adopt(pages, requests, n_req, sequences); });
}

int kvl_pages_fork(kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, uint64_t *forks) {
    if (!pages || (n && (!sequences || !forks))) return KVL_EINVAL;
    return kvl::guarded([&] { return kvl::fork(pages, sequences, n, forks); });
}

int kvl_pages_extend(kvl_pages_t *pages, const uint64_t *sequences, const uint32_t *tokens, uint32_t n, kvl_block_copy_t *copies,
                     uint32_t *n_copies) {
    if (!pages || !n_copies || (n && (!sequences || !tokens || !copies))) return KVL_EINVAL;
    *n_copies = 0;
    return kvl::guarded([&] { return kvl::extend(pages, sequences, tokens, n, copies, n_copies); });
}

int kvl_pages_truncate(kvl_pages_t *pages, const uint64_t *sequences, const uint32_t *tokens, uint32_t n) {
    if (!pages || (n && (!sequences || !tokens)) || !pages->each_once(sequences, n)) return KVL_EINVAL;
    for (uint32_t i = 0; i < n; ++i)
        if (tokens[i] > pages->find(sequences[i])->tokens) return KVL_ERANGE;
    for (uint32_t i = 0; i < n; ++i) pages->keep(*pages->find(sequences[i]), tokens[i]);
    return KVL_OK;
}

int kvl_pages_free(kvl_pages_t *pages, const uint64_t *sequences, uint32_t n) {
    if (!pages || (n && !sequences) || !pages->each_once(sequences, n)) return KVL_EINVAL;
    for (uint32_t i = 0; i < n; ++i) {
        kvl::Sequence &s = *pages->find(sequences[i]);
        pages->keep(s, 0);
        std::vector<int32_t>().swap(s.table);
        s.there = false;
        if (++s.generation != 0) pages->slots.push_back((uint32_t)(&s - pages->sequences.data()));     // (a slot whose numbers have all been used is left)
    }
    return KVL_OK;
}

int kvl_pages_compact(kvl_pages_t *pages, uint32_t most, kvl_block_copy_t *copies, uint32_t *n_copies) {
    if (!pages || !n_copies || (most && !copies)) return KVL_EINVAL;
    *n_copies = 0;
    return kvl::guarded([&] { return kvl::compact(pages, most, copies, n_copies); });
}

int kvl_pages_tables(const kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, int32_t *table, uint64_t capacity, uint64_t *first) {
    if (!pages || !first || (n && !sequences) || (capacity && !table)) return KVL_EINVAL;
    for (uint32_t i = 0; i < n; ++i)
        if (!pages->find(sequences[i])) return KVL_EINVAL;
    first[0] = 0;
    for (uint32_t i = 0; i < n; ++i) first[i + 1] = first[i] + pages->find(sequences[i])->table.size();
    if (first[n] > capacity) return KVL_ESPACE;
    for (uint32_t i = 0; i < n; ++i) {
        const std::vector<int32_t> &t = pages->find(sequences[i])->table;
        if (!t.empty()) std::memcpy(table + first[i], t.data(), t.size() * sizeof(int32_t));
    }
    return KVL_OK;
}

int kvl_pages_tokens(const kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, uint32_t *tokens) {
    if (!pages || (n && (!sequences || !tokens))) return KVL_EINVAL;
    for (uint32_t i = 0; i < n; ++i)
        if (!pages->find(sequences[i])) return KVL_EINVAL;
    for (uint32_t i = 0; i < n; ++i) tokens[i] = pages->find(sequences[i])->tokens;
    return KVL_OK;
}

int kvl_pages_stats(const kvl_pages_t *pages, kvl_pages_stats_t *out) {
    if (!pages || !out) return KVL_EINVAL;
    kvl_pages_stats_t s{};
    s.free_blocks = pages->free.count();
    s.used_blocks = pages->pool_blocks - s.free_blocks;
    for (uint32_t u : pages->users) s.shared_blocks += u > 1;
    s.moves = pages->moves();
    for (const kvl::Sequence &q : pages->sequences) s.sequences += q.there;
    *out = s;
    return KVL_OK;
}

}  // extern "C"
