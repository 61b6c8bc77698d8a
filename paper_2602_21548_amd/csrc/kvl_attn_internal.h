// Declarations shared by the attention operators' translation units.
#pragma once

#include <hip/hip_ext.h>

#include "kvl_attn.h"
#include "kvl_internal.h"

namespace kvl {

// Which kernel takes a request's rows (new tokens times the query heads that share a cache head), and in tiles of how many.
enum AttnClass : uint32_t { kRows16 = 0, kRows32, kRows64, kRows128, kAttnClasses };
constexpr uint32_t kClassRows[kAttnClasses] = {16, 32, 64, 128};

// One piece of work of the attention kernels, for every cache head (kvl_attn_item_t, with what a kernel would have to look up).
struct AttnItem {
    uint32_t token0;        // the request's first new token
    uint32_t hit;           // its position
    uint32_t table;         // the request's first entry in the block tables
    uint32_t first_row;
    uint32_t n_rows;
    uint32_t begin, end;    // places of the visible keys
    uint32_t sinks, gap;    // place v is token v < sinks ? v : v + gap
    uint32_t pieces;        // 1: the item writes the outputs itself
    uint64_t partial;       // else: its first float in the workspace, for head 0
};
static_assert(sizeof(AttnItem) == 48, "three descriptor units");

// What a new token's queries see of their request: tokens [lo, hi), and those before `first` and `hi`.  Within a request lo and hi grow with the token,
// and `first` is the same.
struct AttnBounds {
    uint32_t lo, hi, first;
    uint32_t reserved;
};
static_assert(sizeof(AttnBounds) == 16, "a descriptor unit");

// Rows whose keys were cut into pieces, for every cache head.
struct JoinItem {
    uint32_t token0;
    uint32_t first_row;
    uint32_t n_rows;
    uint32_t pieces;
    uint32_t tile_rows;     // rows of a partial result
    uint32_t reserved;
    uint64_t partial;       // of piece 0 and head 0
};
static_assert(sizeof(JoinItem) == 32, "two descriptor units");

// A block that receives new tokens: rows [row, row + n), from new token `token` on; rows before them hold hit tokens.
struct AppendBlock {
    uint32_t block;
    uint32_t token;
    uint32_t row;
    uint32_t n;
    uint32_t position;      // of `token`
    uint32_t reserved[3];
};
static_assert(sizeof(AppendBlock) == 32, "two descriptor units");

struct AppendToken {
    uint32_t position;
    uint32_t pool_row;
};

// Floats of a partial result of a tile: unnormalised outputs, then each row's maximum and sum.
inline uint64_t partial_floats(uint32_t tile_rows, uint32_t head_dim) { return (uint64_t)tile_rows * (head_dim + 2); }

// Keys of a tile of one wavefront in the kernel for few rows: 8 KB of K, 4 KB of 8-bit ones.
constexpr uint32_t few_rows_tile(uint32_t head_dim) { return head_dim == 64 ? 64 : 32; }
constexpr uint32_t kManyRowsTile = 64;

}  // namespace kvl

struct kvl_attn_plan_s {
    // Holds the device array (the lists below, end to end) and follows its launches, as a copy plan's descriptors are.
    kvl_plan_s base;
    kvl_attn_layout_t layout{};
    uint32_t flags = 0;
    uint64_t new_tokens = 0, last_position = 0;
    uint64_t workspace_bytes = 0;
    std::vector<kvl_attn_item_t> items;                 // as the public call gives them
    uint32_t class_first[kvl::kAttnClasses + 1] = {};   // items of each class
    uint32_t n_join = 0, most_join_rows = 0, most_pieces = 0, n_append_blocks = 0, most_append_rows = 0;
    uint64_t off_items = 0, off_join = 0, off_tables = 0, off_blocks = 0, off_tokens = 0;    // bytes into the device array
    bool masked = false;                                // it has what each new token sees (kvl_attn_plan_masked):
    uint64_t off_bounds = 0;                            // AttnBounds, there
    uint32_t div_mul = 0, div_shift = 0;                // t / block_tokens == 2 t * div_mul >> 32 + div_shift for t < 2^31

    // the join's wavefronts for each row, and its workgroups for each tile of rows and head
    uint32_t join_waves() const { return most_pieces > 8 ? 4 : 1; }
    uint32_t join_groups() const { return join_waves() == 4 ? most_join_rows : (most_join_rows + 3) / 4; }
};

namespace kvl {

inline uint32_t element_bytes(uint32_t dtype) { return dtype == KVL_E4M3 ? 1u : 2u; }

// Checks that a plan may run here and that its pool's planes are what the layout says.
int check_attn_pool(const kvl_attn_plan_t *plan, const void *const *planes);
// n rows of `row` elements of `dtype`, `stride` elements apart: alignment and extent.
int check_rows(const kvl_attn_plan_t *plan, const void *ptr, uint64_t n, uint64_t row, uint64_t *stride, bool half);

// A run of launches on one stream, the last of which carries the plan's event.
struct AttnLaunch {
    hipStream_t stream;
    DefaultStreamEvent *passes = nullptr;
    hipEvent_t done;
    bool ok = false;
    AttnLaunch(const kvl_attn_plan_t *plan, hipStream_t s) : stream(s), done(launch_event(&plan->base, s, &passes)) {}
    ~AttnLaunch() {
        if (passes) launched(passes, ok);
    }
    AttnLaunch(const AttnLaunch &) = delete;
    AttnLaunch &operator=(const AttnLaunch &) = delete;
    template <typename... P, typename... A>
    void operator()(bool last, void (*kernel)(P...), uint32_t groups, uint32_t threads, A... args) {
        if (last && done) hipExtLaunchKernelGGL(kernel, dim3(groups), dim3(threads), 0, stream, nullptr, done, 0, args...);
        else hipLaunchKernelGGL(kernel, dim3(groups), dim3(threads), 0, stream, args...);
    }
    int made() {
        KVL_HIP(hipGetLastError());
        ok = true;
        return KVL_OK;
    }
};

}  // namespace kvl
