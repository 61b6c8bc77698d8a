// Copies of blocks of a paged cache, all layers and planes of them in one launch.
#include <hip/hip_ext.h>

#include <algorithm>
#include <cstring>
#include <new>
#include <type_traits>

#include "kvl_internal.h"
#include "kvl_pages.h"
#include "kvl_vectors.h"

struct kvl_page_pools_s {
    kvl_plan_s base;                                // holds the device array of the planes' addresses, and follows its launches
    kvl_page_layout_t layout{};
    uint32_t width_log2[KVL_MAX_PLANES] = {};       // bytes that blocks of all layers begin at multiples of: 16, 4 or 1
};

namespace kvl {

constexpr uint32_t kCopyThreads = 256;
// Copies that one launch takes: they are among its arguments, of which there may be 4 KB.
constexpr uint32_t kFewCopies = 24, kMostCopies = 320;

// Copies of one block that follow each other in the list share a workgroup, so many at most, which reads the block once: eight ways on from 32 blocks of
// 128 KB, us, apart / together: 16 layers 146 / 121, 4 layers 40 / 22, one (34 MB written) 10.9 / 7.1; but 4 MB written 2.7 / 3.3.
constexpr uint32_t kShare = 8;
constexpr uint64_t kShareBytes = 16u << 20;
// Up to this many bytes the stores are sc1 ones, which the on-die cache takes, beyond it sc1+nt ones (as a move's).  us, sc1 / sc1+nt, 64 KB blocks of 16 layers: 67 MB
// 20 / 22, 134 MB 39.5 / 45.6, 255 MB 73 / 84, 319 MB 95.5 / 103.5, 401 MB 132 / 133, 512 MB 172 / 168, 1006 MB 337 / 328; eight ways on from each block 134 MB 20.7 / 25.7, 255 MB
// 40 / 53, 401 MB 78 / 86.5, 512 MB 110.5 / 113.6, 671 MB 150 / 150: level at 400 MB, or 670; the limit is the size of that cache.
constexpr uint64_t kCachedCopyBytes = 256u << 20;

struct CopyPlane {
    uint32_t tiles_end;         // tiles of the planes up to this one
    uint32_t width_log2;
    uint64_t block_bytes;
};
template <uint32_t N>
struct BlockCopies {
    const uint64_t *planes;     // addresses, [layers][n_planes]
    uint32_t n_planes;
    CopyPlane plane[KVL_MAX_PLANES];
    kvl_block_copy_t copies[N];
    uint32_t runs[N];           // of copies of one block that share workgroups: the first one, and 2^16 times their number
};
static_assert(sizeof(BlockCopies<kMostCopies>) <= 4096, "arguments of a launch");

// A workgroup copies a tile of a block, one vector a lane: grid (tiles of a block's planes, blocks, layers).  The memory bounds it: a pool's
// compaction, 545 MB to other places, at 6.6 TB/s.
template <uint32_t N, int STORE, bool SHARED>
__global__ void __launch_bounds__(kCopyThreads) kvl_copy_blocks_kernel(const BlockCopies<N> a) {
    uint32_t tile = blockIdx.x, p = 0, before = 0;
#pragma unroll
    for (uint32_t i = 0; i + 1 < KVL_MAX_PLANES; ++i) {         // (planes that are not there end where the last one does)
        const bool beyond = tile >= a.plane[i].tiles_end;
        p += beyond;
        before = beyond ? a.plane[i].tiles_end : before;
    }
    tile -= before;
    const uint64_t base = a.planes[blockIdx.z * a.n_planes + p], bytes = a.plane[p].block_bytes;
    const uint32_t run = SHARED ? a.runs[blockIdx.y] : 1u << 16 | blockIdx.y, first = run & 0xffffu, end = first + (run >> 16);
    const uint64_t from = base + (uint64_t)(uint32_t)a.copies[first].from * bytes;
    const uint64_t at = ((uint64_t)tile * kCopyThreads + threadIdx.x) << a.plane[p].width_log2;
    if (at >= bytes) return;
    auto each = [&](auto &&put) {
        if (!SHARED) put(base + (uint64_t)(uint32_t)a.copies[first].to * bytes + at);
        else for (uint32_t i = first; i < end; ++i) put(base + (uint64_t)(uint32_t)a.copies[i].to * bytes + at);
    };
    if (a.plane[p].width_log2 == 4) {
        const v4u x = load16<true>((gsrc_t)(from + at));
        each([&](uint64_t to) { store16<STORE>((gdst_t)to, x); });
    } else if (a.plane[p].width_log2 == 2) {
        const uint32_t x = *reinterpret_cast<const uint32_t *>(from + at);
        each([&](uint64_t to) { *reinterpret_cast<uint32_t *>(to) = x; });
    } else {
        const uint8_t x = *reinterpret_cast<const uint8_t *>(from + at);
        each([&](uint64_t to) { *reinterpret_cast<uint8_t *>(to) = x; });
    }
}

static int make_pools(const kvl_page_layout_t *l, void *const *planes, uint32_t flags, kvl_page_pools_t *pools) {
    pools->layout = *l;
    pools->base.flags = flags;
    pools->base.device = -1;
    int device = -1;
    KVL_HIP(hipGetDevice(&device));
    pools->base.device = device;
    const uint32_t n = l->n_layers * l->n_planes;
    for (uint32_t p = 0; p < l->n_planes; ++p) {
        uint64_t all = l->block_bytes[p];
        for (uint32_t i = p; i < n; i += l->n_planes) all |= reinterpret_cast<uintptr_t>(planes[i]);
        pools->width_log2[p] = all % 16 == 0 ? 4 : all % 4 == 0 ? 2 : 0;
    }
    for (uint32_t i = 0; i < n; ++i) {
        if (!planes[i]) return KVL_EINVAL;
        const int rc = check_buffer(&pools->base, planes[i], l->pool_blocks * l->block_bytes[i % l->n_planes], false);
        if (rc != KVL_OK) return rc;
    }
    pools->base.units.resize(((size_t)n * 8 + 15) / 16);
    std::memcpy(pools->base.units.data(), planes, (size_t)n * 8);
    const int rc = upload_units(&pools->base);
    std::vector<kvl_unit_t>().swap(pools->base.units);
    return rc;
}

// No block is the destination of two copies, or of one and the source of one.
static int check_copies(uint64_t pool_blocks, const kvl_block_copy_t *copies, uint64_t n) {
    // (as in kvl_plan: an entry counts only with this call's stamp)
    static thread_local std::vector<uint32_t> taken;
    static thread_local uint32_t stamp = 0;
    if (taken.size() < pool_blocks) taken.resize((size_t)pool_blocks, 0);
    if (++stamp == 0) {
        std::fill(taken.begin(), taken.end(), 0u);
        stamp = 1;
    }
    for (uint64_t i = 0; i < n; ++i) {
        const kvl_block_copy_t c = copies[i];
        if (c.from < 0 || c.to < 0 || (uint64_t)c.from >= pool_blocks || (uint64_t)c.to >= pool_blocks) return KVL_ERANGE;
        if (taken[(size_t)c.to] == stamp) return KVL_EALIAS;
        taken[(size_t)c.to] = stamp;
    }
    for (uint64_t i = 0; i < n; ++i)
        if (taken[(size_t)copies[i].from] == stamp) return KVL_EALIAS;
    return KVL_OK;
}

template <uint32_t N, int STORE, bool SHARED>
static void launch_copies(const kvl_page_pools_t *pools, const kvl_block_copy_t *copies, uint32_t n, hipEvent_t done, hipStream_t stream) {
    const kvl_page_layout_t &l = pools->layout;
    BlockCopies<N> a;
    a.planes = reinterpret_cast<const uint64_t *>(pools->base.d_units);
    a.n_planes = l.n_planes;
    uint32_t tiles = 0;
    for (uint32_t p = 0; p < KVL_MAX_PLANES; ++p) {
        const uint64_t bytes = p < l.n_planes ? l.block_bytes[p] : 0, tile = (uint64_t)kCopyThreads << pools->width_log2[p];
        tiles += (uint32_t)((bytes + tile - 1) / tile);
        a.plane[p] = {tiles, pools->width_log2[p], bytes};
    }
    std::copy(copies, copies + n, a.copies);
    std::fill(a.copies + n, a.copies + N, kvl_block_copy_t{0, 0});
    uint32_t runs = 0;
    for (uint32_t i = 0; i < n; ++i) {
        if (SHARED && i && copies[i].from == copies[i - 1].from && a.runs[runs - 1] >> 16 < kShare) a.runs[runs - 1] += 1u << 16;
        else a.runs[runs++] = 1u << 16 | i;
    }
    std::fill(a.runs + runs, a.runs + N, 0u);
    const dim3 grid(tiles, runs, l.n_layers);
    constexpr auto kernel = kvl_copy_blocks_kernel<N, STORE, SHARED>;
    if (done) hipExtLaunchKernelGGL(kernel, grid, dim3(kCopyThreads), 0, stream, nullptr, done, 0, a);
    else hipLaunchKernelGGL(kernel, grid, dim3(kCopyThreads), 0, stream, a);
}

static int copy_blocks(const kvl_page_pools_t *pools, const kvl_block_copy_t *copies, uint64_t n, hipStream_t stream) {
    int rc = check_device(&pools->base);
    if (rc != KVL_OK || n == 0) return rc;
    const kvl_page_layout_t &l = pools->layout;
    if ((rc = check_copies(l.pool_blocks, copies, n)) != KVL_OK) return rc;
    // (of one copy: lanes of a launch in every direction together)
    uint64_t lanes = 0, bytes = 0;
    for (uint32_t p = 0; p < l.n_planes; ++p) {
        lanes += ((l.block_bytes[p] >> pools->width_log2[p]) + kCopyThreads) * l.n_layers;
        bytes += l.block_bytes[p] * l.n_layers;
    }
    if (lanes >> 32) return KVL_ERANGE;
    const uint64_t most = std::min<uint64_t>(kMostCopies, UINT32_MAX / lanes);
    bool shared = false;
    if (bytes > kShareBytes / n)
        for (uint64_t i = 1; i < n && !shared; ++i) shared = copies[i].from == copies[i - 1].from;
    const bool cached = bytes <= kCachedCopyBytes / n;
    DefaultStreamEvent *passes = nullptr;
    const hipEvent_t done = launch_event(&pools->base, stream, &passes);
    for (uint64_t at = 0; at < n; at += most) {
        const uint32_t some = (uint32_t)std::min(most, n - at);
        const hipEvent_t event = at + some == n ? done : nullptr;
        auto go = [&](auto most_here, auto store, auto together) {
            launch_copies<decltype(most_here)::value, decltype(store)::value, decltype(together)::value>(pools, copies + at, some, event, stream);
        };
        typedef std::integral_constant<uint32_t, kMostCopies> Most;
        typedef std::integral_constant<int, 2> Cached;
        typedef std::integral_constant<int, 3> Past;
        if (some <= kFewCopies && cached && !shared) go(std::integral_constant<uint32_t, kFewCopies>{}, Cached{}, std::false_type{});
        else if (cached && shared) go(Most{}, Cached{}, std::true_type{});
        else if (cached) go(Most{}, Cached{}, std::false_type{});
        else if (shared) go(Most{}, Past{}, std::true_type{});
        else go(Most{}, Past{}, std::false_type{});
    }
    const hipError_t e = hipGetLastError();
    if (passes) launched(passes, e == hipSuccess);
    if (e != hipSuccess) {
        set_hip_error(e);
        return KVL_EHIP;
    }
    return KVL_OK;
}

}  // namespace kvl

extern "C" {

int kvl_page_pools(const kvl_page_layout_t *layout, void *const *planes, uint32_t flags, kvl_page_pools_t **out) {
    if (!layout || !planes || !out) return KVL_EINVAL;
    *out = nullptr;
    if (flags & ~(KVL_NO_POINTER_CHECKS | KVL_CALLER_SYNCS)) return KVL_EINVAL;
    if (layout->n_layers == 0 || layout->n_layers > 4096 || layout->n_planes == 0 || layout->n_planes > KVL_MAX_PLANES) return KVL_EINVAL;
    if (layout->pool_blocks == 0) return KVL_EINVAL;
    if (layout->pool_blocks > INT32_MAX) return KVL_ERANGE;
    for (uint32_t p = 0; p < layout->n_planes; ++p) {
        if (layout->block_bytes[p] == 0) return KVL_EINVAL;
        if (layout->block_bytes[p] > (1ull << 32)) return KVL_ERANGE;
    }
    kvl_page_pools_t *pools = new (std::nothrow) kvl_page_pools_t;
    if (!pools) return KVL_ENOMEM;
    int rc;
    try {
        rc = kvl::make_pools(layout, planes, flags, pools);
    } catch (const std::exception &) {
        rc = KVL_ENOMEM;
    }
    if (rc != KVL_OK) {
        kvl_page_pools_destroy(pools);
        return rc;
    }
    *out = pools;
    return KVL_OK;
}

void kvl_page_pools_destroy(kvl_page_pools_t *pools) {
    if (!pools) return;
    kvl::release_plan(&pools->base);
    delete pools;
}

int kvl_copy_blocks(const kvl_page_pools_t *pools, const kvl_block_copy_t *copies, uint64_t n, void *stream) {
    if (!pools || (n && !copies)) return KVL_EINVAL;
    try {
        return kvl::copy_blocks(pools, copies, n, static_cast<hipStream_t>(stream));
    } catch (const std::exception &) {
        return KVL_ENOMEM;
    }
}

}  // extern "C"
