// New keys and values into a paged cache, rotated by their positions: kernels and entry point.
//
// Pairs (a, b) of a head's leading rope_dim elements become (a cos - b sin, b cos + a sin).  A lane takes two pieces of 8 elements of a
// head: those at j and j + rope_dim/2, whose elements are pairs (halves), else two that are half of what there is apart, so that neighbouring
// lanes' pieces are neighbours in memory in each load and store.  The cosines and sines are a row of the table, which the heads of a token
// share in the caches.  Memory bounds both kernels: each element is read once and written once.  9131 tokens of 16 + 2 * 4 heads of 128, 16-bit cache:
// 115 MB in 21.5 us, 5.3 TB/s; 40800 of 32 + 2 * 8, 8-bit cache: 940 MB in 195 us, 4.8 TB/s, of which the queries take 110.
#include "kvl_attn_internal.h"
#include "kvl_attn_types.h"

namespace kvl {

struct AppendArgs {
    const AppendToken *tokens;
    const AppendBlock *blocks;
    const char *k, *v, *q;
    char *q_out, *pool_k, *pool_v;
    float *scale_k, *scale_v;
    const float *rope;
    uint64_t k_stride, v_stride, q_stride, q_out_stride;    // elements
    uint64_t tasks;             // of this launch
    uint32_t per_token;         // tasks of a token
    uint32_t token_first;       // of this launch
    uint32_t q_tasks, kv_tasks; // of a token's queries, and of its keys (or values)
    uint32_t rope_dim, rope_pairs;
    uint32_t kv_heads, block_tokens, n_blocks;
};

// A lane's two pieces of 8 elements of a head: where they begin, and which of them the rotation takes (from which pair of the table on).
struct Pieces {
    uint32_t first, second;
    bool turn_first, turn_second;
};
template <int D>
__device__ __forceinline__ Pieces pieces_of(uint32_t p, uint32_t rope_dim, uint32_t pairs, bool turns) {
    const uint32_t turned = turns ? rope_dim : 0;
    if (pairs == KVL_ROPE_NEIGHBOURS) return {8 * p, 8 * p + D / 2, 8 * p < turned, 8 * p + D / 2 < turned};
    if (16 * p < turned) return {8 * p, 8 * p + turned / 2, true, true};
    const uint32_t x = 8 * (p - turned / 16) + turned;
    return {x, x + (D - turned) / 2, false, false};
}

template <typename T, typename W>
__device__ __forceinline__ void widen16(u32x4 x, u32x4 y, W (&e)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 a = T::widen(x[i]), b = T::widen(y[i]);
        e[2 * i] = a[0];
        e[2 * i + 1] = a[1];
        e[8 + 2 * i] = b[0];
        e[8 + 2 * i + 1] = b[1];
    }
}

template <int AT, typename W>
__device__ __forceinline__ void turn_neighbours(W (&e)[16], const float *row, uint32_t first, bool turns) {
    if (!turns) return;
    const f32x4 *from = reinterpret_cast<const f32x4 *>(row + first);
    const f32x4 t[2] = {from[0], from[1]};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const W c = t[j / 2][j % 2 * 2], s = t[j / 2][j % 2 * 2 + 1], a = e[AT + 2 * j], b = e[AT + 2 * j + 1];
        e[AT + 2 * j] = a * c - b * s;
        e[AT + 2 * j + 1] = b * c + a * s;
    }
}

// Pieces turned by the angles of table row `position`.
template <typename W>
__device__ __forceinline__ void turn(W (&e)[16], const float *rope, uint32_t position, const Pieces &at, uint32_t rope_dim, uint32_t pairs) {
    const float *row = rope + (uint64_t)position * rope_dim;
    if (pairs == KVL_ROPE_HALVES) {
        if (!at.turn_first) return;
        f32x4 t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = reinterpret_cast<const f32x4 *>(row + 2 * at.first)[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const W c = t[j / 2][j % 2 * 2], s = t[j / 2][j % 2 * 2 + 1], a = e[j], b = e[8 + j];
            e[j] = a * c - b * s;
            e[8 + j] = b * c + a * s;
        }
        asm volatile("");       // (else the two ways' last stores become one, at an index that is not known, and `e` goes to memory)
        return;
    }
    turn_neighbours<0>(e, row, at.first, at.turn_first);
    turn_neighbours<8>(e, row, at.second, at.turn_second);
}

template <typename T>
__device__ __forceinline__ void store16(char *to, uint32_t first, uint32_t second, const float (&e)[16]) {
    u32x4 x, y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = narrow<T>(e[2 * i], e[2 * i + 1]);
        y[i] = narrow<T>(e[8 + 2 * i], e[8 + 2 * i + 1]);
    }
    *reinterpret_cast<u32x4 *>(to + 2 * first) = x;
    *reinterpret_cast<u32x4 *>(to + 2 * second) = y;
}

// One lane's task: two pieces of a head, turned where they have to be.
template <typename T, int D>
__device__ __forceinline__ void half_task(const AppendArgs &a, const char *from, char *to, uint32_t p, uint32_t position, bool turns) {
    const Pieces at = pieces_of<D>(p, a.rope_dim, a.rope_pairs, turns);
    // (read once: past the caches, 9131 tokens 21.5 us against 22.6)
    const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 2 * at.first));
    const u32x4 y = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 2 * at.second));
    if (!at.turn_first) {                       // (the second is not turned either)
        *reinterpret_cast<u32x4 *>(to + 2 * at.first) = x;
        *reinterpret_cast<u32x4 *>(to + 2 * at.second) = y;
        return;
    }
    float e[16];
    widen16<T>(x, y, e);
    turn(e, a.rope, position, at, a.rope_dim, a.rope_pairs);
    store16<T>(to, at.first, at.second, e);
}

// Queries of any cache, keys and values of a 16-bit one: a lane a task, a token's queries, keys and values in a row.
template <typename T, int D>
__device__ __forceinline__ void append_half(const AppendArgs &a, uint64_t task) {
    if (task >= a.tasks) return;
    const uint32_t n = (uint32_t)task / a.per_token, token = a.token_first + n;
    uint32_t j = (uint32_t)task - n * a.per_token;
    const AppendToken at = a.tokens[token];
    constexpr uint32_t kHeadTasks = D / 16;
    if (j < a.q_tasks) {
        const uint32_t head = j / kHeadTasks, p = j % kHeadTasks;
        half_task<T, D>(a, a.q + 2 * (token * a.q_stride + head * D), a.q_out + 2 * (token * a.q_out_stride + head * D), p, at.position, true);
        return;
    }
    j -= a.q_tasks;
    const bool value = j >= a.kv_tasks;
    if (value) j -= a.kv_tasks;
    const uint32_t head = j / kHeadTasks, p = j % kHeadTasks;
    char *to = (value ? a.pool_v : a.pool_k) + 2 * ((uint64_t)at.pool_row * a.kv_heads + head) * D;
    const char *from = value ? a.v + 2 * (token * a.v_stride + head * D) : a.k + 2 * (token * a.k_stride + head * D);
    half_task<T, D>(a, from, to, p, at.position, !value);
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kvl_append_half_kernel(const AppendArgs a) {
    append_half<T, D>(a, (uint64_t)blockIdx.x * blockDim.x + threadIdx.x);
}

constexpr uint32_t kInfinity = 0x7f800000u;

// A double as a float rounded to odd (cut off, with the last bit set where anything was lost): a later rounding to fewer bits then sees which side of
// a tie, or of a border, it was on.  Below the normal floats 0, above the largest that, what is not finite infinite.  By integers: comparisons in 64 bits
// and their branches took half of the time of the kernel below.
__device__ __forceinline__ float to_odd(double x) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t top = (uint32_t)(bits >> 32), size = top & 0x7fffffffu;
    uint32_t f = (((uint32_t)(bits >> 29) - (896u << 23)) & 0x7fffffffu) | min((uint32_t)bits & 0x1fffffffu, 1u);
    f = size < 897u << 20 ? 0 : f;
    f = size >= 1151u << 20 ? (size >= 2047u << 20 ? kInfinity : kInfinity - 1) : f;
    return __uint_as_float(f | (top & 0x80000000u));
}

// Four codes of e4m3: x / scale to the nearest, where x may have been rounded to odd.  `over` is 1 / scale if that is a power of two (the product
// is exact then), else 0.  `odd`: not all of x need be finite.
__device__ __forceinline__ uint32_t codes4(const float *x, float scale, float over, bool odd) {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_fmed3f(over != 0 ? x[i] * over : to_odd((double)x[i] / (double)scale), -448.f, 448.f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    uint32_t u = (uint32_t)w;
    if (odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((__float_as_uint(x[i]) & 0x7fffffffu) >= kInfinity) u |= 0x7fu << (8 * i);
    }
    return u;
}

// The least e in [-32, 63] with most <= 448 * 2^e: 448 is 1.75 * 2^8.
__device__ __forceinline__ int least_exponent(float most) {
    const uint32_t bits = __float_as_uint(most);
    const int e = (int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return e < -32 ? -32 : e > 63 ? 63 : e;
}

// What a workgroup does for one plane of a block and head.
struct CodesPlane {
    const char *from;           // new rows
    char *pool;                 // the head's codes of the block's first row
    float *scale;
    uint64_t stride;            // bytes between new rows
    bool value;
};

// New rows of one block and head into the 8-bit planes.  The scales need the largest of all their values first: rows of up to 64 (of heads of
// 128) wait for it in registers, longer blocks' are read a second time, out of the caches.  Keys are rotated in 64 bits and rounded to odd in
// 32: their codes are then those of the exact values (a rotation in 32 bits moves about one in a million), and all else goes by 32 bits.
template <typename T, int D>
__device__ __forceinline__ void append_codes(const AppendArgs &a, const AppendBlock &b, uint32_t head, f32x2 *most_of_wave) {
    constexpr uint32_t kHeadTasks = D / 16;
    constexpr int N = 2;                        // a lane's tasks of a plane that wait in registers
    const uint64_t row0 = (uint64_t)b.block * a.block_tokens, row_bytes = (uint64_t)a.kv_heads * D, at_scale = (uint64_t)b.block * a.kv_heads + head;
    const CodesPlane planes[2] = {
        {a.k + 2 * (b.token * a.k_stride + head * D), a.pool_k + (row0 * a.kv_heads + head) * D, a.scale_k + at_scale, 2 * a.k_stride, false},
        {a.v + 2 * (b.token * a.v_stride + head * D), a.pool_v + (row0 * a.kv_heads + head) * D, a.scale_v + at_scale, 2 * a.v_stride, true}};
    const uint32_t position = b.position, n = b.n * kHeadTasks, per = blockDim.x;
    float old[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) old[x] = b.row ? in_range(*planes[x].scale) : 0.f;

    auto load = [&](const CodesPlane &plane, uint32_t i, float (&e)[16]) {
        const uint32_t row = i / kHeadTasks;
        const Pieces at = pieces_of<D>(i % kHeadTasks, a.rope_dim, a.rope_pairs, !plane.value);
        const char *x = plane.from + row * plane.stride;
        const u32x4 first = *reinterpret_cast<const u32x4 *>(x + 2 * at.first), second = *reinterpret_cast<const u32x4 *>(x + 2 * at.second);
        if (!at.turn_first) return widen16<T>(first, second, e);
        double d[16];
        widen16<T>(first, second, d);
        turn(d, a.rope, position + row, at, a.rope_dim, a.rope_pairs);
#pragma unroll
        for (int j = 0; j < 16; ++j) e[j] = to_odd(d[j]);
    };
    // the largest of the finite ones; whether all are finite (sizes of floats compare as their bits do)
    auto largest = [](const float (&e)[16], float most, bool *odd) {
        uint32_t size = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) size = max(size, __float_as_uint(e[j]) & 0x7fffffffu);
        *odd = size >= kInfinity;
        if (*odd) {
            size = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t x = __float_as_uint(e[j]) & 0x7fffffffu;
                size = max(size, x < kInfinity ? x : 0u);
            }
        }
        return fmaxf(most, __uint_as_float(size));
    };
    auto store = [&](const CodesPlane &plane, uint32_t i, const float (&e)[16], float scale, float over, bool odd) {
        const Pieces at = pieces_of<D>(i % kHeadTasks, a.rope_dim, a.rope_pairs, !plane.value);
        char *to = plane.pool + (b.row + i / kHeadTasks) * row_bytes;
        *reinterpret_cast<u32x2 *>(to + at.first) = u32x2{codes4(e, scale, over, odd), codes4(e + 4, scale, over, odd)};
        *reinterpret_cast<u32x2 *>(to + at.second) = u32x2{codes4(e + 8, scale, over, odd), codes4(e + 12, scale, over, odd)};
    };

    // (values wait as they came: in half the registers)
    float e[N][16], most[2] = {0, 0};
    u32x4 raw[N][2];
    bool odd[2][N] = {};
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint32_t i = threadIdx.x + j * per;
        if (i >= n) continue;
        const Pieces at = pieces_of<D>(i % kHeadTasks, a.rope_dim, a.rope_pairs, false);
        const char *x = planes[1].from + i / kHeadTasks * planes[1].stride;
        raw[j][0] = *reinterpret_cast<const u32x4 *>(x + 2 * at.first);
        raw[j][1] = *reinterpret_cast<const u32x4 *>(x + 2 * at.second);
        load(planes[0], i, e[j]);
        most[0] = largest(e[j], most[0], &odd[0][j]);
        float w[16];
        widen16<T>(raw[j][0], raw[j][1], w);
        most[1] = largest(w, most[1], &odd[1][j]);
    }
    for (uint32_t i = threadIdx.x + N * per; i < n; i += per)
        for (int x = 0; x < 2; ++x) {
            float w[16];
            bool any;
            load(planes[x], i, w);
            most[x] = largest(w, most[x], &any);
        }
#pragma unroll
    for (int x = 32; x; x >>= 1) {
        most[0] = fmaxf(most[0], __shfl_xor(most[0], x));
        most[1] = fmaxf(most[1], __shfl_xor(most[1], x));
    }
    if (per > 64) {
        if (threadIdx.x % 64 == 0) most_of_wave[threadIdx.x / 64] = f32x2{most[0], most[1]};
        __syncthreads();
        for (uint32_t w = 0; w < per / 64; ++w) {
            most[0] = fmaxf(most[0], most_of_wave[w][0]);
            most[1] = fmaxf(most[1], most_of_wave[w][1]);
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const CodesPlane &plane = planes[x];
        const float scale = fmaxf(old[x], __uint_as_float((uint32_t)(least_exponent(most[x]) + 127) << 23));
        const float over = (__float_as_uint(scale) & 0x7fffffu) == 0 ? 1.f / scale : 0.f;
        if (scale > old[x] && b.row) {          // the codes that are there, to the new scale, which is a power of two
            for (uint32_t i = threadIdx.x; i < b.row * kHeadTasks; i += per) {
                u32x4 *at = reinterpret_cast<u32x4 *>(plane.pool + i / kHeadTasks * row_bytes + i % kHeadTasks * 16);
                u32x4 w = *at;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 c = widen_codes<0>(w[j]), d = widen_codes<1>(w[j]);
                    const float was[4] = {to_odd((double)c[0] * old[x]), to_odd((double)c[1] * old[x]), to_odd((double)d[0] * old[x]), to_odd((double)d[1] * old[x])};
                    w[j] = codes4(was, scale, over, true);
                }
                *at = w;
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t i = threadIdx.x + j * per;
            if (i >= n) continue;
            if (x == 0) {
                store(plane, i, e[j], scale, over, odd[0][j]);
            } else {
                float w[16];
                widen16<T>(raw[j][0], raw[j][1], w);
                store(plane, i, w, scale, over, odd[1][j]);
            }
        }
        for (uint32_t i = threadIdx.x + N * per; i < n; i += per) {
            float w[16];
            load(plane, i, w);
            store(plane, i, w, scale, over, true);
        }
        if (threadIdx.x == 0) *plane.scale = scale;
    }
}

// 8-bit caches: a workgroup for each block that receives rows and each head, and after those workgroups for the queries.
// (Three wavefronts a SIMD, and nothing in scratch memory, which costs every workgroup its start: two 235 us, three with 24 bytes of scratch 211, so 196.)
template <typename T, int D>
__global__ void __launch_bounds__(256, 3) kvl_append_codes_kernel(const AppendArgs a) {
    __shared__ f32x2 most_of_wave[4];
    const uint32_t work = a.n_blocks * a.kv_heads;
    if (blockIdx.x >= work) {
        append_half<T, D>(a, (uint64_t)(blockIdx.x - work) * blockDim.x + threadIdx.x);
        return;
    }
    // (workgroups go to the 8 XCDs in turn: a block's heads to one of them, which has the rows of the table in its cache)
    uint32_t block = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
    if (blockIdx.x < a.n_blocks / 8 * 8 * a.kv_heads) {
        block = blockIdx.x / 8 / a.kv_heads * 8 + blockIdx.x % 8;
        head = blockIdx.x / 8 % a.kv_heads;
    }
    const AppendBlock b = a.blocks[block];
    append_codes<T, D>(a, b, head, most_of_wave);
}

// Up to so many tasks the queries go in the launch of an 8-bit cache's keys and values, beyond in one of their own: its kernel wants a third of
// the registers.  (32 heads of 128 beside 8, 256 tasks a token, us in one / two: 64 tokens 7.0 / 10.9, 4096 22.9 / 28.6, 8192 46 / 53, 16384 86 / 89,
// 32768 168 / 160.)
constexpr uint64_t kOneLaunchTasks = 5u << 20;

template <typename T, int D>
static void launch_append(const kvl_attn_plan_t *plan, AppendArgs a, AttnLaunch &go) {
    const bool codes = plan->layout.cache_dtype == KVL_E4M3;
    a.q_tasks = a.q ? plan->layout.q_heads * (D / 16) : 0;
    a.kv_tasks = codes ? 0 : a.kv_heads * (D / 16);
    a.per_token = a.q_tasks + 2 * a.kv_tasks;
    const uint64_t all = plan->new_tokens * a.per_token;
    const uint32_t threads = plan->most_append_rows * (D / 16) <= 64 ? 64 : 256;
    if (codes && all <= kOneLaunchTasks) {
        a.tasks = all;
        go(true, kvl_append_codes_kernel<T, D>, a.n_blocks * a.kv_heads + (uint32_t)((all + threads - 1) / threads), threads, a);
        return;
    }
    if (codes) go(false, kvl_append_codes_kernel<T, D>, a.n_blocks * a.kv_heads, threads, a);
    // a launch has fewer than 2^32 lanes, and its tasks are numbered in 32 bits
    const uint64_t most_tokens = (1ull << 30) / a.per_token;
    for (uint64_t t = 0; t < plan->new_tokens; t += most_tokens) {
        const uint64_t n = plan->new_tokens - t < most_tokens ? plan->new_tokens - t : most_tokens;
        a.token_first = (uint32_t)t;
        a.tasks = n * a.per_token;
        go(t + n == plan->new_tokens, kvl_append_half_kernel<T, D>, (uint32_t)((a.tasks + 255) / 256), 256, a);
    }
}

static int append_layer(const kvl_attn_plan_t *plan, const kvl_append_t *in, void *const *planes, hipStream_t stream) {
    if (!plan || !in || !planes || !(plan->flags & KVL_SCATTER) || (plan->flags & KVL_HOST_ONLY)) return KVL_EINVAL;
    const kvl_attn_layout_t &l = plan->layout;
    kvl_append_t a = *in;
    if ((a.q == nullptr) != (a.q_out == nullptr) || (l.rope_dim && !a.rope) || reinterpret_cast<uintptr_t>(a.rope) % 16) return KVL_EINVAL;
    int rc = check_attn_pool(plan, planes);
    if (rc != KVL_OK || plan->new_tokens == 0) return rc;
    const uint64_t n = plan->new_tokens;
    if ((rc = check_rows(plan, a.k, n, (uint64_t)l.kv_heads * l.head_dim, &a.k_stride, true)) != KVL_OK) return rc;
    if ((rc = check_rows(plan, a.v, n, (uint64_t)l.kv_heads * l.head_dim, &a.v_stride, true)) != KVL_OK) return rc;
    if (a.q) {
        if ((rc = check_rows(plan, a.q, n, (uint64_t)l.q_heads * l.head_dim, &a.q_stride, true)) != KVL_OK) return rc;
        if ((rc = check_rows(plan, a.q_out, n, (uint64_t)l.q_heads * l.head_dim, &a.q_out_stride, true)) != KVL_OK) return rc;
        if (a.q == a.q_out && a.q_stride != a.q_out_stride) return KVL_EINVAL;
    }
    if (l.rope_dim) {
        if (a.rope_positions <= plan->last_position) return KVL_ESPACE;
        if ((rc = check_buffer(&plan->base, a.rope, (plan->last_position + 1) * l.rope_dim * 4ull, false)) != KVL_OK) return rc;
    }
    const char *lists = reinterpret_cast<const char *>(plan->base.d_units);
    const bool codes = l.cache_dtype == KVL_E4M3;
    AppendArgs args{};
    args.tokens = reinterpret_cast<const AppendToken *>(lists + plan->off_tokens);
    args.blocks = reinterpret_cast<const AppendBlock *>(lists + plan->off_blocks);
    args.k = static_cast<const char *>(a.k);
    args.v = static_cast<const char *>(a.v);
    args.q = static_cast<const char *>(a.q);
    args.q_out = static_cast<char *>(a.q_out);
    args.pool_k = static_cast<char *>(planes[0]);
    args.pool_v = static_cast<char *>(planes[1]);
    args.scale_k = codes ? static_cast<float *>(planes[2]) : nullptr;
    args.scale_v = codes ? static_cast<float *>(planes[3]) : nullptr;
    args.rope = a.rope;
    args.k_stride = a.k_stride;
    args.v_stride = a.v_stride;
    args.q_stride = a.q_stride;
    args.q_out_stride = a.q_out_stride;
    args.rope_dim = l.rope_dim;
    args.rope_pairs = l.rope_pairs;
    args.kv_heads = l.kv_heads;
    args.block_tokens = l.block_tokens;
    args.n_blocks = plan->n_append_blocks;
    AttnLaunch go(plan, stream);
    if (l.dtype == KVL_BF16) {
        if (l.head_dim == 128) launch_append<Bf16, 128>(plan, args, go);
        else launch_append<Bf16, 64>(plan, args, go);
    } else {
        if (l.head_dim == 128) launch_append<F16, 128>(plan, args, go);
        else launch_append<F16, 64>(plan, args, go);
    }
    return go.made();
}

}  // namespace kvl

extern "C" int kvl_append_layer(const kvl_attn_plan_t *plan, const kvl_append_t *args, void *const *pool_planes, void *stream) {
    try {
        return kvl::append_layer(plan, args, pool_planes, static_cast<hipStream_t>(stream));
    } catch (const std::exception &) {
        return KVL_ENOMEM;
    }
}
