// New keys and values into a paged cache, rotated by their positions: kernels and entry point.
//
// Pairs (a, b) of a head's leading rope_dim elements become (a cos - b sin, b cos + a sin).  A lane takes 16 elements
// that belong together: pieces of 8 at j and j + rope_dim/2 (halves), or 16 in a row (neighbours, and what is not rotated);
// either way its 8 pairs' cosines and sines are 64 bytes in a row of the table, which the heads of a token share in the
// caches.  Memory bounds both kernels: each element is read once and written once.
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

// Where a lane's two pieces of 8 elements lie in a head.
template <int D>
__device__ __forceinline__ void pieces_of(uint32_t p, uint32_t rope_dim, uint32_t pairs, bool turns, uint32_t *first, uint32_t *second, bool *rotate) {
    *rotate = turns && p < rope_dim / 16;
    *first = *rotate && pairs == KVL_ROPE_HALVES ? 8 * p : 16 * p;
    *second = *rotate && pairs == KVL_ROPE_HALVES ? 8 * p + rope_dim / 2 : 16 * p + 8;
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

// The 8 pairs of 16 elements turned by the angles of table row `position`, from pair 8 p on.
template <typename W>
__device__ __forceinline__ void turn(W (&e)[16], const float *rope, uint32_t position, uint32_t p, uint32_t rope_dim, uint32_t pairs) {
    const f32x4 *cs = reinterpret_cast<const f32x4 *>(rope + (uint64_t)position * rope_dim + 16 * p);
    f32x4 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = cs[i];
    if (pairs == KVL_ROPE_HALVES) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const W c = t[j / 2][j % 2 * 2], s = t[j / 2][j % 2 * 2 + 1], a = e[j], b = e[8 + j];
            e[j] = a * c - b * s;
            e[8 + j] = b * c + a * s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const W c = t[j / 2][j % 2 * 2], s = t[j / 2][j % 2 * 2 + 1], a = e[2 * j], b = e[2 * j + 1];
            e[2 * j] = a * c - b * s;
            e[2 * j + 1] = b * c + a * s;
        }
    }
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

// One task of 16 elements of a row of half-precision elements, turned where it has to be.
template <typename T, int D>
__device__ __forceinline__ void half_task(const AppendArgs &a, const char *from, char *to, uint32_t p, uint32_t position, bool turns) {
    uint32_t first, second;
    bool rotate;
    pieces_of<D>(p, a.rope_dim, a.rope_pairs, turns, &first, &second, &rotate);
    const u32x4 x = *reinterpret_cast<const u32x4 *>(from + 2 * first), y = *reinterpret_cast<const u32x4 *>(from + 2 * second);
    if (!rotate) {
        *reinterpret_cast<u32x4 *>(to + 2 * first) = x;
        *reinterpret_cast<u32x4 *>(to + 2 * second) = y;
        return;
    }
    float e[16];
    widen16<T>(x, y, e);
    turn(e, a.rope, position, p, a.rope_dim, a.rope_pairs);
    store16<T>(to, first, second, e);
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

// The code of e4m3 nearest to x / scale, where `over` is 1 / scale if that is exact and else 0.  x goes to 32 bits by
// rounding to odd, so that the rounding to 8 that follows sees which side of a tie it was on.
__device__ __forceinline__ float for_code(double x, double scale, double over) {
    const double y = over != 0 ? x * over : x / scale;
    float f = (float)fmin(fmax(y, -448.0), 448.0);
    const double rest = y - (double)f;
    const uint32_t bits = __float_as_uint(f);
    if (rest != 0 && !(bits & 1u) && fabsf(f) >= 0x1p-20f && fabsf(f) < 448.f) f = __uint_as_float((rest > 0) == (f > 0) ? bits + 1 : bits - 1);
    return f;
}
__device__ __forceinline__ uint32_t codes4(const double *x, double scale, double over) {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = for_code(x[i], scale, over);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    uint32_t u = (uint32_t)w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabs(x[i]) < __builtin_inf())) u |= 0x7fu << (8 * i);
    return u;
}

// The least e in [-32, 63] with most <= 448 * 2^e: 448 is 1.75 * 2^8.
__device__ __forceinline__ int least_exponent(double most) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, most);
    if (bits == 0) return -32;
    const int e = (int)(bits >> 52) - 1023 - ((bits & 0xfffffffffffffull) <= 0xc000000000000ull ? 8 : 7);
    return e < -32 ? -32 : e > 63 ? 63 : e;
}

// New rows of one block and head into an 8-bit plane.  The scale needs the largest of all of them first, so the rows are gone
// through twice; the second time they come from the caches.  Rotated in 64 bits: the values' rounding to 8 bits is then that of
// the exact ones (a 32-bit rotation moves about one code in a million), and 64-bit arithmetic is a small part of the time.
template <typename T, int D>
__device__ __forceinline__ void append_codes(const AppendArgs &a, const AppendBlock &b, uint32_t head, bool value, double *most_of_wave) {
    constexpr uint32_t kHeadTasks = D / 16;
    const uint64_t stride = value ? a.v_stride : a.k_stride;
    const char *from = (value ? a.v : a.k) + 2 * (b.token * stride + head * D);
    const uint64_t row0 = (uint64_t)b.block * a.block_tokens;
    char *pool = (value ? a.pool_v : a.pool_k) + (row0 * a.kv_heads + head) * D;
    const uint64_t row_bytes = (uint64_t)a.kv_heads * D;
    float *scales = (value ? a.scale_v : a.scale_k) + (uint64_t)b.block * a.kv_heads + head;
    const uint32_t position = a.tokens[b.token].position, n = b.n * kHeadTasks;
    const float old = b.row ? *scales : 0.f;

    auto load = [&](uint32_t i, double (&e)[16], uint32_t *first, uint32_t *second) {
        const uint32_t row = i / kHeadTasks, p = i % kHeadTasks;
        bool rotate;
        pieces_of<D>(p, a.rope_dim, a.rope_pairs, !value, first, second, &rotate);
        const char *x = from + 2 * row * stride;
        widen16<T>(*reinterpret_cast<const u32x4 *>(x + 2 * *first), *reinterpret_cast<const u32x4 *>(x + 2 * *second), e);
        if (rotate) turn(e, a.rope, position + row, p, a.rope_dim, a.rope_pairs);
    };
    double most = 0;
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        double e[16];
        uint32_t first, second;
        load(i, e, &first, &second);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const double m = fabs(e[j]);
            if (m < __builtin_inf()) most = fmax(most, m);
        }
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) most = fmax(most, __shfl_xor(most, x));
    if (blockDim.x > 64) {
        __syncthreads();                        // (the plane before has read it)
        if (threadIdx.x % 64 == 0) most_of_wave[threadIdx.x / 64] = most;
        __syncthreads();
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) most = fmax(most, most_of_wave[w]);
    }
    const float fresh = __uint_as_float((uint32_t)(least_exponent(most) + 127) << 23);
    const float scale = fmaxf(old, fresh);
    const bool power = (__float_as_uint(scale) & 0x7fffffu) == 0;
    const double over = power ? 1.0 / (double)scale : 0.0;
    if (scale > old && b.row) {                 // the codes that are there, to the new scale
        const double ratio = (double)old / (double)scale;
        for (uint32_t i = threadIdx.x; i < b.row * kHeadTasks; i += blockDim.x) {
            u32x4 *at = reinterpret_cast<u32x4 *>(pool + i / kHeadTasks * row_bytes + i % kHeadTasks * 16);
            u32x4 w = *at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 x = widen_codes<0>(w[j]), y = widen_codes<1>(w[j]);
                const double e[4] = {x[0] * ratio, x[1] * ratio, y[0] * ratio, y[1] * ratio};
                w[j] = codes4(e, 1.0, 1.0);
            }
            *at = w;
        }
    }
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        double e[16];
        uint32_t first, second;
        load(i, e, &first, &second);
        char *to = pool + (b.row + i / kHeadTasks) * row_bytes;
        *reinterpret_cast<u32x2 *>(to + first) = u32x2{codes4(e, scale, over), codes4(e + 4, scale, over)};
        *reinterpret_cast<u32x2 *>(to + second) = u32x2{codes4(e + 8, scale, over), codes4(e + 12, scale, over)};
    }
    if (threadIdx.x == 0) *scales = scale;
}

// 8-bit caches: a workgroup for each block that receives rows and each head, and after those workgroups for the queries.
template <typename T, int D>
__global__ void __launch_bounds__(256) kvl_append_codes_kernel(const AppendArgs a) {
    __shared__ double most_of_wave[4];
    const uint32_t work = a.n_blocks * a.kv_heads;
    if (blockIdx.x >= work) {
        append_half<T, D>(a, (uint64_t)(blockIdx.x - work) * blockDim.x + threadIdx.x);
        return;
    }
    const AppendBlock b = a.blocks[blockIdx.x / a.kv_heads];
    const uint32_t head = blockIdx.x % a.kv_heads;
    append_codes<T, D>(a, b, head, false, most_of_wave);
    append_codes<T, D>(a, b, head, true, most_of_wave);
}

template <typename T, int D>
static void launch_append(const kvl_attn_plan_t *plan, AppendArgs a, AttnLaunch &go) {
    const bool codes = plan->layout.cache_dtype == KVL_E4M3;
    a.q_tasks = a.q ? plan->layout.q_heads * (D / 16) : 0;
    a.kv_tasks = codes ? 0 : a.kv_heads * (D / 16);
    a.per_token = a.q_tasks + 2 * a.kv_tasks;
    // a launch has fewer than 2^32 lanes, and its tasks are numbered in 32 bits
    const uint64_t most_tokens = a.per_token ? (1ull << 30) / a.per_token : plan->new_tokens;
    for (uint64_t t = 0; t < plan->new_tokens; t += most_tokens) {
        const uint64_t n = plan->new_tokens - t < most_tokens ? plan->new_tokens - t : most_tokens;
        const bool last = t + n == plan->new_tokens;
        a.token_first = (uint32_t)t;
        a.tasks = n * a.per_token;
        if (codes && t == 0) {
            const uint32_t threads = plan->most_append_rows * (D / 16) <= 64 ? 64 : 256;
            go(last, kvl_append_codes_kernel<T, D>, a.n_blocks * a.kv_heads + (uint32_t)((a.tasks + threads - 1) / threads), threads, a);
        } else {
            const uint32_t threads = 256;
            go(last, kvl_append_half_kernel<T, D>, (uint32_t)((a.tasks + threads - 1) / threads), threads, a);
        }
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
