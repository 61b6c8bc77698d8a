// Results of attention over different keys, joined.
#include "kvl_attn_internal.h"
#include "kvl_attn_types.h"
#include "kvl_vectors.h"

namespace kvl {

struct JoinParts {
    const char *parts[KVL_JOIN_MOST];
    uint64_t strides[KVL_JOIN_MOST];    // elements
    const float *lses[KVL_JOIN_MOST];
    char *out;
    float *lse;
    uint64_t out_stride, pieces;        // pieces: of 8 elements, of all tokens
    uint32_t n, per_token, heads;       // per_token: pieces
};

// With w_i = 2^(log2(e) (lse_i - m)), m the largest lse:  out = sum_i w_i x_i / sum_i w_i,  lse = m + log(sum_i w_i).
//
// The bytes bound it: a lane has 8 elements of all parts (at most N) on their way at once, and its row's lses, which the D / 8 lanes of the row
// read together.  PAST: loads and stores pass by the caches, in workgroups of half the size, which suits what is more than these hold (four parts of 64
// heads of 128, us, with the caches / past them: 83 MB 13.9 / 16.2, 166 MB 32.3 / 30.2, 333 MB 62.5 / 56.8, 666 MB, 6.1 TB/s, 122.9 / 108.6).
constexpr uint64_t kJoinPastBytes = 128u << 20;
template <bool PAST>
constexpr uint32_t kJoinThreads = PAST ? 128 : 256;

template <typename T, int D, int N, bool PAST>
__global__ void __launch_bounds__(kJoinThreads<PAST>) kvl_attn_join_parts_kernel(const JoinParts a) {
    const uint64_t first = (uint64_t)blockIdx.x * kJoinThreads<PAST>, token0 = first / a.per_token;
    if (first + threadIdx.x >= a.pieces) return;
    const uint32_t at = (uint32_t)(first - token0 * a.per_token) + threadIdx.x, beyond = at / a.per_token, piece = at - beyond * a.per_token;
    const uint64_t token = token0 + beyond, row = token * a.heads + piece / (D / 8);
    float w[N];
    u32x4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w[i] = -__builtin_inff();
        x[i] = u32x4{0, 0, 0, 0};
        if ((uint32_t)i < a.n) {
            w[i] = a.lses[i][row];
            x[i] = load16<PAST>((gsrc_t)(uintptr_t)(a.parts[i] + 2 * (token * a.strides[i] + piece * 8)));
        }
    }
    float top = w[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, w[i]);
    const float from = top == -__builtin_inff() ? 0.f : top;
    float sum = 0, e[8] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float by = __builtin_amdgcn_exp2f(1.4426950408889634f * (w[i] - from));
        sum += by;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 v = T::widen(x[i][j]);
            // (a part without a share may hold anything)
            e[2 * j] = __builtin_fmaf(by, w[i] == -__builtin_inff() ? 0.f : v[0], e[2 * j]);
            e[2 * j + 1] = __builtin_fmaf(by, w[i] == -__builtin_inff() ? 0.f : v[1], e[2 * j + 1]);
        }
    }
    const float over = sum == 0.f ? 0.f : 1.f / sum;
    u32x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = narrow<T>(e[2 * j] * over, e[2 * j + 1] * over);
    store16<PAST ? 1 : 0>((gdst_t)(uintptr_t)(a.out + 2 * (token * a.out_stride + piece * 8)), y);
    // (the lanes of a row are in one wavefront: all have read its lses)
    if (a.lse && piece % (D / 8) == 0) a.lse[row] = top + 0.69314718055994531f * __log2f(sum);
}

template <typename T, int D, bool PAST>
static void launch_parts(const JoinParts &a, hipStream_t stream) {
    constexpr uint32_t kThreads = kJoinThreads<PAST>;
    const uint32_t groups = (uint32_t)((a.pieces + kThreads - 1) / kThreads);
    if (a.n <= 2) kvl_attn_join_parts_kernel<T, D, 2, PAST><<<groups, kThreads, 0, stream>>>(a);
    else if (a.n <= 4) kvl_attn_join_parts_kernel<T, D, 4, PAST><<<groups, kThreads, 0, stream>>>(a);
    else kvl_attn_join_parts_kernel<T, D, (int)KVL_JOIN_MOST, PAST><<<groups, kThreads, 0, stream>>>(a);
}
template <typename T, int D>
static void launch_join(const JoinParts &a, hipStream_t stream) {
    if ((a.n + 1) * a.pieces * 16 > kJoinPastBytes) launch_parts<T, D, true>(a, stream);
    else launch_parts<T, D, false>(a, stream);
}

static int attn_join(const kvl_attn_plan_t *plan, const kvl_attn_join_t *in, hipStream_t stream) {
    if (!plan || !in || !(plan->flags & KVL_GATHER) || (plan->flags & KVL_HOST_ONLY)) return KVL_EINVAL;
    if (in->n_parts == 0 || in->n_parts > KVL_JOIN_MOST || !in->parts || !in->lses) return KVL_EINVAL;
    int rc = check_device(&plan->base);
    const uint64_t n = plan->new_tokens;
    if (rc != KVL_OK || n == 0) return rc;
    const kvl_attn_layout_t &l = plan->layout;
    const uint64_t row = (uint64_t)l.q_heads * l.head_dim;
    JoinParts a{};
    a.n = in->n_parts;
    a.heads = l.q_heads;
    a.per_token = (uint32_t)(row / 8);
    a.pieces = n * a.per_token;
    a.out_stride = in->out_stride;
    if (a.pieces > UINT32_MAX - 256) return KVL_ERANGE;      // (a lane each, in whole workgroups)
    auto lse_row = [&](const float *lse) {
        uint64_t dense = 0;
        return reinterpret_cast<uintptr_t>(lse) % 4 ? (int)KVL_EINVAL : check_rows(plan, lse, n, l.q_heads, &dense, false);
    };
    if ((rc = check_rows(plan, in->out, n, row, &a.out_stride, true)) != KVL_OK) return rc;
    if (in->lse && (rc = lse_row(in->lse)) != KVL_OK) return rc;
    for (uint32_t i = 0; i < a.n; ++i) {
        a.strides[i] = in->part_strides ? in->part_strides[i] : 0;
        if ((rc = check_rows(plan, in->parts[i], n, row, &a.strides[i], true)) != KVL_OK) return rc;
        if ((rc = lse_row(in->lses[i])) != KVL_OK) return rc;
        // (a lane reads what it writes, and nobody else does)
        if (in->parts[i] == in->out && a.strides[i] != a.out_stride) return KVL_EINVAL;
        a.parts[i] = static_cast<const char *>(in->parts[i]);
        a.lses[i] = in->lses[i];
    }
    a.out = static_cast<char *>(in->out);
    a.lse = in->lse;
    if (l.dtype == KVL_F16) l.head_dim == 128 ? launch_join<F16, 128>(a, stream) : launch_join<F16, 64>(a, stream);
    else l.head_dim == 128 ? launch_join<Bf16, 128>(a, stream) : launch_join<Bf16, 64>(a, stream);
    KVL_HIP(hipGetLastError());
    return KVL_OK;
}

}  // namespace kvl

extern "C" int kvl_attn_join(const kvl_attn_plan_t *plan, const kvl_attn_join_t *args, void *stream) {
    try {
        return kvl::attn_join(plan, args, static_cast<hipStream_t>(stream));
    } catch (const std::exception &) {
        return KVL_ENOMEM;
    }
}
