// Launcher and entry point of attention over a paged cache.
#include <cmath>

#include "kvl_attn_kernels.h"

namespace kvl {

template <typename T, bool E4M3, int D>
static void launch_attn(const kvl_attn_plan_t *plan, AttnArgs a, AttnLaunch &go) {
    const char *lists = reinterpret_cast<const char *>(plan->base.d_units);
    const AttnItem *items = reinterpret_cast<const AttnItem *>(lists + plan->off_items);
    uint32_t left = plan->n_join ? 1 : 0;
    for (uint32_t c = 0; c < kAttnClasses; ++c) left += plan->class_first[c + 1] != plan->class_first[c];
    for (uint32_t c = kAttnClasses; c-- > 0;) {             // the longest workgroups first
        const uint32_t n = plan->class_first[c + 1] - plan->class_first[c];
        if (!n) continue;
        a.items = items + plan->class_first[c];
        const uint32_t groups = n * a.kv_heads;
        const bool last = --left == 0;
        if (c == kRows16) go(last, kvl_attn_few_kernel<T, E4M3, D, 1, 1>, groups, 256, a);
        else if (c == kRows32) go(last, kvl_attn_few_kernel<T, E4M3, D, 2, 1>, groups, 256, a);
        else if (c == kRows64) go(last, kvl_attn_few_kernel<T, E4M3, D, 2, 2>, groups, 256, a);
        else go(last, kvl_attn_many_kernel<T, E4M3, D>, groups, 256, a);
    }
    if (plan->n_join) {
        const JoinItem *joins = reinterpret_cast<const JoinItem *>(lists + plan->off_join);
        const uint32_t groups = plan->join_groups(), all = plan->n_join * a.kv_heads * groups;
        if (plan->join_waves() == 1) go(true, kvl_attn_join_kernel<T, D, 1>, all, 256, a, joins, groups);
        else go(true, kvl_attn_join_kernel<T, D, 4>, all, 256, a, joins, groups);
    }
}

static int attn_layer(const kvl_attn_plan_t *plan, const kvl_attn_t *in, const void *const *planes, hipStream_t stream) {
    if (!plan || !in || !planes || !(plan->flags & KVL_GATHER) || (plan->flags & KVL_HOST_ONLY)) return KVL_EINVAL;
    const kvl_attn_layout_t &l = plan->layout;
    kvl_attn_t t = *in;
    if (!(t.scale > 0) || !std::isfinite(t.scale)) return KVL_EINVAL;
    int rc = check_attn_pool(plan, planes);
    if (rc != KVL_OK || plan->new_tokens == 0) return rc;
    const uint64_t n = plan->new_tokens, row = (uint64_t)l.q_heads * l.head_dim;
    if ((rc = check_rows(plan, t.q, n, row, &t.q_stride, true)) != KVL_OK) return rc;
    if ((rc = check_rows(plan, t.out, n, row, &t.out_stride, true)) != KVL_OK) return rc;
    // (a row's queries are read by the workgroups of its tile alone, before the one or the join that writes it)
    if (t.q == t.out && t.q_stride != t.out_stride) return KVL_EINVAL;
    if (t.lse) {
        uint64_t dense = 0;
        if (reinterpret_cast<uintptr_t>(t.lse) % 4) return KVL_EINVAL;
        if ((rc = check_rows(plan, t.lse, n, l.q_heads, &dense, false)) != KVL_OK) return rc;
    }
    if (plan->workspace_bytes) {
        if (!t.workspace || reinterpret_cast<uintptr_t>(t.workspace) % 256) return KVL_EINVAL;
        if (t.workspace_bytes < plan->workspace_bytes) return KVL_ESPACE;
        if ((rc = check_buffer(&plan->base, t.workspace, plan->workspace_bytes, false)) != KVL_OK) return rc;
    }
    AttnArgs a{};
    const bool codes = l.cache_dtype == KVL_E4M3;
    a.tables = reinterpret_cast<const int32_t *>(reinterpret_cast<const char *>(plan->base.d_units) + plan->off_tables);
    a.k = static_cast<const char *>(planes[0]);
    a.v = static_cast<const char *>(planes[1]);
    a.scale_k = codes ? static_cast<const float *>(planes[2]) : nullptr;
    a.scale_v = codes ? static_cast<const float *>(planes[3]) : nullptr;
    a.q = static_cast<const char *>(t.q);
    a.out = static_cast<char *>(t.out);
    a.lse = t.lse;
    a.workspace = static_cast<float *>(t.workspace);
    a.q_stride = t.q_stride;
    a.out_stride = t.out_stride;
    a.div_mul = plan->div_mul;
    a.div_shift = plan->div_shift;
    a.block_tokens = l.block_tokens;
    a.kv_heads = l.kv_heads;
    a.group = l.q_heads / l.kv_heads;
    a.window = l.window && l.window < (1u << 31) ? l.window : 1u << 31;
    a.sinks = l.sinks;
    a.c = t.scale * 1.4426950408889634f;
    AttnLaunch go(plan, stream);
    const int which = (l.dtype == KVL_F16 ? 4 : 0) + (codes ? 2 : 0) + (l.head_dim == 128 ? 1 : 0);
    switch (which) {
        case 0: launch_attn<Bf16, false, 64>(plan, a, go); break;
        case 1: launch_attn<Bf16, false, 128>(plan, a, go); break;
        case 2: launch_attn<Bf16, true, 64>(plan, a, go); break;
        case 3: launch_attn<Bf16, true, 128>(plan, a, go); break;
        case 4: launch_attn<F16, false, 64>(plan, a, go); break;
        case 5: launch_attn<F16, false, 128>(plan, a, go); break;
        case 6: launch_attn<F16, true, 64>(plan, a, go); break;
        default: launch_attn<F16, true, 128>(plan, a, go); break;
    }
    return go.made();
}

}  // namespace kvl

extern "C" int kvl_attn_layer(const kvl_attn_plan_t *plan, const kvl_attn_t *args, const void *const *pool_planes, void *stream) {
    try {
        return kvl::attn_layer(plan, args, pool_planes, static_cast<hipStream_t>(stream));
    } catch (const std::exception &) {
        return KVL_ENOMEM;
    }
}
