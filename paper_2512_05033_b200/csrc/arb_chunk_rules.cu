// Launch of the tensor-core chunk kernel (arb_chunk_mma.cuh) with ranges of keys and a cap on the scores.
#include "arb_chunk_mma.cuh"

namespace arb {

namespace {

template <int G>
arb_status launch_g(Ctx *ctx, const RuledArgs &a, int head_dim, const CUtensorMap &km, const CUtensorMap &vm, int max_items,
                    cudaStream_t stream) {
    return head_dim == 64 ? launch_one<G, false, 64, kRules>(ctx, a, km, vm, max_items, stream)
                          : launch_one<G, false, 128, kRules>(ctx, a, km, vm, max_items, stream);
}

}  // namespace

arb_status launch_chunk_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                              const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                              void *out, cudaStream_t stream) {
    if (rules.slopes) return launch_chunk_bias(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    if (rules.to_cap <= 0.f) return launch_chunk_range(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    alignas(64) CUtensorMap km, vm;
    const PoolView view = p.head_dim == 64 ? PoolView::kBf16D64 : PoolView::kBf16HalfRows;
    if (!pool_map(ctx, &km, k_pages, p.num_pages, p.num_kv_heads, view) ||
        !pool_map(ctx, &vm, v_pages, p.num_pages, p.num_kv_heads, view))
        return ARB_ERR_CUDA;
    RuledArgs a;
    fill_args(a, ctx, p, q, k_pages, v_pages, 1.0f, 1.0f, block_table, seq_lens, q_lens, out, false);
    a.rules = rules;
    fill_cap(a);
    const int g = p.num_q_heads / p.num_kv_heads, max_items = most_items(a, p);
    switch (g) {
        case 1: return launch_g<1>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 2: return launch_g<2>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 3: return launch_g<3>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 4: return launch_g<4>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 5: return launch_g<5>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 6: return launch_g<6>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 7: return launch_g<7>(ctx, a, p.head_dim, km, vm, max_items, stream);
        case 8: return launch_g<8>(ctx, a, p.head_dim, km, vm, max_items, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace arb
