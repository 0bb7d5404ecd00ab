// Launch of the single-launch token kernel (arb_decode_step.cuh) with rules on the scores.
#include "arb_decode_step.cuh"

namespace arb {

namespace {

template <int G>
arb_status launch_g(Ctx *ctx, const RuledStepArgs &a, int head_dim, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t stream) {
    return head_dim == 64 ? launch_variant<G, false, kKvBf16, 64, true>(ctx, a, km, vm, stream)
                          : launch_variant<G, false, kKvBf16, 128, true>(ctx, a, km, vm, stream);
}

}  // namespace

arb_status launch_step_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                             const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                             void *out, cudaStream_t stream) {
    alignas(64) CUtensorMap km, vm;
    bool whole_rows;
    if (!bf16_maps(ctx, p, k_pages, v_pages, km, vm, whole_rows)) return ARB_ERR_CUDA;
    RuledStepArgs a;
    fill_args(a, ctx, p, q, nullptr, nullptr, const_cast<void *>(k_pages), const_cast<void *>(v_pages), nullptr, block_table,
              const_cast<int32_t *>(seq_lens), q_lens, out, whole_rows, false, nullptr, nullptr);
    a.rules = rules;
    a.inv_cap_log2 = rules.to_cap > 0.f ? 1.0f / rules.cap_log2 : 0.f;
    switch (p.num_q_heads / p.num_kv_heads) {
        case 1: return launch_g<1>(ctx, a, p.head_dim, km, vm, stream);
        case 2: return launch_g<2>(ctx, a, p.head_dim, km, vm, stream);
        case 3: return launch_g<3>(ctx, a, p.head_dim, km, vm, stream);
        case 4: return launch_g<4>(ctx, a, p.head_dim, km, vm, stream);
        case 5: return launch_g<5>(ctx, a, p.head_dim, km, vm, stream);
        case 6: return launch_g<6>(ctx, a, p.head_dim, km, vm, stream);
        case 7: return launch_g<7>(ctx, a, p.head_dim, km, vm, stream);
        case 8: return launch_g<8>(ctx, a, p.head_dim, km, vm, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace arb
