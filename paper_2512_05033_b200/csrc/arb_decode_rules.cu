// Launch of the CUDA-core decode kernel (arb_decode.cuh) with rules on the scores.
#include "arb_decode.cuh"

namespace arb {

namespace {

template <typename T, int D>
arb_status launch_g(Ctx *ctx, int g, const RuledDecodeArgs &a, cudaStream_t stream) {
    switch (g) {
        case 1: return launch_one<T, D, 1, true>(ctx, a, false, stream);
        case 2: return launch_one<T, D, 2, true>(ctx, a, false, stream);
        case 3: return launch_one<T, D, 3, true>(ctx, a, false, stream);
        case 4: return launch_one<T, D, 4, true>(ctx, a, false, stream);
        case 5: return launch_one<T, D, 5, true>(ctx, a, false, stream);
        case 6: return launch_one<T, D, 6, true>(ctx, a, false, stream);
        case 7: return launch_one<T, D, 7, true>(ctx, a, false, stream);
        case 8: return launch_one<T, D, 8, true>(ctx, a, false, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace

arb_status launch_decode_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                               const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                               void *out, cudaStream_t stream) {
    note_unnumbered_decode(ctx, decode_workspace_bytes(p, ctx->num_sms));   // region 0, no generation number
    RuledDecodeArgs a;
    fill_args(a, ctx, p, q, k_pages, v_pages, block_table, seq_lens, q_lens, out);
    a.rules = rules;
    a.inv_cap_log2 = rules.to_cap > 0.f ? 1.0f / rules.cap_log2 : 0.f;
    a.rows = p.total_q;
    const int g = p.num_q_heads / p.num_kv_heads;
    if (p.dtype == ARB_BF16)
        return p.head_dim == 128 ? launch_g<__nv_bfloat16, 128>(ctx, g, a, stream) : launch_g<__nv_bfloat16, 64>(ctx, g, a, stream);
    return p.head_dim == 128 ? launch_g<float, 128>(ctx, g, a, stream) : launch_g<float, 64>(ctx, g, a, stream);
}

}  // namespace arb
