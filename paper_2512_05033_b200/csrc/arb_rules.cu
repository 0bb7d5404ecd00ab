// Dispatch of arb_attn_rules: decode rows and chunks of a call go to the kernels that serve arb_attn's, compiled with the rules.
#include "arb_rules.cuh"

namespace arb {

arb_status launch_attn_rules(Ctx *ctx, const arb_attn_params &p, const arb_score_rules &rules, const void *q, const void *k_pages,
                             const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                             void *out, cudaStream_t stream) {
    const float scale = p.softmax_scale > 0.f ? p.softmax_scale : 1.0f / sqrtf((float)p.head_dim);
    const Rules r = {rules.cap > 0.f ? scale / rules.cap : 0.f, rules.cap * 1.4426950408889634f, rules.window, rules.slopes,
                     rules.prefix_lens, rules.first_keys};
    // the host knows only the total and the maximum of q_lens
    if (p.max_q_len == 1 || p.total_q > p.max_q_len) {
        // the single launch plans from lengths alone; documents' first keys and fp32 take the other kernel
        const arb_status st = decode_step_supported(p) && !r.first_keys
                                  ? launch_step_rules(ctx, p, r, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream)
                                  : launch_decode_rules(ctx, p, r, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
        if (st != ARB_OK) return st;
    }
    if (p.max_q_len < 2) return ARB_OK;
    // With every rule off a chunk is arb_attn's, bit for bit (the rules' kernel has one bf16 term of the weights at 64 dimensions, where that
    // kernel has two).
    const bool off = !(rules.cap > 0.f) && rules.window == 0 && !rules.slopes && !rules.prefix_lens && !rules.first_keys;
    if (off && p.dtype == ARB_F32) return launch_chunk_f32(ctx, p, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    if (off && chunk_mma_supported(p)) return launch_chunk_mma(ctx, p, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, false, stream);
    if (p.dtype == ARB_F32) return launch_chunk_f32_rules(ctx, p, r, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    if (!chunk_mma_supported(p)) return ARB_ERR_UNSUPPORTED;
    return launch_chunk_rules(ctx, p, r, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
}

}  // namespace arb
