// The tensor-core chunk kernel (arb_chunk_mma.cuh) with ranges of keys and a cap on the scores; the other forms' choice.
#include "arb_chunk_mma.cuh"

namespace arb {

arb_status launch_chunk_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                              const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                              void *out, cudaStream_t stream) {
    if (rules.slopes) return launch_chunk_bias(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    if (rules.to_cap <= 0.f) return launch_chunk_range(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    return launch_ruled<kRules>(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
}

}  // namespace arb
