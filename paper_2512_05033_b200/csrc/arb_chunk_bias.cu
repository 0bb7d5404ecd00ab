// The tensor-core chunk kernel (arb_chunk_mma.cuh) with a bias by distance beside the other rules.
#include "arb_chunk_mma.cuh"

namespace arb {

arb_status launch_chunk_bias(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                              const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                              void *out, cudaStream_t stream) {
    return launch_ruled<kRulesBias>(ctx, p, rules, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
}

}  // namespace arb
