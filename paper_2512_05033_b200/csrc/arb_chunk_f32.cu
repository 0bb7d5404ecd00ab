// Launch of the fp32 chunk kernel (arb_chunk_f32.cuh).
#include "arb_chunk_f32.cuh"

namespace arb {

namespace {

template <int D>
arb_status launch_g(Ctx *ctx, int g, const F32Args &a, cudaStream_t stream) {
    switch (g) {
        case 1: return launch_one<D, 1>(ctx, a, stream);
        case 2: return launch_one<D, 2>(ctx, a, stream);
        case 3: return launch_one<D, 3>(ctx, a, stream);
        case 4: return launch_one<D, 4>(ctx, a, stream);
        case 5: return launch_one<D, 5>(ctx, a, stream);
        case 6: return launch_one<D, 6>(ctx, a, stream);
        case 7: return launch_one<D, 7>(ctx, a, stream);
        case 8: return launch_one<D, 8>(ctx, a, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace

arb_status launch_chunk_f32(Ctx *ctx, const arb_attn_params &p, const void *q, const void *k_pages, const void *v_pages,
                            const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens, void *out,
                            cudaStream_t stream) {
    F32Args a;
    fill_args(a, ctx, p, q, k_pages, v_pages, block_table, seq_lens, q_lens, out);
    const int g = p.num_q_heads / p.num_kv_heads;
    return p.head_dim == 64 ? launch_g<64>(ctx, g, a, stream) : launch_g<128>(ctx, g, a, stream);
}

}  // namespace arb
