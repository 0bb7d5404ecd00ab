// Launches of the tensor-core chunk kernel (arb_chunk_mma.cuh) over a bf16 and over an E4M3 cache.
#include "arb_chunk_mma.cuh"

namespace arb {

bool chunk_mma_supported(const arb_attn_params &p) {
    return p.dtype == ARB_BF16 && (p.head_dim == 64 || p.head_dim == 128) && p.max_q_len >= 2 && tma_available();
}

namespace {

template <int G>
arb_status launch_g(Ctx *ctx, const MmaArgs &a, bool e4m3, int head_dim, const CUtensorMap &km, const CUtensorMap &vm,
                    int max_items, cudaStream_t stream) {
    if (e4m3) return launch_one<G, true, 128>(ctx, a, km, vm, max_items, stream);
    if (head_dim == 64) return launch_one<G, false, 64>(ctx, a, km, vm, max_items, stream);
    return launch_one<G, false, 128>(ctx, a, km, vm, max_items, stream);
}

arb_status launch_chunk_tc(Ctx *ctx, const arb_attn_params &p, const void *q, const void *k_pages, const void *v_pages,
                           bool e4m3, float k_scale, float v_scale, const int32_t *block_table, const int32_t *seq_lens,
                           const int32_t *q_lens, void *out, bool beside, cudaStream_t stream) {
    alignas(64) CUtensorMap km, vm;
    const PoolView view = e4m3 ? PoolView::kE4m3 : p.head_dim == 64 ? PoolView::kBf16D64 : PoolView::kBf16HalfRows;
    if (!pool_map(ctx, &km, k_pages, p.num_pages, p.num_kv_heads, view) ||
        !pool_map(ctx, &vm, v_pages, p.num_pages, p.num_kv_heads, view))
        return ARB_ERR_CUDA;
    MmaArgs a;
    fill_args(a, ctx, p, q, k_pages, v_pages, k_scale, v_scale, block_table, seq_lens, q_lens, out, beside);
    const int g = p.num_q_heads / p.num_kv_heads, max_items = most_items(a, p);
    switch (g) {
        case 1: return launch_g<1>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 2: return launch_g<2>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 3: return launch_g<3>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 4: return launch_g<4>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 5: return launch_g<5>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 6: return launch_g<6>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 7: return launch_g<7>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        case 8: return launch_g<8>(ctx, a, e4m3, p.head_dim, km, vm, max_items, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace

arb_status launch_chunk_mma(Ctx *ctx, const arb_attn_params &p, const void *q, const void *k_pages,
                            const void *v_pages, const int32_t *block_table, const int32_t *seq_lens,
                            const int32_t *q_lens, void *out, bool beside, cudaStream_t stream) {
    return launch_chunk_tc(ctx, p, q, k_pages, v_pages, false, 1.0f, 1.0f, block_table, seq_lens, q_lens, out, beside, stream);
}

// step chunks over an E4M3 cache (q, out bf16): keys are k_scale * code, values v_scale * code
arb_status launch_chunk_e4m3(Ctx *ctx, const arb_attn_params &p, const void *q, const void *k_codes,
                             const void *v_codes, float k_scale, float v_scale, const int32_t *block_table,
                             const int32_t *seq_lens, const int32_t *q_lens, void *out, bool beside, cudaStream_t stream) {
    if (p.num_q_heads / p.num_kv_heads > 8 || p.batch > kMaxBatchE4m3 || !tma_available()) return ARB_ERR_UNSUPPORTED;
    return launch_chunk_tc(ctx, p, q, k_codes, v_codes, true, k_scale, v_scale, block_table, seq_lens, q_lens, out, beside, stream);
}

}  // namespace arb
