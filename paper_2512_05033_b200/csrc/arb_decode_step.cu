// Launches of the single-launch token kernel (arb_decode_step.cuh) over bf16, E4M3 and 4-bit caches.
#include "arb_decode_step.cuh"

namespace arb {

namespace {

// The 4-bit form exists with the cache write only.
template <int G>
arb_status launch_g(Ctx *ctx, const StepArgs &a, int kv, int head_dim, const CUtensorMap &km, const CUtensorMap &vm,
                    cudaStream_t stream) {
    if (kv == kKvE4m3)
        return a.k_new != nullptr ? launch_variant<G, true, kKvE4m3>(ctx, a, km, vm, stream)
                                  : launch_variant<G, false, kKvE4m3>(ctx, a, km, vm, stream);
    if (kv == kKvI4) return launch_variant<G, true, kKvI4>(ctx, a, km, vm, stream);
    if (head_dim == 64)
        return a.k_new != nullptr ? launch_variant<G, true, kKvBf16, 64>(ctx, a, km, vm, stream)
                                  : launch_variant<G, false, kKvBf16, 64>(ctx, a, km, vm, stream);
    return a.k_new != nullptr ? launch_variant<G, true, kKvBf16>(ctx, a, km, vm, stream)
                              : launch_variant<G, false, kKvBf16>(ctx, a, km, vm, stream);
}

}  // namespace

// every word kEmpty between calls: memset to 0xff
size_t decode_step_slot_bytes(int num_sms) { return sizeof(float) * 2 * (size_t)num_sms * kMaxGroup * (kD + 2); }

bool decode_step_supported(const arb_attn_params &p) {
    const int g = p.num_q_heads / p.num_kv_heads;
    return p.dtype == ARB_BF16 && (p.head_dim == 64 || p.head_dim == 128) && g >= 1 && g <= 8 && tma_available();
}

// k_new == nullptr: attention only (seq_lens is not written).  scales != nullptr: an E4M3 cache with scales =
// {k_scale, v_scale, k_inv_scale, v_inv_scale}; k_row_scales != nullptr: a 4-bit cache with its two scale pools
// (k_new is required); neither: a bf16 cache.
// beside: the decode rows of a call that has chunks too.  The chunk kernel, launched next, reads and writes nothing that this
// one does, so it starts as soon as this kernel's predecessor is known to have completed, and this one takes only its share
// of the SMs (kBesideWeight).
arb_status launch_decode_step(Ctx *ctx, const arb_attn_params &p, const void *q, const void *k_new, const void *v_new,
                              void *k_pages, void *v_pages, const float *scales, const int32_t *block_table,
                              int32_t *seq_lens, const int32_t *q_lens, void *out, cudaStream_t stream, bool beside,
                              float *k_row_scales, float *v_row_scales) {
    alignas(64) CUtensorMap km, vm;
    const bool e4m3 = scales != nullptr, i4 = k_row_scales != nullptr;
    if (i4 && k_new == nullptr) return ARB_ERR_INVALID_ARG;
    if (e4m3 && i4) return ARB_ERR_INVALID_ARG;
    bool whole_rows = false;
    if (i4) {
        if (!pool_map(ctx, &km, k_pages, p.num_pages, p.num_kv_heads, PoolView::kI4) ||
            !pool_map(ctx, &vm, v_pages, p.num_pages, p.num_kv_heads, PoolView::kI4))
            return ARB_ERR_CUDA;
    } else if (e4m3) {
        if (!pool_map(ctx, &km, k_pages, p.num_pages, p.num_kv_heads, PoolView::kE4m3) ||
            !pool_map(ctx, &vm, v_pages, p.num_pages, p.num_kv_heads, PoolView::kE4m3))
            return ARB_ERR_CUDA;
    } else if (!bf16_maps(ctx, p, k_pages, v_pages, km, vm, whole_rows)) {
        return ARB_ERR_CUDA;
    }
    const int g = p.num_q_heads / p.num_kv_heads;
    StepArgs a;
    fill_args(a, ctx, p, q, k_new, v_new, k_pages, v_pages, scales, block_table, seq_lens, q_lens, out, whole_rows, beside, k_row_scales,
              v_row_scales);
    const int kv = i4 ? kKvI4 : e4m3 ? kKvE4m3 : kKvBf16;
    switch (g) {
        case 1: return launch_g<1>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 2: return launch_g<2>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 3: return launch_g<3>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 4: return launch_g<4>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 5: return launch_g<5>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 6: return launch_g<6>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 7: return launch_g<7>(ctx, a, kv, p.head_dim, km, vm, stream);
        case 8: return launch_g<8>(ctx, a, kv, p.head_dim, km, vm, stream);
        default: return ARB_ERR_UNSUPPORTED;
    }
}

}  // namespace arb
