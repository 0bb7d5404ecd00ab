// Rules on the scores of arb_attn_rules: the range of keys a query token sees, the cap and the bias by distance.
#pragma once

#include "arb_common.cuh"

namespace arb {

// What the kernels get: scores are kept in log2 units (times log2 e), like the unruled kernels' scaled products.
struct Rules {
    float to_cap;       // softmax scale / cap: raw product -> argument of the tanh; 0: no cap
    float cap_log2;     // cap * log2 e
    int window;
    const float *slopes;
    const int32_t *prefix_lens, *first_keys;
};

// Keys [from, to) that the query token in row `row` of q, at position pos of sequence b, sees; to <= L.
__device__ __forceinline__ void visible_keys(const Rules &r, int b, int row, int pos, int L, int &from, int &to) {
    from = r.first_keys ? max(0, r.first_keys[row]) : 0;
    if (r.window > 0) from = max(from, pos - r.window + 1);
    to = pos + 1;
    if (r.prefix_lens) {
        const int prefix = min(r.prefix_lens[b], L);
        if (pos < prefix) to = prefix;
    }
}

// tanh of |x| <= 1: x + x^3 P(x^2), the coefficients a least-maximum fit of (tanh(x) / x - 1) / x^2 on [0, 1]; relative error
// 1.6e-7 in fp32.
__device__ __forceinline__ float tanh_small(float x) {
    const float u = x * x;
    float p = 1.0582642862573266e-3f;
    p = fmaf(p, u, -6.259338464587927e-3f);
    p = fmaf(p, u, 2.0359758287668228e-2f);
    p = fmaf(p, u, -5.3498707711696625e-2f);
    p = fmaf(p, u, 0.13326409459114075f);
    p = fmaf(p, u, -0.33332985639572144f);
    return fmaf(x * u, p, x);
}

// tanh of any x: beyond 1 as 1 - 2 / (1 + e^2|x|), whose error is a few units of 2^-24 there.  NaN stays NaN.
__device__ __forceinline__ float tanh_any(float x) {
    const float e = fast_exp2(fabsf(x) * 2.8853900817779268f);
    const float big = copysignf(1.0f - __fdividef(2.0f, 1.0f + fminf(e, 1e30f)), x);
    return fabsf(x) <= 1.0f ? tanh_small(x) : (x == x ? big : x);
}

// Launchers (one per translation unit): decode rows of a bf16 cache, without first keys; decode rows of every type; chunks of bf16 with
// ranges alone, with a cap, with slopes; chunks of fp32
arb_status launch_step_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                             const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                             void *out, cudaStream_t stream);
arb_status launch_decode_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                               const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                               void *out, cudaStream_t stream);
arb_status launch_chunk_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                              const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                              void *out, cudaStream_t stream);
arb_status launch_chunk_range(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                              const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                              void *out, cudaStream_t stream);
arb_status launch_chunk_bias(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                             const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                             void *out, cudaStream_t stream);
arb_status launch_chunk_f32_rules(Ctx *ctx, const arb_attn_params &p, const Rules &rules, const void *q, const void *k_pages,
                                  const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                                  void *out, cudaStream_t stream);

}  // namespace arb
