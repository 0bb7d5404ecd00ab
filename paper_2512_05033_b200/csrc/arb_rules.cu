// Attention with rules on the scores (arb_attn_rules): bf16 on the tensor-core chunk kernel; fp32 here, a warp per (query row,
// head), keys in groups of 32.
#include "arb_rules.cuh"

namespace arb {

namespace {

constexpr int kThreads = 256;

struct RulesArgs {
    const char *q, *k_pages, *v_pages;
    const int32_t *block_table, *seq_lens, *q_lens;
    char *out;
    uint32_t *status;
    int batch, Hq, Hkv, num_pages, max_pages, rows;
    float scale, scale_log2;
    Rules rules;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
rules_kernel(const RulesArgs a) {
    constexpr int kPer = D / 32;
    extern __shared__ int row0[];   // [B + 1] rows of q before sequence b
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = a.batch, G = a.Hq / a.Hkv;
    pdl_enter();
    if (threadIdx.x == 0) {
        row0[0] = 0;
        for (int b = 0; b < B; ++b) row0[b + 1] = row0[b] + max(a.q_lens[b], 0);
    }
    __syncthreads();
    const int rows = min(a.rows, row0[B]);
    for (long long u = (long long)blockIdx.x * (kThreads / 32) + warp; u < (long long)rows * a.Hq; u += (long long)gridDim.x * (kThreads / 32)) {
        const int row = (int)(u / a.Hq), h = (int)(u - (long long)row * a.Hq), kvh = h / G;
        int b = 0, hi = B;
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (row0[mid] <= row) b = mid; else hi = mid;
        }
        const int n = a.q_lens[b], L = a.seq_lens[b], pos = L - n + (row - row0[b]);
        int from = 0, to = 0;
        if (L < n || n > a.rows || L > a.max_pages * kPage) {
            if (lane == 0) atomicOr(a.status, (uint32_t)ARB_DEV_BAD_SEQ_LEN);
        } else {
            visible_keys(a.rules, b, row, pos, L, from, to);
        }
        const T *q = reinterpret_cast<const T *>(a.q) + ((size_t)row * a.Hq + h) * D;
        const float slope = a.rules.slopes ? a.rules.slopes[h] * 1.4426950408889634f : 0.f;
        float m = -INFINITY, l = 0.f, o[kPer] = {};
        for (int j0 = from; j0 < to; j0 += 32) {
            const int j = j0 + lane;
            float s = -INFINITY;
            long long at = 0;
            if (j < to) {
                int page = a.block_table[(size_t)b * a.max_pages + j / kPage];
                if ((unsigned)page >= (unsigned)a.num_pages) { atomicOr(a.status, (uint32_t)ARB_DEV_BAD_PAGE); page = 0; }
                at = (((long long)page * a.Hkv + kvh) * kPage + j % kPage) * D;
                const T *k = reinterpret_cast<const T *>(a.k_pages) + at;
                float dot = 0.f;
                for (int d = 0; d < D; ++d) dot = fmaf(Elt<T>::to_float(q[d]), Elt<T>::to_float(k[d]), dot);
                s = a.rules.to_cap > 0.f ? a.rules.cap_log2 * tanh_any(dot * a.rules.to_cap) : dot * a.scale_log2;
                s = fmaf(-slope, (float)abs(pos - j), s);
            }
            float mx = s;
            for (int off = 16; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.f : mn, f = fast_exp2(m - base), p = fast_exp2(s - base);
            m = mn;
            float sum = p;
            for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            l = fmaf(l, f, sum);
            for (int i = 0; i < kPer; ++i) o[i] *= f;
            for (int k = 0; k < min(32, to - j0); ++k) {
                const float pk = __shfl_sync(0xffffffffu, p, k);
                const long long vat = __shfl_sync(0xffffffffu, at, k);
                const T *v = reinterpret_cast<const T *>(a.v_pages) + vat;
                for (int i = 0; i < kPer; ++i) o[i] = fmaf(pk, Elt<T>::to_float(v[lane + 32 * i]), o[i]);
            }
        }
        T *out = reinterpret_cast<T *>(a.out) + ((size_t)row * a.Hq + h) * D;
        for (int i = 0; i < kPer; ++i) out[lane + 32 * i] = Elt<T>::from_float(l > 0.f ? o[i] / l : 0.f);
    }
}

}  // namespace

arb_status launch_attn_rules(Ctx *ctx, const arb_attn_params &p, const arb_score_rules &rules, const void *q, const void *k_pages,
                             const void *v_pages, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens,
                             void *out, cudaStream_t stream) {
    RulesArgs a;
    a.q = static_cast<const char *>(q);
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.q_lens = q_lens;
    a.out = static_cast<char *>(out);
    a.status = ctx->status;
    a.batch = p.batch;
    a.Hq = p.num_q_heads;
    a.Hkv = p.num_kv_heads;
    a.num_pages = p.num_pages;
    a.max_pages = p.max_pages_per_seq;
    a.rows = p.total_q;
    a.scale = p.softmax_scale > 0.f ? p.softmax_scale : 1.0f / sqrtf((float)p.head_dim);
    a.scale_log2 = a.scale * 1.4426950408889634f;
    a.rules = {rules.cap > 0.f ? a.scale / rules.cap : 0.f, rules.cap * 1.4426950408889634f, rules.window, rules.slopes,
               rules.prefix_lens, rules.first_keys};
    if (p.dtype == ARB_BF16)
        return launch_chunk_rules(ctx, p, a.rules, 1, q, k_pages, v_pages, block_table, seq_lens, q_lens, out, stream);
    const dim3 grid(ctx->num_sms * 8);
    const size_t smem = sizeof(int) * ((size_t)p.batch + 1);
    const cudaError_t err =
        p.head_dim == 128 ? launch_pdl(rules_kernel<float, 128>, grid, dim3(kThreads), smem, stream, a)
                                : launch_pdl(rules_kernel<float, 64>, grid, dim3(kThreads), smem, stream, a);
    ctx->launches++;
    return err == cudaSuccess ? ARB_OK : ARB_ERR_CUDA;
}

}  // namespace arb
