// From logits to the next token (arb_logits, see arb.h for the formulas): penalties for tokens a row's history holds, biases,
// temperature, an allowed-token mask, the arg max of x + noise and its log-probability.
//
// One pass over memory: a row of logits is cut into slices of kSlice tokens and a CTA takes one slice.  It asks for its logits
// and noise first, then counts the history's tokens that fall into the slice (integer atomics in shared memory: any order
// gives the same counts) and adds up the biases (one warp walks the list in order, so that a token listed twice gets its sum
// in the order of the list), and only then adjusts, writes and reduces what it holds in registers.  A history is read by every
// CTA of its row, from L2.  The slices' maxima and sums go to the workspace; the CTA of a row that arrives last at the row's
// counter puts them together, slice by slice in order.
//
// Rows of an odd vocabulary start at any element, so a thread's eight tokens are cut at multiples of eight of the flat element
// index: full groups are aligned in every array whose rows lie alike, a row's first and last group are read one by one.
#include "arb_common.cuh"

namespace arb {

namespace {

constexpr int kLogitsThreads = 256;
constexpr int kGroup = 8;                                   // tokens of a vector load
constexpr int kPerThread = 2;                               // groups of a thread
constexpr int kSlice = kLogitsThreads * kPerThread * kGroup;

struct Record {      // what a slice leaves: max and sum of exponentials of x, the best x + noise with its token and its x
    float m, l, best, best_x;
    int token;
    int pad[3];
};

struct LogitsArgs {
    arb_logits_params p;
    Record *records;
    int *counters;
    int slices;      // most that a row has
};

// the better of two candidates: larger, then lower token; token < 0: none
__device__ __forceinline__ bool beats(float a, int ta, float b, int tb) {
    return ta >= 0 && (tb < 0 || a > b || (a == b && ta < tb));
}

__device__ __forceinline__ void merge(Record &a, const Record &o) {
    const float m = fmaxf(a.m, o.m), base = m == -INFINITY ? 0.f : m;
    a.l = a.l * __expf(a.m - base) + o.l * __expf(o.m - base);
    a.m = m;
    if (beats(o.best, o.token, a.best, a.token)) { a.best = o.best; a.best_x = o.best_x; a.token = o.token; }
}

__device__ __forceinline__ Record shfl_xor(const Record &r, int off) {
    Record o;
    o.m = __shfl_xor_sync(0xffffffffu, r.m, off);
    o.l = __shfl_xor_sync(0xffffffffu, r.l, off);
    o.best = __shfl_xor_sync(0xffffffffu, r.best, off);
    o.best_x = __shfl_xor_sync(0xffffffffu, r.best_x, off);
    o.token = __shfl_xor_sync(0xffffffffu, r.token, off);
    return o;
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&x)[8]) {
    Elt<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4 *>(p), x);
}

template <typename T>
__global__ void __launch_bounds__(kLogitsThreads)
logits_kernel(const LogitsArgs a) {
    const arb_logits_params &p = a.p;
    extern __shared__ int counts[];                       // [kSlice], then the biases [kSlice]; each where the call has any
    __shared__ Record warp_rec[kLogitsThreads / 32];
    __shared__ int last;
    const bool history = p.history != nullptr, biased = p.bias_offsets != nullptr;
    float *bias = reinterpret_cast<float *>(counts + (history ? kSlice : 0));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.y, V = p.vocab;
    const long long stride = p.logits_stride ? p.logits_stride : V;
    const T *x_in = static_cast<const T *>(p.logits) + row * stride;
    const float *noise = p.noise ? p.noise + (size_t)row * V : nullptr;
    float *out = p.out ? p.out + (size_t)row * V : nullptr;
    pdl_enter();

    // groups of eight start where the logits' own alignment has them; the dense fp32 arrays' groups agree or are taken one by one
    const int skew = (int)((reinterpret_cast<uintptr_t>(x_in) / sizeof(T)) & (kGroup - 1));
    const bool noise_alike = noise && (int)((reinterpret_cast<uintptr_t>(noise) / 4) & 3) == (skew & 3);
    const bool out_alike = out && (int)((reinterpret_cast<uintptr_t>(out) / 4) & 3) == (skew & 3);
    const int lo = (int)blockIdx.x * kSlice - skew;       // first token of the slice (below 0: the row starts inside a group)
    const float temperature = p.temperature ? p.temperature[row] : 1.0f;
    const bool noisy = noise && temperature > 0.f;

    float x[kPerThread][kGroup], g[kPerThread][kGroup];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int t0 = lo + (k * kLogitsThreads + tid) * kGroup;
        if (t0 >= 0 && t0 + kGroup <= V) {
            load8<T>(x_in + t0, x[k]);
            if (noisy && noise_alike) load8<float>(noise + t0, g[k]);
        } else {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) x[k][i] = (t0 + i >= 0 && t0 + i < V) ? Elt<T>::to_float(x_in[t0 + i]) : -INFINITY;
        }
        if (noisy && !(noise_alike && t0 >= 0 && t0 + kGroup <= V)) {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) g[k][i] = (t0 + i >= 0 && t0 + i < V) ? noise[t0 + i] : 0.f;
        }
    }

    if (history || biased) {
        for (int i = tid; i < kSlice / 4; i += kLogitsThreads) {
            if (history) reinterpret_cast<int4 *>(counts)[i] = make_int4(0, 0, 0, 0);
            if (biased) reinterpret_cast<float4 *>(bias)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        __syncthreads();
        if (history) {
            const int n = p.history_lens ? max(0, min(p.history_lens[row], p.history_stride)) : p.history_stride;
            const int32_t *h = p.history + (size_t)row * p.history_stride;
            for (int i = tid; i < n; i += kLogitsThreads) {
                const int t = h[i];
                if (t >= 0 && t < V && (unsigned)(t - lo) < (unsigned)kSlice) atomicAdd(&counts[t - lo], 1);
            }
        }
        if (biased && warp == 0) {
            const int begin = max(0, min(p.bias_offsets[row], p.bias_total)), end = max(0, min(p.bias_offsets[row + 1], p.bias_total));
            for (int i0 = begin; i0 < end; i0 += 32) {
                const int i = i0 + lane;
                const int t = i < end ? p.bias_tokens[i] : -1;
                const bool mine = t >= 0 && t < V && (unsigned)(t - lo) < (unsigned)kSlice;
                const float value = mine ? p.bias_values[i] : 0.f;
                const int key = mine ? t - lo : -1 - lane;
                const uint32_t same = __match_any_sync(0xffffffffu, key);
                if (__any_sync(0xffffffffu, __popc(same) > 1)) {   // a token listed twice: its values one after the other
                    for (int k = 0; k < 32; ++k) {
                        if (lane == k && mine) bias[key] = __fadd_rn(bias[key], value);
                        __syncwarp();
                    }
                } else if (mine) {
                    bias[key] = __fadd_rn(bias[key], value);
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }

    const float repetition = history && p.repetition ? p.repetition[row] : 1.0f;
    const float presence = history && p.presence ? p.presence[row] : 0.0f;
    const float frequency = history && p.frequency ? p.frequency[row] : 0.0f;
    const uint32_t *mask = p.mask ? p.mask + (size_t)row * p.mask_stride : nullptr;
    Record r;
    r.m = -INFINITY; r.l = 0.f; r.best = -INFINITY; r.best_x = -INFINITY; r.token = -1;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int at = (k * kLogitsThreads + tid) * kGroup, t0 = lo + at;
        if (t0 >= V) continue;
        uint32_t allowed = 0xffu;
        if (mask) {   // bits t0 .. t0 + 7; t0 may lie below 0 and the eight bits in two words
            const int w = max(t0, 0) >> 5, w_last = (V - 1) >> 5;
            const unsigned long long bits = (unsigned long long)mask[w] | (unsigned long long)mask[min(w + 1, w_last)] << 32;
            allowed = t0 >= 0 ? (uint32_t)(bits >> (t0 & 31)) : (uint32_t)bits << -t0;
        }
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int t = t0 + i;
            float v = x[k][i];
            if (history) {
                const int c = counts[at + i];
                if (c > 0) {
                    v = v > 0.f ? __fdiv_rn(v, repetition) : __fmul_rn(v, repetition);
                    v = __fsub_rn(v, presence);
                    v = __fsub_rn(v, __fmul_rn(frequency, (float)c));
                }
            }
            if (biased) v = __fadd_rn(v, bias[at + i]);
            if (p.temperature && temperature > 0.f) v = __fdiv_rn(v, temperature);
            const bool real = t >= 0 && t < V;
            if (!real || !((allowed >> i) & 1u)) v = -INFINITY;
            x[k][i] = v;
            const float y = noisy ? __fadd_rn(v, g[k][i]) : v;
            if (y > r.best) { r.best = y; r.best_x = v; r.token = t; }
        }
        if (out) {
            if (out_alike && t0 >= 0 && t0 + kGroup <= V) {
                *reinterpret_cast<float4 *>(out + t0) = make_float4(x[k][0], x[k][1], x[k][2], x[k][3]);
                *reinterpret_cast<float4 *>(out + t0 + 4) = make_float4(x[k][4], x[k][5], x[k][6], x[k][7]);
            } else {
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                    if (t0 + i >= 0 && t0 + i < V) out[t0 + i] = x[k][i];
            }
        }
    }
    if (!p.tokens && !p.logprobs) return;

#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (lo + (k * kLogitsThreads + tid) * kGroup >= V) continue;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) r.m = fmaxf(r.m, x[k][i]);
    }
    const float base = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (lo + (k * kLogitsThreads + tid) * kGroup >= V) continue;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) r.l += __expf(x[k][i] - base);
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) merge(r, shfl_xor(r, off));
    if (lane == 0) warp_rec[warp] = r;
    __syncthreads();
    if (warp != 0) return;
    r = warp_rec[lane & (kLogitsThreads / 32 - 1)];
    if (lane >= kLogitsThreads / 32) { r.m = -INFINITY; r.l = 0.f; r.token = -1; }
#pragma unroll
    for (int off = kLogitsThreads / 64; off >= 1; off >>= 1) merge(r, shfl_xor(r, off));
    Record *slots = a.records + (size_t)row * a.slices;
    if (a.slices > 1) {
        if (lane == 0) {
            slots[blockIdx.x] = r;
            __threadfence();
            last = atomicAdd(&a.counters[row], 1) == a.slices - 1;
            if (last) a.counters[row] = 0;   // every slice has arrived: ready for the next call
            __threadfence();
        }
        __syncwarp();
        if (!last) return;
        r.m = -INFINITY; r.l = 0.f; r.best = -INFINITY; r.best_x = -INFINITY; r.token = -1;
        for (int i = lane; i < a.slices; i += 32) {
            const float4 f = __ldcg(reinterpret_cast<const float4 *>(slots + i));
            Record o;
            o.m = f.x; o.l = f.y; o.best = f.z; o.best_x = f.w;
            o.token = __ldcg(&slots[i].token);
            merge(r, o);
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) merge(r, shfl_xor(r, off));
    }
    if (lane == 0) {
        if (p.tokens) p.tokens[row] = r.token;
        if (p.logprobs) p.logprobs[row] = r.token < 0 && r.l == r.l ? -INFINITY : r.best_x - r.m - __logf(r.l);
    }
}

}  // namespace

arb_status launch_logits(Ctx *ctx, const arb_logits_params &p, cudaStream_t stream) {
    LogitsArgs a;
    a.p = p;
    a.slices = (p.vocab + kGroup - 1 + kSlice - 1) / kSlice;   // a row may start up to seven elements into a group
    a.records = reinterpret_cast<Record *>(ctx->chunk_ws);
    a.counters = ctx->counters;
    if ((p.tokens || p.logprobs) && (size_t)p.rows * a.slices * sizeof(Record) > ctx->chunk_ws_bytes) return ARB_ERR_WORKSPACE;
    const size_t smem = sizeof(int) * kSlice * ((p.history ? 1 : 0) + (p.bias_offsets ? 1 : 0));
    const dim3 grid(a.slices, p.rows);
    const cudaError_t err = p.dtype == ARB_BF16
                                ? launch_pdl(logits_kernel<__nv_bfloat16>, grid, dim3(kLogitsThreads), smem, stream, a)
                                : launch_pdl(logits_kernel<float>, grid, dim3(kLogitsThreads), smem, stream, a);
    ctx->launches++;
    return err == cudaSuccess ? ARB_OK : ARB_ERR_CUDA;
}

}  // namespace arb
