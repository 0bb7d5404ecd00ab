// Norm, rotation and cache write in one pass: a projection's raw query, key and value rows come in, normed and rotated queries
// go out, keys and values go into the paged cache (arb_rope_append and its two quantising forms, see arb.h for the formulas).
//
// Plain memory movement with some arithmetic on the way: every row is read once and written once, (Hq + 2 Hkv) D elements a
// token each way.  A row of D values is held by D / 8 neighbouring lanes, eight values each, as two vectors of four that hold
// both members of four rotation pairs: (p .. p + 3, p + rot / 2 ..) or eight neighbours, so that no lane needs another's
// values to rotate.  The rows of one token share their four angles per lane: a warp takes neighbouring heads of a token, works
// out sines and cosines once (position times frequency in 64 bits, reduced to a part of a turn: the error of an angle does not
// grow with the position) and goes through its rows kind by kind, so that the lane groups of a warp never part ways.
// Prompts of 256 to 2048 tokens, 32 / 8 heads of 128 (453 MB, 70 us at the copy rate): a lane group per token's rows, each looking
// up its kind, 122 us (200 instructions a row); this way 103; with equal shares of a token 89 us, 5.1 TB/s.  Four CTAs per SM with
// two rows in flight 96 us, five 126.  A token of 8 sequences, 12 / 2 heads: 3.6 us, launch and look-ups.
#include "arb_append.cuh"

#include <type_traits>

namespace arb {

namespace {

enum class Kv { kSame, kE4m3, kI4 };

struct RopeArgs {
    AppendArgs a;       // k_new, v_new: tokens k_stride, v_stride bytes apart
    const char *q;
    char *q_out;
    const float *q_weight, *k_weight, *inv_freq;
    const int32_t *positions;
    long long q_stride, k_stride, v_stride;   // bytes from a token to the next
    float *k_scales, *v_scales;               // 4-bit cache
    float k_inv_scale, v_inv_scale;           // E4M3 cache
    float eps;
    int Hq, rot;
    int heads_per_unit, units_per_token;      // a lane group's share: so many of a token's Hq + 2 Hkv rows
};

constexpr int kRopeRows = 4;   // rows of a lane group in flight
constexpr int kRopeCtas = 3;   // resident CTAs of an SM

template <typename T> struct Four;
template <> struct Four<float> { using V = uint4; };
template <> struct Four<__nv_bfloat16> { using V = uint2; };

__device__ __forceinline__ void unpack4(const uint4 &v, float *x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack4(const uint2 &v, float *x) {
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void pack4(const float *x, uint4 &v) {
    v = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ void pack4(const float *x, uint2 &v) { v = make_uint2(bf16x2_of(x[0], x[1]), bf16x2_of(x[2], x[3])); }

__device__ __forceinline__ uint32_t e4m3x4(const float *x, float s) {
    return e4m3x2(x[0] * s, x[1] * s) | (e4m3x2(x[2] * s, x[3] * s) << 16);
}

// The 4-bit words of a row's dimensions off0 .. off0 + 3 (x[0..3]) and off1 .. off1 + 3 (x[4..7]); the other four dimensions
// of either group of eight are lane ^ 1's.  The even lane writes the first group's word, the odd lane the second's.
__device__ __forceinline__ void store_i4_halves(char *row, const float (&x)[8], float inv, int off0, int off1, uint32_t group_mask) {
    uint32_t w[2] = {0u, 0u};
    const int odd = threadIdx.x & 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = max(-7, min(7, __float2int_rn(__fmul_rn(x[i], inv)))), j = 4 * odd + (i & 3);
        w[i >> 2] |= (uint32_t)(c + 8) << (4 * ((j >> 1) + 4 * (j & 1)));
    }
    w[0] |= __shfl_xor_sync(group_mask, w[0], 1);
    w[1] |= __shfl_xor_sync(group_mask, w[1], 1);
    *reinterpret_cast<uint32_t *>(row + ((odd ? off1 : off0) >> 3) * 4) = w[odd];
}

template <typename T, int D, Kv KV, bool INTER>
__global__ void __launch_bounds__(kAppendThreads, kRopeCtas)
rope_append_kernel(const RopeArgs r) {
    using V = typename Four<T>::V;
    constexpr int kLanes = D / 8;                       // lanes of a row
    constexpr int kGroups = 32 / kLanes;                // lane groups of a warp: neighbouring heads of a token
    constexpr int kRowBytes = D * (int)sizeof(T);
    extern __shared__ int asm_[];
    const AppendArgs &a = r.a;
    pdl_enter();
    const AppendPlan pl = append_plan(a, asm_);
    const int l = threadIdx.x % kLanes, p0 = 4 * l;
    const uint32_t group_mask = (uint32_t)((1ull << kLanes) - 1) << (threadIdx.x & 31 & ~(kLanes - 1));
    const bool turns = p0 < r.rot / 2;
    int off0 = 8 * l, off1 = 8 * l + 4;                 // this lane's dimensions: off0 .. + 3, off1 .. + 3
    if (!INTER) {
        off0 = turns ? p0 : r.rot + (p0 - r.rot / 2);
        off1 = off0 + (turns ? r.rot / 2 : (D - r.rot) / 2);
    }
    const int heads = r.Hq + 2 * a.Hkv, mine = (threadIdx.x & 31) / kLanes;   // this lane's group of the warp
    const unsigned units = (unsigned)pl.pref[a.batch] * (unsigned)r.units_per_token;
    const unsigned warps = gridDim.x * (kAppendThreads / 32);
    for (unsigned u = blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32; u < units; u += warps) {
        const int tok = (int)(u / (unsigned)r.units_per_token), h_begin = ((int)u - tok * r.units_per_token) * r.heads_per_unit;
        const int h_end = min(h_begin + r.heads_per_unit, heads);
        // Rows h .. seg_end - 1 of the unit (the same for the whole warp) are of one kind (0: queries, 1: keys, 2: values) and lie D elements apart.  The first
        // rows are asked for before anything else is looked up.
        int h = h_begin, kind, seg_end;
        const char *src;
        auto aim = [&]() {
            const int k_begin = r.Hq, v_begin = r.Hq + a.Hkv;
            kind = (h >= k_begin) + (h >= v_begin);
            seg_end = min(h_end, kind == 0 ? k_begin : kind == 1 ? v_begin : heads);
            src = kind == 0 ? r.q + tok * r.q_stride : kind == 1 ? a.k_new + tok * r.k_stride : a.v_new + tok * r.v_stride;
            src += (h - (kind == 0 ? 0 : kind == 1 ? k_begin : v_begin) + mine) * kRowBytes;
        };
        V raw[kRopeRows][2];
        auto load = [&]() {
            const char *at0 = src + off0 * (int)sizeof(T), *at1 = src + off1 * (int)sizeof(T);
#pragma unroll
            for (int k = 0; k < kRopeRows; ++k) {
                if (h + k * kGroups + mine < seg_end) {
                    raw[k][0] = *reinterpret_cast<const V *>(at0 + k * kGroups * kRowBytes);
                    raw[k][1] = *reinterpret_cast<const V *>(at1 + k * kGroups * kRowBytes);
                }
            }
        };
        aim();
        load();
        int b = 0, hi = a.batch;
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (pl.pref[mid] <= tok) b = mid; else hi = mid;
        }
        const bool okay = pl.okay[b];
        const int place = okay ? pl.start[b] + (tok - pl.pref[b]) : 0;
        long long slot = okay ? (long long)a.block_table[(size_t)b * a.max_pages + place / kPage] * a.Hkv * kPage + place % kPage : 0;
        if (!ARB_IN_RANGE(a.status, slot, (long long)a.num_pages * a.Hkv * kPage - (a.Hkv - 1) * kPage)) slot = 0;
        float c[4], s[4];
        if (turns && kind < 2) {
            const double pos = (double)(r.positions ? r.positions[tok] : place) * 0.15915494309189533577;   // 1 / (2 pi): in turns
            const float4 f = __ldg(reinterpret_cast<const float4 *>(r.inv_freq + p0));
            const float ff[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double t = pos * (double)ff[i];
                const float part = (float)(t - rint(t));   // -0.5 .. 0.5 of a turn
                if constexpr (sizeof(T) == 4) {
                    sincospif(2.0f * part, &s[i], &c[i]);
                } else {   // 2^-20 absolute, where the rows are known to 2^-9
                    __sincosf(6.2831853071795865f * part, &s[i], &c[i]);
                }
            }
        }
        // kRopeRows rows of one kind, which is a constant of each instance
        auto rows = [&](auto kind_c) {
            constexpr int K = decltype(kind_c)::value;
            float w[8];
            const float *weight = K == 0 ? r.q_weight : r.k_weight;
            const bool norm = K < 2 && weight != nullptr;
            if (norm) {
                const float4 w0 = __ldg(reinterpret_cast<const float4 *>(weight + off0)), w1 = __ldg(reinterpret_cast<const float4 *>(weight + off1));
                w[0] = w0.x; w[1] = w0.y; w[2] = w0.z; w[3] = w0.w; w[4] = w1.x; w[5] = w1.y; w[6] = w1.z; w[7] = w1.w;
            }
            const int head = (K == 0 ? h : K == 1 ? h - r.Hq : h - r.Hq - a.Hkv) + mine;   // of its kind
            constexpr int kOutRow = K == 0 || KV == Kv::kSame ? kRowBytes : KV == Kv::kE4m3 ? D : D / 2;   // bytes
            constexpr int kOutStep = kGroups * (K == 0 ? kOutRow : kPage * kOutRow);                        // from row to row of the lane
            const long long row0 = K == 0 ? (long long)tok * r.Hq + head : slot + (long long)head * kPage;
            char *dst = (K == 0 ? r.q_out : K == 1 ? a.k_pages : a.v_pages) + row0 * kOutRow;
#pragma unroll
            for (int k = 0; k < kRopeRows; ++k) {
                if (h + k * kGroups + mine >= seg_end) continue;   // (the same for the lanes of a group)
                float x[8];
                unpack4(raw[k][0], x);
                unpack4(raw[k][1], x + 4);
                if (norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
                    for (int off = kLanes / 2; off >= 1; off >>= 1) ss += __shfl_xor_sync(group_mask, ss, off);
                    const float inv = rsqrtf(ss * (1.0f / D) + r.eps);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= inv * w[i];
                }
                if (K < 2 && turns) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &e = INTER ? x[2 * i] : x[i], &o = INTER ? x[2 * i + 1] : x[4 + i];
                        const float y = e * c[i] - o * s[i];
                        o = e * s[i] + o * c[i];
                        e = y;
                    }
                }
                char *at = dst + k * kOutStep;
                if constexpr (K == 0 || KV == Kv::kSame) {
                    V y0 = raw[k][0], y1 = raw[k][1];   // values bit for bit
                    if (K < 2) { pack4(x, y0); pack4(x + 4, y1); }
                    if (K == 0 && !okay) y0 = y1 = V{};   // (a refused sequence: rows of zeros)
                    *reinterpret_cast<V *>(at + off0 * (int)sizeof(T)) = y0;
                    *reinterpret_cast<V *>(at + off1 * (int)sizeof(T)) = y1;
                } else if constexpr (KV == Kv::kE4m3) {
                    const float scale = K == 1 ? r.k_inv_scale : r.v_inv_scale;
                    *reinterpret_cast<uint32_t *>(at + off0) = e4m3x4(x, scale);
                    *reinterpret_cast<uint32_t *>(at + off1) = e4m3x4(x + 4, scale);
                } else {
                    float m = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
#pragma unroll
                    for (int off = kLanes / 2; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(group_mask, m, off));
                    float scale;
                    if constexpr (INTER) {
                        *reinterpret_cast<uint32_t *>(at + l * 4) = i4_word(x, m, scale);
                    } else {
                        scale = m > 0.f ? __fdiv_rn(m, 7.f) : 0.f;
                        store_i4_halves(at, x, m > 0.f ? __fdiv_rn(7.f, m) : 0.f, off0, off1, group_mask);
                    }
                    if (l == 0) (K == 1 ? r.k_scales : r.v_scales)[row0 + (long long)k * kGroups * kPage] = scale;
                }
            }
        };
        while (h < h_end) {
            if (kind == 0) rows(std::integral_constant<int, 0>());
            else if (okay && kind == 1) rows(std::integral_constant<int, 1>());
            else if (okay) rows(std::integral_constant<int, 2>());
            h = min(h + kRopeRows * kGroups, seg_end);
            src += kRopeRows * kGroups * kRowBytes;
            if (h < h_end) {
                if (h == seg_end) aim();
                load();
            }
        }
    }
    advance_lens_when_last(a, pl);
}

template <typename T, int D, Kv KV, bool INTER>
arb_status launch_one(Ctx *ctx, const RopeArgs &r, int grid, cudaStream_t stream) {
    const size_t smem = sizeof(int) * (3 * (size_t)r.a.batch + 1);
    const cudaError_t err = launch_pdl(rope_append_kernel<T, D, KV, INTER>, dim3(grid), dim3(kAppendThreads), smem, stream, r);
    ctx->launches++;
    return err == cudaSuccess ? ARB_OK : ARB_ERR_CUDA;
}

template <typename T, int D, Kv KV>
arb_status launch_pairing(Ctx *ctx, const RopeArgs &r, bool interleaved, int grid, cudaStream_t stream) {
    return interleaved ? launch_one<T, D, KV, true>(ctx, r, grid, stream) : launch_one<T, D, KV, false>(ctx, r, grid, stream);
}

template <Kv KV>
arb_status launch_typed(Ctx *ctx, const RopeArgs &r, const arb_attn_params &p, bool interleaved, int grid, cudaStream_t stream) {
    if (p.dtype == ARB_BF16) {
        return p.head_dim == 128 ? launch_pairing<__nv_bfloat16, 128, KV>(ctx, r, interleaved, grid, stream)
                                 : launch_pairing<__nv_bfloat16, 64, KV>(ctx, r, interleaved, grid, stream);
    }
    return p.head_dim == 128 ? launch_pairing<float, 128, KV>(ctx, r, interleaved, grid, stream)
                             : launch_pairing<float, 64, KV>(ctx, r, interleaved, grid, stream);
}

}  // namespace

arb_status launch_rope_append(Ctx *ctx, const arb_attn_params &p, const arb_rope_params &rope, int total_new, const void *q,
                              const void *k_new, const void *v_new, RopeCache cache, float k_inv_scale, float v_inv_scale,
                              const int32_t *block_table, int32_t *seq_lens, const int32_t *new_lens, int update_lens,
                              void *q_out, void *k_pages, void *v_pages, float *k_scales, float *v_scales, cudaStream_t stream) {
    const int esz = p.dtype == ARB_BF16 ? 2 : 4, D = p.head_dim;
    RopeArgs r = {};
    r.a.k_new = static_cast<const char *>(k_new);
    r.a.v_new = static_cast<const char *>(v_new);
    r.a.k_pages = static_cast<char *>(k_pages);
    r.a.v_pages = static_cast<char *>(v_pages);
    r.a.block_table = block_table;
    r.a.seq_lens = seq_lens;
    r.a.new_lens = new_lens;
    r.a.status = ctx->status;
    r.a.batch = p.batch;
    r.a.Hkv = p.num_kv_heads;
    r.a.num_pages = p.num_pages;
    r.a.max_pages = p.max_pages_per_seq;
    r.a.total_new = total_new;
    r.a.update_lens = update_lens;
    r.a.done_counter = ctx->rot + (size_t)kRotSets * kRotCounters + kRotSets + 3;
    r.q = static_cast<const char *>(q);
    r.q_out = static_cast<char *>(q_out);
    r.q_weight = rope.q_weight;
    r.k_weight = rope.k_weight;
    r.inv_freq = rope.inv_freq;
    r.positions = rope.positions;
    r.q_stride = (rope.q_stride ? rope.q_stride : (long long)p.num_q_heads * D) * esz;
    r.k_stride = (rope.k_stride ? rope.k_stride : (long long)p.num_kv_heads * D) * esz;
    r.v_stride = (rope.v_stride ? rope.v_stride : (long long)p.num_kv_heads * D) * esz;
    r.k_scales = k_scales;
    r.v_scales = v_scales;
    r.k_inv_scale = k_inv_scale;
    r.v_inv_scale = v_inv_scale;
    r.eps = rope.eps;
    r.Hq = p.num_q_heads;
    r.rot = rope.rot_dim;
    // A warp takes a row per lane group in a small call, and in a large one so many heads of a token that eight shares remain
    // for every resident warp: fewer and larger ones leave warps idle at the end, smaller ones work the angles out more often.
    const int heads = p.num_q_heads + 2 * p.num_kv_heads, groups = 256 / D;
    const long long resident = (long long)ctx->num_sms * kRopeCtas * (kAppendThreads / 32), rows = (long long)total_new * heads;
    const int batch = kRopeRows * groups;
    const long long share = (rows / (8 * resident) + batch) / batch * batch;
    // (and the shares of a token alike: a warp that strides through the units by an even number meets the same one every time)
    const int parts = (int)(rows <= resident * groups ? heads : (heads + share - 1) / share), most = (heads + parts - 1) / parts;
    r.heads_per_unit = (most + groups - 1) / groups * groups;
    r.units_per_token = (heads + r.heads_per_unit - 1) / r.heads_per_unit;
    const long long want = ((long long)total_new * r.units_per_token * 32 + kAppendThreads - 1) / kAppendThreads,
                    cap = (long long)ctx->num_sms * kRopeCtas;
    const int grid = (int)(want < 1 ? 1 : want > cap ? cap : want);
    const bool inter = rope.interleaved != 0;
    switch (cache) {
        case RopeCache::kSame: return launch_typed<Kv::kSame>(ctx, r, p, inter, grid, stream);
        case RopeCache::kE4m3: return launch_typed<Kv::kE4m3>(ctx, r, p, inter, grid, stream);
        default: return launch_pairing<__nv_bfloat16, 128, Kv::kI4>(ctx, r, inter, grid, stream);
    }
}

}  // namespace arb
