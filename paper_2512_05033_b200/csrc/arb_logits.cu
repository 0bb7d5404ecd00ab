// From logits to the next token (arb_logits, see arb.h for the formulas): penalties for tokens a row's history holds, biases,
// temperature, an allowed-token mask, the arg max of x + noise and its log-probability.
//
// One pass over memory: a row is cut into pieces of kPiece tokens, and its pieces into as many runs as keep every resident CTA
// busy, one CTA a run.  Few tokens of a vocabulary are in a history or a list of biases, so these are gone through on their own,
// for a window of up to kWindow pieces: the CTA marks each in a bitmap in shared memory; the number of bits before its own
// is a special token's slot, whichever thread comes first; a second look at the lists counts occurrences (integer atomics: any
// order gives the same), and the slots get their penalties and biases (each bias added by any thread, unless a token is
// listed more than once: the sums of such tokens are taken by the warps, each for its own slots, which go through the list in order).  The stream over the pieces, which does
// temperature, mask, noise, maximum and sum, takes a marked token's value from its slot.  A window with more special tokens than
// slots is done a piece at a time.  A history is read by every CTA of its row, from L2.  The runs' records (maximum, sum,
// best) go to the workspace; the CTA of a row that arrives last at the row's counter puts them together, run by run in order.
//
// What bounds it is instruction issue and the chain of steps before a window's stream.  64 rows of 128001 bf16 logits (49 MB; a
// plain bf16 -> fp32 copy of them takes 24 us): 15 us without options, 26 with a history of up to 4096 tokens, 18 with 64 biases, 34 with
// a history, biases, mask, temperature and noise (84 MB).  Special tokens found piece by piece, in a list in order of arrival and a counter
// per token, 47 us; windows of 4 pieces instead of 8 39; a count and a bias looked up for every token 53; the special tokens in a kernel of
// their own 61; a CTA per piece instead of a run of pieces 19 us without and 56 with everything (every CTA's reduction, fence and arrival
// cost 7 us).  Pieces of 4096 tokens 36, of 1024 35; three CTAs per SM 40, five 34.  No difference: the first tokens of the
// history read ahead of its length and kept in registers, 8 in flight instead of 4.
//
// Rows of an odd vocabulary start at any element, so groups of four tokens are cut at multiples of four of the flat element
// index: full groups are aligned in every array whose rows lie alike, a row's first and last group are read one by one.
#include <type_traits>

#include "arb_common.cuh"

namespace arb {

namespace {

constexpr int kLogitsThreads = 256;
constexpr int kLogitsCtas = 4;                              // resident CTAs of an SM
constexpr int kGroup = 4;                                   // tokens of a vector load
constexpr int kPer = 2;                                     // groups of a thread and piece
constexpr int kPiece = kLogitsThreads * kPer * kGroup;
constexpr int kAhead = 2;                                   // pieces asked into L2 ahead
constexpr int kCap = 4096;                                  // special tokens of a window, a piece's at least
constexpr int kWindow = 8;                                  // pieces whose special tokens are found together
constexpr int kHeld = 4;                                    // history tokens of a thread in flight
constexpr int kWalk = 4;                                    // entries of a lane in flight where a list is gone through in order
constexpr int kBiasOne = 1 << 24;                           // in a token's counter: occurrences in the history below, listed among the biases

struct Record {      // what a run leaves of a row: max and sum of exponentials of x, the best x + noise with its token and its x
    float m, l, best, best_x;
    int token;
    int pad[3];
};

struct LogitsArgs {
    arb_logits_params p;
    Record *records;     // [rows][runs]
    int *counters;
    uint32_t *status;    // of the bounds-check build
    int pieces;          // of a row
};

// asks [from, from + bytes) into L2, but for the ends that share a 16-byte piece with something else
__device__ __forceinline__ void prefetch_l2(const void *from, long long bytes) {
    const uintptr_t begin = (reinterpret_cast<uintptr_t>(from) + 15) & ~uintptr_t(15), end = (reinterpret_cast<uintptr_t>(from) + bytes) & ~uintptr_t(15);
    if (bytes > 0 && end > begin)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(begin), "r"((uint32_t)(end - begin)) : "memory");
}

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

// floats as unsigned integers of the same order; NaN is not among them
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float warp_max(float x) {
    const uint32_t u = __reduce_max_sync(0xffffffffu, ordered(x));
    return __uint_as_float(u ^ ((int)u < 0 ? 0x80000000u : 0xffffffffu));
}
// best, best_x and token of the warp's best candidate, in every lane
__device__ __forceinline__ void best_of_warp(Record &r) {
    const float best = warp_max(r.token < 0 ? -INFINITY : r.best + 0.0f);   // (-0 and 0 are a tie)
    const uint32_t token = __reduce_min_sync(0xffffffffu, r.token >= 0 && r.best == best ? (uint32_t)r.token : 0xffffffffu);
    const uint32_t who = __ballot_sync(0xffffffffu, r.token >= 0 && (uint32_t)r.token == token);
    r.best_x = __shfl_sync(0xffffffffu, r.best_x, who ? __ffs(who) - 1 : 0);
    r.best = best;
    r.token = (int)token;   // -1: nobody had one
}
// the records of a warp's lanes into one, in every lane
__device__ __forceinline__ void merge_warp(Record &r) {
    const float m = warp_max(r.m), base = m == -INFINITY ? 0.f : m;
    r.l *= __expf(r.m - base);
    r.m = m;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) r.l += __shfl_xor_sync(0xffffffffu, r.l, off);
    best_of_warp(r);
}

__device__ __forceinline__ void none_yet(Record &r) { r.m = -INFINITY; r.l = 0.f; r.best = -INFINITY; r.best_x = -INFINITY; r.token = -1; }

// A CTA's records into one, in every lane of warp 0; `of_warps` has a place for each warp.
template <int WARPS>
__device__ __forceinline__ void merge_block(Record &r, Record *of_warps) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    merge_warp(r);
    __syncthreads();   // (the records of the row before have been read)
    if (lane == 0) of_warps[warp] = r;
    __syncthreads();
    if (warp != 0) return;
    r = of_warps[lane & (WARPS - 1)];
    if (lane >= WARPS) none_yet(r);
    merge_warp(r);
}

// a group of elements, as they are and as floats
template <typename T> struct Group;
template <> struct Group<float> {
    float4 a;
    __device__ __forceinline__ void load(const float *p) { a = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void unpack(float (&x)[kGroup]) const { x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; }
};
template <> struct Group<__nv_bfloat16> {
    uint2 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void unpack(float (&x)[kGroup]) const {
        x[0] = __uint_as_float(a.x << 16); x[1] = __uint_as_float(a.x & 0xffff0000u);
        x[2] = __uint_as_float(a.y << 16); x[3] = __uint_as_float(a.y & 0xffff0000u);
    }
};

// x / t, correctly rounded.  With r = 1 / t correctly rounded and q = x r within a unit in the last place of the quotient,
// fma(fma(-q, t, x), r, q) is the correctly rounded quotient (Markstein, 1990), as long as nothing leaves the normal
// numbers: otherwise the division itself.
// (One element of N far from 1 sends them all the long way.)
__device__ __noinline__ float divided_slowly(float x, float t) { return __fdiv_rn(x, t); }
template <int N>
__device__ __forceinline__ void divide(float (&x)[N][kGroup], float t, float r) {
    bool plain = r != 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < kGroup; ++i) plain = plain && fabsf(x[k][i]) < 1e25f && fabsf(x[k][i]) > 1e-25f;
    if (plain) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                const float q = x[k][i] * r;
                x[k][i] = fmaf(fmaf(-q, t, x[k][i]), r, q);
            }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < kGroup; ++i) x[k][i] = divided_slowly(x[k][i], t);
    }
}

// The best of a group's four (y = x + noise) where it beats what the thread has.
__device__ __forceinline__ void best_of(Record &r, const float (&x)[kGroup], float y0, float y1, float y2, float y3, int t0) {
    const float top = fmaxf(fmaxf(y0, y1), fmaxf(y2, y3));   // (passes NaN over)
    if (top > r.best) {
        const int i = y0 == top ? 0 : y1 == top ? 1 : y2 == top ? 2 : 3;
        r.best = top;
        r.best_x = i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3];
        r.token = t0 + i;
    }
}

__device__ __forceinline__ bool in_window(int t, int first, unsigned tokens) { return (unsigned)t - (unsigned)first < tokens; }
// the slot of a marked token: the number of bits before its own
__device__ __forceinline__ int slot_at(const uint32_t *touched, const uint16_t *before, int at) {
    return before[at >> 5] + __popc(touched[at >> 5] & ((1u << (at & 31)) - 1u));
}

struct Window {
    const uint32_t *touched;
    const uint16_t *before;
    int first, lo;     // first token of the row in it; where its bits start
    unsigned tokens;
};

// Adds the n listed values of every slot in `twice` to its sum, in the order of the list: a warp takes its own slots, 32 entries
// at a time, and of those the entries of one slot one after the other.  Two rows, one with a list of 60000 tokens: 0.15 ms; with one of them
// twice 0.46 ms (a thread per entry that looks for its first and for its others: 424 ms), one token 60000 times 2.4 ms.  The room that sums
// and bits take and the code cost the batch with every option 1 us (33 -> 34).
__device__ __forceinline__ void add_in_order(const int32_t *tokens, const float *values, int n, const Window w, const uint32_t *twice, float *sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i0 = 0; i0 < n; i0 += 32 * kWalk) {
        int slot[kWalk];
#pragma unroll
        for (int k = 0; k < kWalk; ++k) slot[k] = i0 + 32 * k + lane < n ? __ldg(tokens + i0 + 32 * k + lane) : -1;
#pragma unroll
        for (int k = 0; k < kWalk; ++k) {
            const int t = slot[k];
            slot[k] = in_window(t, w.first, w.tokens) ? slot_at(w.touched, w.before, t - w.lo) : -1;
            if (slot[k] >= 0 && (slot[k] % (kLogitsThreads / 32) != warp || !(twice[slot[k] >> 5] >> (slot[k] & 31) & 1u))) slot[k] = -1;
        }
#pragma unroll
        for (int k = 0; k < kWalk; ++k) {
            if (!__any_sync(0xffffffffu, slot[k] >= 0)) continue;
            const float value = slot[k] >= 0 ? __ldg(values + i0 + 32 * k + lane) : 0.f;
            const uint32_t alike = __match_any_sync(0xffffffffu, slot[k]);
            const int rank = slot[k] >= 0 ? __popc(alike & ((1u << lane) - 1u)) : -1, most = __reduce_max_sync(0xffffffffu, rank);
            for (int r = 0; r <= most; ++r) {
                if (rank == r) sums[slot[k]] = __fadd_rn(sums[slot[k]], value);
                __syncwarp();
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLogitsThreads, kLogitsCtas)
logits_kernel(const LogitsArgs a) {
    constexpr int kPc = kPiece, PER = kPer, kWarps = kLogitsThreads / 32;
    constexpr int kWords = kWindow * kPc / 32, kOwn = kWords / kLogitsThreads;
    static_assert(kWindow * kPc <= 65536 && kCap >= kPc && kCap % (4 * kLogitsThreads) == 0 && kWords % kLogitsThreads == 0, "16 bits a token; cleared by fours; as many words for every thread");
    const arb_logits_params &p = a.p;
    extern __shared__ __align__(16) int counts[];         // [kCap] counters of the special tokens, then their x
    uint32_t *touched = reinterpret_cast<uint32_t *>(counts + kCap);          // [kWords] a bit per token of the window
    uint16_t *before = reinterpret_cast<uint16_t *>(touched + kWords);        // [kWords] bits set in the words before
    uint16_t *list = before + kWords;                                         // [kCap] the special tokens in their order
    float *xs = reinterpret_cast<float *>(counts);
    float *sums = reinterpret_cast<float *>(list + kCap);                     // [kCap] with biases: what a token that is listed more than once gets
    uint32_t *twice = reinterpret_cast<uint32_t *>(sums + kCap);              // [kCap / 32] with biases: a bit per slot of such a token
    __shared__ Record warp_rec[kWarps];
    __shared__ int warp_bits[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = p.vocab, row = blockIdx.y, runs = gridDim.x;
    const bool special = p.history || p.bias_offsets, wanted = p.tokens || p.logprobs;
    const T *x_in = static_cast<const T *>(p.logits) + row * (p.logits_stride ? p.logits_stride : (long long)V);
    // groups start where the logits' own alignment has them; the dense fp32 arrays' groups agree or are taken one by one
    const int skew = (int)((reinterpret_cast<uintptr_t>(x_in) / sizeof(T)) & (kGroup - 1));
    const int piece_begin = (int)((long long)a.pieces * blockIdx.x / runs), piece_end = (int)((long long)a.pieces * (blockIdx.x + 1) / runs);
    auto fetch = [&](int from, int to) {   // pieces into L2 (before the kernel ahead has ended, too: L2 holds what it then writes)
        const long long first = max(from * kPc - skew, 0), tokens = min((long long)to * kPc - skew, (long long)V) - first;
        prefetch_l2(x_in + first, tokens * (long long)sizeof(T));
        if (p.noise) prefetch_l2(p.noise + (size_t)row * V + first, tokens * 4);
    };
    let_successor_start();
    if (tid == 0) fetch(piece_begin, min(piece_begin + kAhead, piece_end));
    if (special) {   // all zero at the start of a window
#pragma unroll
        for (int i = 0; i < kCap / 4 / kLogitsThreads; ++i) reinterpret_cast<uint4 *>(counts)[i * kLogitsThreads + tid] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) touched[i * kLogitsThreads + tid] = 0;
        if (p.bias_offsets && tid < kCap / 32) twice[tid] = 0;
        __syncthreads();
    }
    wait_for_predecessor();
    const float temperature = p.temperature ? p.temperature[row] : 1.0f;
    const bool scaled = p.temperature && temperature > 0.f;
    const float per_temperature = temperature > 1e-6f && temperature < 1e6f ? __frcp_rn(temperature) : 0.f;
    const float *noise = p.noise && temperature > 0.f ? p.noise + (size_t)row * V : nullptr;
    float *out = p.out ? p.out + (size_t)row * V : nullptr;
    const uint32_t *mask = p.mask ? p.mask + (size_t)row * p.mask_stride : nullptr;
    const bool noise_alike = noise && (int)((reinterpret_cast<uintptr_t>(noise) / 4) & 3) == skew;
    const bool out_alike = out && (int)((reinterpret_cast<uintptr_t>(out) / 4) & 3) == skew;
    Record r;
    none_yet(r);

    int n_history = 0, b_begin = 0, b_end = 0;
    float repetition = 1.f, presence = 0.f, frequency = 0.f;
    if (p.history) {
        if (p.repetition) repetition = p.repetition[row];
        if (p.presence) presence = p.presence[row];
        if (p.frequency) frequency = p.frequency[row];
    }
    if (p.history) n_history = p.history_lens ? max(0, min(p.history_lens[row], p.history_stride)) : p.history_stride;
    if (p.bias_offsets) {
        b_begin = max(0, min(p.bias_offsets[row], p.bias_total));
        b_end = max(b_begin, min(p.bias_offsets[row + 1], p.bias_total));
    }
    const bool alike = (!noise || noise_alike) && (!out || out_alike);
    int window = kWindow;   // pieces
#pragma unroll 1
    for (int w_begin = piece_begin, w_end; w_begin < piece_end; w_begin = w_end) {
    w_end = min(w_begin + window, piece_end);
    const int w_lo = w_begin * kPc - skew;   // first token of the window (below 0: the row starts inside a group)

    // ---- the window's special tokens
    int n_listed = 0;
    if (special) {
        const int32_t *history = p.history + (size_t)row * p.history_stride;
        const int first = max(w_lo, 0);
        unsigned tokens_here;   // none where a row's skew leaves its last window behind the row
        auto here = [&](int t) { return in_window(t, first, tokens_here); };
        // f(t) for every token of a list that lies in the window, the loads of kHeld in flight together
        auto each = [&](const int32_t *tokens, int n, auto f) {
            for (int i0 = tid; i0 < n; i0 += kHeld * kLogitsThreads) {
                int t[kHeld];
#pragma unroll
                for (int k = 0; k < kHeld; ++k) t[k] = i0 + k * kLogitsThreads < n ? __ldg(tokens + i0 + k * kLogitsThreads) : -1;
#pragma unroll
                for (int k = 0; k < kHeld; ++k)
                    if (here(t[k])) f(t[k] - w_lo);
            }
        };
        auto mark = [&](int at) {
            if (ARB_IN_RANGE(a.status, at >> 5, kWords)) atomicOr(&touched[at >> 5], 1u << (at & 31));
        };
        auto slot_of = [&](int at) {
            const int slot = slot_at(touched, before, ARB_IN_RANGE(a.status, at >> 5, kWords) ? at : 0);
            return ARB_IN_RANGE(a.status, slot, n_listed) ? slot : 0;
        };
        for (;;) {
            tokens_here = (unsigned)max(min(w_end * kPc - skew, V) - first, 0);
            each(history, n_history, mark);
            each(p.bias_tokens + b_begin, b_end - b_begin, mark);
            __syncthreads();
            // a token's slot is the number of bits before its own
            uint32_t word[kOwn];
            int bits = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                word[i] = touched[tid * kOwn + i];
                bits += __popc(word[i]);
            }
            int upto = bits;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int other = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += other;
            }
            if (lane == 31) warp_bits[warp] = upto;
            __syncthreads();
            int at = upto - bits;
            n_listed = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const int n = warp_bits[w];
                at += w < warp ? n : 0;
                n_listed += n;
            }
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                before[tid * kOwn + i] = (uint16_t)at;
                at += __popc(word[i]);
            }
            if (n_listed <= kCap) break;
            // more than there is room for: a piece at a time from here on
            window = 1;
            w_end = w_begin + 1;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) touched[tid * kOwn + i] = 0;
            __syncthreads();
        }
        __syncthreads();
        each(history, n_history, [&](int at) {
            const int slot = slot_of(at);
            atomicAdd(&counts[slot], 1);
            list[slot] = (uint16_t)at;   // (whoever else writes it writes the same)
        });
        bool again = false;   // a token is listed more than once among the biases
        each(p.bias_tokens + b_begin, b_end - b_begin, [&](int at) {
            const int slot = slot_of(at);
            if (atomicOr(&counts[slot], kBiasOne) >= kBiasOne) {
                atomicOr(&twice[slot >> 5], 1u << (slot & 31));
                again = true;
            }
            list[slot] = (uint16_t)at;
        });
        again = __syncthreads_or(again);
        for (int i = tid; i < n_listed; i += kLogitsThreads) {
            const int c = counts[i] & (kBiasOne - 1);
            const int t = w_lo + list[i];
            float v = Elt<T>::to_float(x_in[ARB_IN_RANGE(a.status, t, V) ? t : 0]);
            if (c > 0) {
                v = v > 0.f ? __fdiv_rn(v, repetition) : __fmul_rn(v, repetition);
                v = __fsub_rn(v, presence);
                v = __fsub_rn(v, __fmul_rn(frequency, (float)c));
            }
            xs[i] = v;
            if (again) sums[i] = -0.0f;   // (what adds nothing to any value, a zero's sign included)
        }
        __syncthreads();
        auto repeated = [&](int slot) { return again && (twice[slot >> 5] >> (slot & 31) & 1u); };
        for (int i = b_begin + tid; i < b_end; i += kLogitsThreads) {
            const int t = __ldg(p.bias_tokens + i);
            if (!here(t)) continue;
            const int slot = slot_of(t - w_lo);
            if (!repeated(slot)) xs[slot] = __fadd_rn(xs[slot], __ldg(p.bias_values + i));
        }
        if (again) {   // (the same for the whole block)
            add_in_order(p.bias_tokens + b_begin, p.bias_values + b_begin, b_end - b_begin, Window{touched, before, first, w_lo, tokens_here}, twice, sums);
            __syncthreads();
            for (int i = tid; i < n_listed; i += kLogitsThreads)
                if (repeated(i)) xs[i] = __fadd_rn(xs[i], sums[i]);
        }
        if (p.bias_offsets) __syncthreads();
    }

#pragma unroll 1
    for (int piece = w_begin; piece < w_end; ++piece) {
    const int lo = piece * kPc - skew;
    if (tid == 0 && piece + kAhead < piece_end) fetch(piece + kAhead, piece + kAhead + 1);

    // ---- the stream, compiled twice: every group of the piece whole and alike in all arrays, or with a look at each.  What a row
    //      does not use costs a branch per piece, not an instruction per token.
    auto stream = [&](auto inner_c) {
        constexpr bool kInner = decltype(inner_c)::value;
        constexpr int kStep = kLogitsThreads * kGroup;
        auto whole = [&](int t0) { return kInner || (t0 >= 0 && t0 + kGroup <= V); };
        const int t_first = lo + tid * kGroup, w_last = (V - 1) >> 5;   // group k: kStep tokens on
        Group<T> raw[PER];
        Group<float> nz[PER];
        float x[PER][kGroup];
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (whole(t_first + k * kStep)) raw[k].load(x_in + t_first + k * kStep);
        if (noise) {
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (kInner || (noise_alike && whole(t_first + k * kStep))) nz[k].load(noise + t_first + k * kStep);
        }
        uint32_t hide[PER];   // of a group: tokens that are not allowed, or not there
#pragma unroll
        for (int k = 0; k < PER; ++k) hide[k] = 0;
        if (mask) {   // t0 may lie below 0 and the bits in two words
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int t0 = t_first + k * kStep, w = kInner ? t0 >> 5 : max(t0, 0) >> 5;
                const uint32_t w0 = __ldg(mask + (kInner ? w : min(w, w_last))), w1 = __ldg(mask + min(w + 1, w_last));
                hide[k] = ~(kInner || t0 >= 0 ? __funnelshift_r(w0, w1, t0 & 31) : w0 << -t0);
            }
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) raw[k].unpack(x[k]);
        if (!kInner) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int t0 = t_first + k * kStep;
                if (whole(t0)) continue;
#pragma unroll
                for (int i = 0; i < kGroup; ++i) {
                    const bool real = (unsigned)(t0 + i) < (unsigned)V;
                    x[k][i] = real ? Elt<T>::to_float(x_in[t0 + i]) : 0.f;
                    if (!real) hide[k] |= 1u << i;
                }
            }
        }
        if (special) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int at = t_first + k * kStep - w_lo;
                const uint32_t word = touched[at >> 5], those = word >> (at & 31);
                if (those & ((1u << kGroup) - 1u)) {
                    int slot = before[at >> 5] + __popc(word & ((1u << (at & 31)) - 1u));
#pragma unroll
                    for (int i = 0; i < kGroup; ++i)
                        if (those & (1u << i)) x[k][i] = xs[slot++];
                }
            }
        }
        if (scaled) divide(x, temperature, per_temperature);
        if (!kInner || mask) {
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                    if (hide[k] & (1u << i)) x[k][i] = -INFINITY;
        }
        if (out) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int t0 = t_first + k * kStep;
                if (kInner || (out_alike && whole(t0))) {
                    *reinterpret_cast<float4 *>(out + t0) = make_float4(x[k][0], x[k][1], x[k][2], x[k][3]);
                } else {
#pragma unroll
                    for (int i = 0; i < kGroup; ++i)
                        if ((unsigned)(t0 + i) < (unsigned)V) out[t0 + i] = x[k][i];
                }
            }
        }
        if (!wanted) return;
        float m = r.m;
#pragma unroll
        for (int k = 0; k < PER; ++k) m = fmaxf(fmaxf(fmaxf(m, x[k][0]), fmaxf(x[k][1], x[k][2])), x[k][3]);   // (passes NaN over)
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int i = 0; i < kGroup; ++i) l += __expf(x[k][i] - base);   // (scaled before the difference, the type's lowest value would overflow)
        r.l = r.l * __expf(r.m - base) + l;
        r.m = m;
        if (noise) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int t0 = t_first + k * kStep;
                float n[kGroup];
                nz[k].unpack(n);
                if (!kInner && !(noise_alike && whole(t0))) {
#pragma unroll
                    for (int i = 0; i < kGroup; ++i) n[i] = (unsigned)(t0 + i) < (unsigned)V ? noise[t0 + i] : 0.f;
                }
                best_of(r, x[k], __fadd_rn(x[k][0], n[0]), __fadd_rn(x[k][1], n[1]), __fadd_rn(x[k][2], n[2]), __fadd_rn(x[k][3], n[3]), t0);
            }
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k) best_of(r, x[k], x[k][0], x[k][1], x[k][2], x[k][3], t_first + k * kStep);
        }
    };
    if (alike && lo >= 0 && lo + kPc <= V) stream(std::true_type());
    else stream(std::false_type());

    }
    if (special && w_end < piece_end) {
        __syncthreads();   // (everyone has read what it needs of the window)
        for (int i = tid; i < n_listed; i += kLogitsThreads) counts[i] = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) touched[tid * kOwn + i] = 0;
        if (p.bias_offsets && tid < kCap / 32) twice[tid] = 0;
        __syncthreads();
    }
    }
    if (!wanted) return;
    merge_block<kWarps>(r, warp_rec);
    if (warp != 0) return;
    if (runs > 1) {
        Record *records = a.records + (size_t)row * runs;
        bool last = false;
        if (lane == 0) {
            records[blockIdx.x] = r;
            __threadfence();
            last = atomicAdd(&a.counters[row], 1) == runs - 1;
            if (last) a.counters[row] = 0;   // every run has arrived: ready for the next call
            __threadfence();
        }
        if (!__shfl_sync(0xffffffffu, (int)last, 0)) return;
        none_yet(r);
        for (int i = lane; i < runs; i += 32) {
            const float4 f = __ldcg(reinterpret_cast<const float4 *>(records + i));
            Record o;
            o.m = f.x; o.l = f.y; o.best = f.z; o.best_x = f.w;
            o.token = __ldcg(&records[i].token);
            merge(r, o);
        }
        merge_warp(r);
    }
    if (lane == 0) {
        if (p.tokens) p.tokens[row] = r.token;
        if (p.logprobs) p.logprobs[row] = r.token < 0 && r.l == r.l ? -INFINITY : r.best_x - r.m - __logf(r.l);
    }
}

template <typename T>
arb_status launch_typed(Ctx *ctx, LogitsArgs a, cudaStream_t stream) {
    constexpr int kSmem = kCap * (int)(sizeof(int) + sizeof(uint16_t)) + kWindow * kPiece / 32 * (int)(sizeof(uint32_t) + sizeof(uint16_t));   // of a call with history or biases
    constexpr int kSmemBiases = kCap * (int)sizeof(float) + kCap / 8;                                                                       // ... and what biases need besides
    static_assert(kSmem + kSmemBiases <= 48 * 1024 && kSmem % 4 == 0, "no opt-in needed");
    static_assert(kCap / 32 <= kLogitsThreads, "a word of a thread");
    const int smem = a.p.bias_offsets ? kSmem + kSmemBiases : a.p.history ? kSmem : 0;
    a.pieces = (int)(((long long)a.p.vocab + kGroup - 1 + kPiece - 1) / kPiece);   // (a row may start up to three elements into a group)
    const long long share = (long long)ctx->num_sms * kLogitsCtas / a.p.rows;
    const int runs = (int)(share < 1 ? 1 : share < a.pieces ? share : a.pieces);   // of a row
    const bool records = runs > 1 && (a.p.tokens || a.p.logprobs);   // a row of one run, or whose token nobody wants, leaves none
    if (records && (size_t)a.p.rows * runs * sizeof(Record) > ctx->chunk_ws_bytes) return ARB_ERR_WORKSPACE;
    const cudaError_t err = launch_pdl(logits_kernel<T>, dim3(runs, a.p.rows), dim3(kLogitsThreads), smem, stream, a);
    ctx->launches++;
    return err == cudaSuccess ? ARB_OK : ARB_ERR_CUDA;
}

}  // namespace

arb_status launch_logits(Ctx *ctx, const arb_logits_params &p, cudaStream_t stream) {
    LogitsArgs a;
    a.p = p;
    a.records = reinterpret_cast<Record *>(ctx->chunk_ws);
    a.counters = ctx->counters;
    a.status = ctx->status;
    return p.dtype == ARB_BF16 ? launch_typed<__nv_bfloat16>(ctx, a, stream) : launch_typed<float>(ctx, a, stream);
}

}  // namespace arb
