// What the cache-writing kernels share: the plan every CTA derives from the lengths, the place of a row in the pools, the
// length update by the CTA that finishes last, and the two quantised formats' encoders.
#pragma once

#include "arb_common.cuh"

namespace arb {

namespace {

constexpr int kAppendThreads = 256;

struct AppendArgs {
    const char *k_new, *v_new;
    char *k_pages, *v_pages;
    const int32_t *block_table;
    int32_t *seq_lens;
    const int32_t *new_lens;
    uint32_t *status;
    int batch, Hkv, num_pages, max_pages;
    int row_bytes;   // D * element size: bytes of one (token, kv head) row
    int total_new;
    int update_lens;     // seq_lens += new_lens once every CTA has placed its rows
    int *done_counter;   // CTAs of this call that have; zero between calls
};

// The tables every CTA derives, in shared memory.
struct AppendPlan {
    int *pref;    // [B + 1] new rows before sequence b; at most total_new, whatever the lengths on the device add up to
    int *okay;    // [B] the sequence's new tokens may be written: they fit its table row, its pages exist, its rows are there
    int *start;   // [B] tokens it holds
};

// a + b, at most `most`; both lie in 0 .. most
__device__ __forceinline__ int capped_sum(int a, int b, int most) { return (int)min((unsigned)a + (unsigned)b, (unsigned)most); }

__device__ __forceinline__ AppendPlan append_plan(const AppendArgs &a, int *tables) {
    const int tid = threadIdx.x, lane = tid & 31, B = a.batch;
    const AppendPlan pl = {tables, tables + B + 1, tables + 2 * B + 1};
    const int behind = a.total_new + (a.total_new < INT32_MAX);   // where the sums stop: one row behind the last
    if (tid == 0) pl.pref[0] = 0;
    // as many lanes per sequence as the block has to spare, at most a warp: each looks at every g-th of its pages
    int g = 32;
    while (g > 1 && kAppendThreads / g < B) g >>= 1;
    const int mine = tid & (g - 1);
    for (int b0 = 0; b0 < B; b0 += kAppendThreads / g) {   // (uniform: the lanes of a sequence meet in shuffles)
        const int b = b0 + tid / g;
        const int n = b < B ? a.new_lens[b] : 0, L = b < B ? a.seq_lens[b] : 0;
        uint32_t bad = 0;
        if (n != 0) {
            if (n < 0 || L < 0 || (long long)L + n > (long long)a.max_pages * kPage) {
                bad = ARB_DEV_BAD_SEQ_LEN;
            } else {
                const int32_t *row = a.block_table + (size_t)b * a.max_pages;
#pragma unroll 4
                for (int pg = L / kPage + mine; pg <= (L + n - 1) / kPage; pg += g)
                    if ((unsigned)__ldg(row + pg) >= (unsigned)a.num_pages) bad = ARB_DEV_BAD_PAGE;
            }
        }
        for (int off = g >> 1; off >= 1; off >>= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, off);
        if (mine == 0 && b < B) {
            if (bad && blockIdx.x == 0) atomicOr(a.status, bad);
            pl.okay[b] = bad == 0;
            pl.start[b] = L;
            pl.pref[b + 1] = n > 0 ? min(n, behind) : 0;
        }
    }
    __syncthreads();
    if (tid < 32) {
        int carry = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const int b = b0 + lane;
            const int n = b < B ? pl.pref[b + 1] : 0;
            int v = n;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int t = __shfl_up_sync(0xffffffffu, v, off);
                if (lane >= off) v = capped_sum(v, t, behind);
            }
            v = capped_sum(v, carry, behind);
            if (b < B) {
                if (n > 0 && v > a.total_new) {   // some of its rows, or all, are not there
                    if (blockIdx.x == 0) atomicOr(a.status, (uint32_t)ARB_DEV_BAD_SEQ_LEN);
                    pl.okay[b] = 0;
                }
                pl.pref[b + 1] = min(v, a.total_new);
            }
            carry = __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
    return pl;
}

// New row r (token-major, a token's kv heads adjacent) -> its row in the pools, or -1 if its sequence is left alone.
__device__ __forceinline__ long long append_row(const AppendArgs &a, const AppendPlan &pl, unsigned r) {
    const int tok = (int)(r / (unsigned)a.Hkv), h = (int)r - tok * a.Hkv;
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.pref[mid] <= tok) lo = mid; else hi = mid;
    }
    if (!pl.okay[lo]) return -1;
    const int pos = pl.start[lo] + (tok - pl.pref[lo]);
    const int page = a.block_table[(size_t)lo * a.max_pages + pos / kPage];
    const long long row = ((long long)page * a.Hkv + h) * kPage + pos % kPage;
    return ARB_IN_RANGE(a.status, row, (long long)a.num_pages * a.Hkv * kPage) ? row : -1;
}

constexpr int kRowsInFlight = 4;   // rows a thread loads before it stores the first

// The lengths move forward inside the append kernel: every CTA reads the old lengths for the rows it places, so
// the CTA that finishes last (a counter tells it) adds new_lens, and leaves the counter at zero for the next call.
// The plan holds this CTA's copy of the per-sequence checks, taken from the old lengths.
__device__ __forceinline__ void advance_lens_when_last(const AppendArgs &a, const AppendPlan &pl) {
    if (!a.update_lens) return;
    __shared__ int is_last;
    __syncthreads();   // all rows of this CTA are placed, all its reads of seq_lens are done
    if (threadIdx.x == 0) {
        __threadfence();
        is_last = atomicAdd(a.done_counter, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!is_last) return;
    for (int b = threadIdx.x; b < a.batch; b += kAppendThreads) {
        const int n = a.new_lens[b];
        if (n > 0 && pl.okay[b]) a.seq_lens[b] = pl.start[b] + n;
    }
    if (threadIdx.x == 0) *a.done_counter = 0;
}

// two values -> two E4M3 codes; lo lands in the low byte
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Eight values of a row whose largest magnitude is m -> the row's scale and one word of the 4-bit format.
__device__ __forceinline__ uint32_t i4_word(const float (&x)[8], float m, float &scale) {
    scale = m > 0.f ? __fdiv_rn(m, 7.f) : 0.f;
    const float inv = m > 0.f ? __fdiv_rn(7.f, m) : 0.f;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = max(-7, min(7, __float2int_rn(__fmul_rn(x[j], inv))));
        word |= (uint32_t)(c + 8) << (4 * ((j >> 1) + 4 * (j & 1)));
    }
    return word;
}

}  // namespace

}  // namespace arb
