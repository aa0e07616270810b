// prompt.cuh -- the prompt's attention as its kernels see it.
#pragma once

#include "serve.cuh"

#include <math.h>

namespace gkv {
namespace serve {

// A launch with few blocks splits each block's keys into parts that run beside
// one another and leave O, M and Z in the workspace; a second launch joins them
// in order.  Most parts kept at once: two a SM (tcgen05, one CTA resident), four
// a SM (fp32, whose parts are a quarter of the rows and two CTAs are resident).
constexpr int kSms = 152, kPartsTc = 2 * kSms, kPartsF32 = 4 * kSms;
constexpr int kRowsTc = 256, kRowsF32 = 64;        // rows of a block
constexpr int kKeysF32 = 64;                       // keys of a tile
__host__ __device__ constexpr int keys_tc(int d) { return d == 64 ? 96 : 128; }

struct PromptArgs {
    const void *q, *k, *v;
    void *out;
    float *lse;
    const int32_t *cu_q, *cu_k;
    int n_seqs, G, Hq;
    int64_t n_q, n_k, q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;
    float scale;                   // 1 / sqrt(d)
    int *status;
    int *disorder;                 // above kScanSeqs sequences: whether cu_q's words run backwards or past n_q anywhere
    float *part;                   // partial results
    int split;                     // most parts of a block's keys (set by the launchers)
};

// The rows of a sequence from its cu words; false when they do not fit.
__device__ __forceinline__ bool bounds_fit(const PromptArgs &a, int cq0, int cq1, int ck0, int ck1, int64_t &q0, int64_t &nq,
                                           int64_t &k0, int64_t &nk) {
    q0 = cq0;
    nq = (int64_t)cq1 - q0;
    k0 = ck0;
    nk = (int64_t)ck1 - k0;
    return q0 >= 0 && nq >= 0 && q0 + nq <= a.n_q && k0 >= 0 && nk >= 0 && k0 + nk <= a.n_k;
}
__device__ __forceinline__ bool seq_bounds(const PromptArgs &a, int s, int64_t &q0, int64_t &nq, int64_t &k0, int64_t &nk) {
    return bounds_fit(a, a.cu_q[s], a.cu_q[s + 1], a.cu_k[s], a.cu_k[s + 1], q0, nq, k0, nk);
}

// Work slots of `tok` queries: sequence s owns the slots from cu_q[s] / tok + s
// on, which is room for its ceil(nq / tok) blocks whatever the lengths (the
// floors of two bounds nq apart differ by at least floor(nq / tok), and one
// more slot a sequence is left), so n_q / tok + n_seqs slots cover every
// packing without a pass over the lengths.
// 32-bit arithmetic: row counts are below 2^31, and the launchers keep the slots there too.
__host__ __device__ __forceinline__ int64_t prompt_slots(int64_t n_q, int n_seqs, int tok) {
    return (int64_t)((uint32_t)n_q / (uint32_t)tok) + n_seqs;
}
// How a block finds its sequence and sees that the query bounds ascend: below kLaneSeqs sequences with a bound a lane,
// up to kScanSeqs 32 bounds a step, beyond them by halves, and a launch of its own looks at the order.  (32 / 8 heads
// of 128: 40 sequences of 4000 tokens 41.0 us by steps, 43.8 by halves; 200 of 9000 138.9 and 133.1.)
constexpr int kLaneSeqs = 32, kScanSeqs = 64;
__device__ __forceinline__ bool ascend(int lo, int hi, int64_t n) { return lo >= 0 && lo <= hi && hi <= n; }

// The sequence of a slot where cu_q's words do not ascend, -1 for none.  A sequence is left out when its own do
// not, or when it begins below the end of an earlier one whose own do; what is left owns its rows alone.  One that
// is left out takes that end for its start, so the starts ascend and the count of them up to the slot still finds
// the owner, 32 sequences a step.  A call, so that it costs the callers no registers.
static __device__ __noinline__ int slot_owner_disordered(const int32_t *cu_q, int n_seqs, int64_t n_q, int slot, int tok) {
    const int lane = threadIdx.x & 31;
    int end = 0, found = -1;                             // end: the largest so far
    for (int s0 = 0; s0 < n_seqs; s0 += 32) {
        const int i = s0 + lane;
        const bool in = i < n_seqs;
        const int lo = in ? cu_q[i] : 0, hi = in ? cu_q[i + 1] : 0;
        const bool fits = in && ascend(lo, hi, n_q);
        int upto = fits ? max(hi, end) : end;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto = max(upto, v);
        }
        int before = __shfl_up_sync(0xffffffffu, upto, 1);
        if (lane == 0) before = end;
        const bool own = fits && lo >= before;
        const unsigned up = __ballot_sync(0xffffffffu, in && (own ? lo : before) / tok + i <= slot);
        if (up) {
            const int last = 31 - __clz(up);
            found = __shfl_sync(0xffffffffu, own, last) ? s0 + last : -1;
        }
        if (up != 0xffffffffu) break;
        end = __shfl_sync(0xffffffffu, upto, 31);
    }
    return found;
}

// The sequence of a slot and its rows; false when its cu words do not fit.  Whole warps call it.
__device__ __forceinline__ bool slot_rows(const PromptArgs &a, int slot, int tok, int &s, int64_t &q0, int64_t &nq, int64_t &k0,
                                          int64_t &nk) {
    bool owned = true;
    if (a.n_seqs < kLaneSeqs) {                          // a lane a bound: one round of loads instead of a search
        const int lane = threadIdx.x & 31;
        const int cq = lane <= a.n_seqs ? a.cu_q[lane] : 0, ck = lane <= a.n_seqs ? a.cu_k[lane] : 0;
        const int next = __shfl_down_sync(0xffffffffu, cq, 1);
        s = __all_sync(0xffffffffu, lane >= a.n_seqs || ascend(cq, next, a.n_q))
                ? max(0, __popc(__ballot_sync(0xffffffffu, lane < a.n_seqs && cq / tok + lane <= slot)) - 1)
                : slot_owner_disordered(a.cu_q, a.n_seqs, a.n_q, slot, tok);
        owned = s >= 0;
        s = max(s, 0);
        return bounds_fit(a, __shfl_sync(0xffffffffu, cq, s), __shfl_sync(0xffffffffu, cq, s + 1),
                          __shfl_sync(0xffffffffu, ck, s), __shfl_sync(0xffffffffu, ck, s + 1), q0, nq, k0, nk) && owned;
    }
    bool fine;
    if (a.n_seqs <= kScanSeqs) {
        bool mine = true;
        int up = 0;
#pragma unroll 4
        for (int s0 = 0; s0 < a.n_seqs; s0 += 32) {
            const int i = s0 + (threadIdx.x & 31);
            const bool in = i < a.n_seqs;
            const int lo = in ? a.cu_q[i] : 0, next = in ? a.cu_q[i + 1] : 0;
            mine = mine && (!in || ascend(lo, next, a.n_q));
            // lo / tok + i <= slot
            up += __popc(__ballot_sync(0xffffffffu, in && i <= slot && (uint32_t)lo < (uint32_t)(slot - i + 1) * (uint32_t)tok));
        }
        fine = __all_sync(0xffffffffu, mine);
        s = max(up - 1, 0);
    } else {
        fine = *a.disorder == 0;                         // on its way beside the search's first words
        int hi = a.n_seqs;
        s = 0;
        while (hi - s > 1) {
            const int mid = (s + hi) >> 1;
            if (a.cu_q[mid] / tok + mid <= slot) s = mid; else hi = mid;
        }
    }
    if (!fine) {
        s = slot_owner_disordered(a.cu_q, a.n_seqs, a.n_q, slot, tok);
        owned = s >= 0;
        s = max(s, 0);
    }
    return seq_bounds(a, s, q0, nq, k0, nk) && owned;
}

// Flags the sequences whose cu words do not fit (one block of a launch calls it).
__device__ __forceinline__ void check_bounds(const PromptArgs &a) {
    for (int s = threadIdx.x; s < a.n_seqs; s += blockDim.x) {
        int64_t q0, nq, k0, nk;
        if (!seq_bounds(a, s, q0, nq, k0, nk)) atomicOr(a.status, kStRange);
    }
}

// Key tiles of a part at least: what joining costs (about 4 us) against a tile
// (about 1 us for 128 keys on tcgen05, 6 us for 64 on CUDA cores).
constexpr int kLeastF32 = 1;
__host__ __device__ constexpr int least_tc(int d) { return 512 / keys_tc(d); }
// Parts of a block of n key tiles when a launch splits blocks `split` ways.
__host__ __device__ __forceinline__ int parts_of(int n, int split, int least) {
    const int most = n / least;
    return most < 1 ? 1 : most < split ? most : split;
}
// The first key tile of part p of np, floor(p n / np) in 32 bits (p <= np <= kPartsF32).
__device__ __forceinline__ int part_first(int n, int np, int p) { return p * (n / np) + p * (n % np) / np; }
// Floats of a part: 4-channel groups of the sums (by row or by group), then the
// rows' maxima (base 2) and weight sums.
__host__ __device__ constexpr size_t part_floats(int rows, int d) { return (size_t)rows * (d + 2); }

// What a row's sums are multiplied by, and its lse, from its reference (base 2) and its weights' sum: 0 and -inf where it
// saw no key, NaN where a weight was NaN or (tcgen05) none was in range.
__device__ __forceinline__ float row_scale(float m, float z) { return z > 0.f ? 1.f / z : m == -INFINITY ? 0.f : NAN; }
__device__ __forceinline__ float row_lse(float m, float z) {
    return z == 0.f && m == -INFINITY ? m : z > 0.f ? (m + log2f(z)) * 0.6931471805599453f : NAN;
}

// Joins the parts of a split launch of the tcgen05 kernel (sums [d / 4][rows])
// or of the fp32 kernel ([rows][d / 4]).
cudaError_t launch_prompt_join(const PromptArgs &a, int d, int dtype, bool tc_parts, cudaStream_t s);

// bf16 on tcgen05; cudaErrorNotSupported when a tensor's strides have no tensor map.
cudaError_t launch_prompt_tc(const PromptArgs &a, int d, cudaStream_t s);
// fp32, and bf16 tensors that launch_prompt_tc does not take.
cudaError_t launch_prompt_f32(const PromptArgs &a, int d, int dtype, cudaStream_t s);

}  // namespace serve
}  // namespace gkv
