// shared_plan.cuh -- the plan of the attention over a shared prefix: the blocks of
// rows of all slots, and how many pieces each one's keys are cut into, so that the
// pieces fill the SMs and the longest one is short.
#pragma once

#include "shared.cuh"

#include <limits.h>

namespace gkv {
namespace serve {

constexpr int kPlanBlocks = 512;           // blocks that are kept in shared memory too
// What a key tile costs: of one row tile, and (SharedArgs::two) of two.  Measured (shared_tc.cu) 1.68 and 1.43 times as much
// for bf16 of d = 128, in L2 and from HBM, 1.55 to 1.8 for the others.
constexpr int kPlanOne = 4, kPlanTwoWide = 6, kPlanTwo = 7;
constexpr int kPlanSearch = 64;            // blocks up to which lengths are compared, for as many pieces as run at once

template <int T>
struct PlanSmem {
    int w_max[T / 32], w_sum[T / 32], lo[T], n[T], rb[T], np[T], first[T];
    int used[T / 32];
    long long total[T / 32];
    int4 blk[kPlanBlocks];
};

template <typename Op>
__device__ __forceinline__ int plan_scan(int v, Op op) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v = op(v, u);
    }
    return v;
}

// By a block of T threads, behind the wait for the launch before.
template <int T>
__device__ __noinline__ void make_plan(const SharedArgs &a, PlanSmem<T> &sm) {
    constexpr int W = T / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.c.G, keys = a.keys, most = a.pieces;
    auto larger = [](int x, int y) { return max(x, y); };
    auto sum = [](int x, int y) { return x + y; };
    for (int b = tid; b < a.B; b += T) a.plan.req[b] = make_int2(-1, 0);
    __syncthreads();

    // ---- the slots' requests.  A slot is left out when its words do not ascend within the batch, or when it
    // begins below the end of an earlier one whose own do; the others have their requests to themselves.
    int end = 0, base = 0;                               // largest end, blocks of rows so far
    long long total = 0;                                 // what all tiles cost; blocks that have any
    int used = 0;
    auto cost = [&](int4 k) { return (k.z > a.tok / 2 ? a.two : kPlanOne) * ((k.w + keys - 1) / keys); };
    for (int p0 = 0; p0 < a.P; p0 += T) {
        const int p = p0 + tid;
        int lo = 0, hi = 0;
        if (p < a.P) {
            lo = a.cu ? a.cu[p] : 0;
            hi = a.cu ? a.cu[p + 1] : a.B;
        }
        const bool fits = lo >= 0 && lo <= hi && hi <= a.B;
        const int upto = plan_scan(fits ? hi : 0, larger);
        if (lane == 31) sm.w_max[warp] = upto;
        __syncthreads();
        int before = __shfl_up_sync(0xffffffffu, upto, 1);
        if (lane == 0) before = 0;
        before = max(before, end);
        for (int w = 0; w < W; w++) {
            if (w < warp) before = max(before, sm.w_max[w]);
            end = max(end, sm.w_max[w]);
        }
        const bool owned = p < a.P && fits && (lo >= before || lo == hi);
        if (p < a.P && !owned) atomicOr(a.status, kStRange);
        const int n = owned ? hi - lo : 0, rb = (n + a.tok - 1) / a.tok;
        const int incl = plan_scan(rb, sum);
        if (lane == 31) sm.w_sum[warp] = incl;
        __syncthreads();
        int first = base + incl - rb;
        for (int w = 0; w < W; w++) {
            if (w < warp) first += sm.w_sum[w];
            base += sm.w_sum[w];
        }
        sm.lo[tid] = lo;
        sm.n[tid] = n;
        sm.rb[tid] = first;
        __syncthreads();
        for (int s = warp; s < min(T, a.P - p0); s += W) {
            const int l0 = sm.lo[s], ns = sm.n[s], r0 = sm.rb[s];
            for (int i = lane; i < ns; i += 32) a.plan.req[l0 + i] = make_int2(r0 + i / a.tok, i % a.tok);
            const int nb = (ns + a.tok - 1) / a.tok * G;
            for (int i = lane; i < nb; i += 32) {
                const int rb_i = i / G, g = i % G, len = a.lens[(int64_t)(p0 + s) * G + g];
                const int cap = a.c.page_size * a.c.max_pages, k = max(0, min(len, cap)), at = (r0 + rb_i) * G + g;
                if (len > cap) atomicOr(a.status, kStRange);
                const int4 w = make_int4(p0 + s, l0 + rb_i * a.tok, min(a.tok, ns - rb_i * a.tok), k);
                a.plan.blk[at] = w;
                if (at < kPlanBlocks) sm.blk[at] = w;
                const int t = cost(w);
                total += t;
                used += t > 0;
            }
        }
        __syncthreads();
    }
    const int blocks = base * G;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        used += __shfl_xor_sync(0xffffffffu, used, o);
    }
    if (lane == 0) {
        sm.total[warp] = total;
        sm.used[warp] = used;
    }
    __syncthreads();
    total = used = 0;
    for (int w = 0; w < W; w++) {
        total += sm.total[w];
        used += sm.used[w];
    }
    auto block = [&](int i) { return i < kPlanBlocks ? sm.blk[i] : a.plan.blk[i]; };

    // ---- the cost of a piece, the least that gives no more pieces than there is room for.  It lies between an even
    // share of all and what is sure to (sum of ceil(t / run) <= total / run + used); a candidate a thread.
    // (Room for more pieces than SMs, as slots without requests leave, is of no use to few blocks: a piece has its own
    // start of some ten tiles.)
    const int target = blocks <= kPlanSearch ? min(most, shared_at_once(keys == kShKeysTc)) : most;
    const int room = target - used;                      // at least half of the SMs, or twice the SMs
    const int share = (int)min((total + target - 1) / target, (long long)INT_MAX), sure = (int)min((total + room - 1) / room, (long long)INT_MAX);
    int run = max(1, sure);
    if (blocks <= kPlanSearch) {
        const int r = max(1, (int)(share + (long long)(sure - share) * tid / (T - 1)));
        int n = 0;
        for (int i = 0; i < blocks; i++) n = min(n + (int)(((unsigned)cost(block(i)) + r - 1) / (unsigned)r), target + 1);
        const int least = __reduce_min_sync(0xffffffffu, n > target ? run : r);
        if (lane == 0) sm.w_max[warp] = least;
        __syncthreads();
        for (int w = 0; w < W; w++) run = min(run, sm.w_max[w]);
    }

    // ---- the pieces
    int pieces = 0;
    for (int i0 = 0; i0 < blocks; i0 += T) {
        const int i = i0 + tid;
        const int4 at = i < blocks ? block(i) : make_int4(0, 0, 0, 0);
        const int np = min((at.w + keys - 1) / keys, (int)(((unsigned)cost(at) + run - 1) / (unsigned)run));
        const int incl = plan_scan(np, sum);
        if (lane == 31) sm.w_sum[warp] = incl;
        __syncthreads();
        int first = pieces + incl - np;
        for (int w = 0; w < W; w++) {
            if (w < warp) first += sm.w_sum[w];
            pieces += sm.w_sum[w];
        }
        if (i < blocks) a.plan.first[i] = first;
        sm.np[tid] = np;
        sm.first[tid] = first;
        __syncthreads();
        for (int s = warp; s < min(T, blocks - i0); s += W) {
            const int n = sm.np[s], f = sm.first[s];
            const int4 k = block(i0 + s);
            const int t = (k.w + keys - 1) / keys, g = (i0 + s) % G;
            for (int j = lane; j < n; j += 32) {
                a.plan.piece[2 * (f + j)] = k;
                a.plan.piece[2 * (f + j) + 1] = make_int4(g, (int)((long long)j * t / n), (int)((j + 1ll) * t / n), 0);
            }
        }
        __syncthreads();
    }
    if (tid == 0) {
        a.plan.first[blocks] = pieces;
        *a.plan.pieces = pieces;
    }
}

}  // namespace serve
}  // namespace gkv
