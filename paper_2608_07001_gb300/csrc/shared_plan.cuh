// shared_plan.cuh -- the plan of the attention over a shared prefix: the blocks of
// rows of all slots, and how many pieces each one's keys are cut into, so that
// the pieces fill the SMs at a time that is the least of 32 candidates'.
#pragma once

#include "shared.cuh"

#include <limits.h>

namespace gkv {
namespace serve {

constexpr int kPieceStart = 5;             // what a piece costs beside its tiles, in tiles
constexpr int kPlanBlocks = 512;           // blocks that are kept in shared memory too
constexpr int kPlanSearch = 64;            // blocks up to which candidates are compared

template <int T>
struct PlanSmem {
    int w_max[T / 32], w_sum[T / 32], lo[T], n[T], rb[T], np[T], first[T];
    int used[T / 32], longest[T / 32], run;
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
    long long total = 0;                                 // tiles; blocks that have any; the most of a block
    int used = 0, longest = 0;
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
                const int t = (k + keys - 1) / keys;
                total += t;
                used += t > 0;
                longest = max(longest, t);
            }
        }
        __syncthreads();
    }
    const int blocks = base * G;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        used += __shfl_xor_sync(0xffffffffu, used, o);
        longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
    }
    if (lane == 0) {
        sm.total[warp] = total;
        sm.used[warp] = used;
        sm.longest[warp] = longest;
    }
    __syncthreads();
    total = used = longest = 0;
    for (int w = 0; w < W; w++) {
        total += sm.total[w];
        used += sm.used[w];
        longest = max(longest, sm.longest[w]);
    }
    auto block = [&](int i) { return i < kPlanBlocks ? sm.blk[i] : a.plan.blk[i]; };
    auto tiles = [&](int i) { return (block(i).w + keys - 1) / keys; };

    // ---- tiles of a piece: the candidates lie between an even share of all tiles and what is sure to give no more
    // pieces than there is room for (sum of ceil(t / run) <= total / run + used)
    const int room = most - used;                        // at least half of the SMs, or twice the SMs
    const int share = (int)min((total + most - 1) / most, (long long)INT_MAX), sure = (int)min((total + room - 1) / room, (long long)INT_MAX);
    int run = max(1, sure);
    if (blocks <= kPlanSearch) {
        if (warp == 0) {
            const long long widest = max((long long)sure, min((long long)longest, 4ll * sure));
            const int r = max(1, (int)(share + (widest - share) * lane / 31));
            int n = 0;                                   // pieces, above `most` too many anyway
            for (int i = 0; i < blocks; i++) n = min(n + (tiles(i) + r - 1) / r, most + 1);
            // the cost and the candidate in one word, the least of all lanes
            long long cost = n > most ? LLONG_MAX : (long long)((n + kShSms - 1) / kShSms) * (r + kPieceStart) * 32 + lane;
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) cost = min(cost, __shfl_xor_sync(0xffffffffu, cost, o));
            const int best = __shfl_sync(0xffffffffu, r, (int)(cost & 31));
            if (lane == 0) sm.run = cost == LLONG_MAX ? run : best;
        }
        __syncthreads();
        run = sm.run;
    }

    // ---- the pieces
    int pieces = 0;
    for (int i0 = 0; i0 < blocks; i0 += T) {
        const int i = i0 + tid;
        const int np = i < blocks ? (tiles(i) + run - 1) / run : 0;
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
