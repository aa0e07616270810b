// paged_attention.cu -- attention of one token per request over the paged
// cache (gracekv_paged_attention; App. A.3, Eq. app_decode_logit).
//
// For every sequence s = (b, g) and its gq = Hq / G query heads h, over its
// lens[s] entries e:
//     x_e = q_h . k_e / sqrt(d) + log m_e,  out_h = sum_e softmax(x)_e v_e .
// Every entry is read once (2 d elements and log m) for 4 gq d operations, so
// HBM bounds it, or the latency of a launch when there is little to read.
//
//   * Work split.  The sequences' tiles of TE entries form one line that is cut
//     into equal runs, one per CTA, whatever the lengths (the compression gives
//     every head its own).  A CTA finds its run from the lengths alone: its
//     threads sum them in segments and one thread walks the segment its run
//     begins in.  A run meets one or more sequences; each meeting is a piece.
//     Where the longest sequence has few tiles (kPaSnap), a run takes the
//     sequences that begin in it whole instead: joining pieces costs more than
//     the tiles that it would spread.
//   * One producer warp streams a piece's tiles through a ring of shared memory:
//     TMA boxes of up to 64 rows that do not cross a page (the box height is the
//     largest of 64, 32, 16 dividing the page), 128-byte swizzle, log m as a
//     bulk copy, all on one mbarrier a stage.  Its lanes look 32 boxes ahead in
//     the table, so the page numbers are not in the way of the copies.
//   * bf16: four consumer warps take 16 entries of every tile each and keep
//     their own running maximum, sum and 16 x d accumulator, so no warp waits
//     for another inside a piece.  Products on mma.m16n8k16 (exact bf16
//     products, fp32 sums): the heads are the 16 rows, and since gq <= 8 the
//     upper 8 rows carry the same queries again -- the logits come out twice,
//     and the value product's rows 0-7 take the weights' bf16 part and rows
//     8-15 the remainder's, two parts (2^-16 of a weight) for one product.  That is
//     2^-8 of what rounding the output to bf16 moves; a third part, as for one
//     request's packed cache (decode.cu), would double the value product.
//     tcgen05 would need 128 rows for the same 8 heads.
//   * fp32: a warp takes whole tiles of 32 entries, the tiles of its own stages
//     of the ring; lanes are entries for the logits (no reduction) and channels for the values; packed fp32x2 FMA.
//   * Rows past a length, entries of pages outside the pool: weight 0, and
//     their values are replaced by 0 before the product, whatever they hold.
//   * A piece that is not its whole sequence leaves (max, sum, weighted sums);
//     the CTA finishing the sequence's last piece, found with a counter, joins
//     them in order.  Nothing waits for another CTA, and results do not depend
//     on timing.
//
// Measured, GPU time: 88 us for 1M entries of 2 x 128 bf16 and log m (32 requests x 8
// heads, uneven; 6.1 TB/s, 0.90 of a plain copy's rate), the same for one request of
// 131072 entries; 6.1 us for one request of 8 x 256 entries (a call from Python
// takes 8 to 11).
//
// log m joins in base 2 with log m log2(e) held between the finite values, so
// that entries of the lowest or the largest log m keep equal weights; -inf stays
// no weight.  A logit that is NaN or +inf makes its head's output NaN: the
// quotient is 0 only where no weight at all was summed.
#include "paged.cuh"
#include "tc.cuh"

#include <float.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace gkv {
namespace {

using namespace serve;

constexpr int kPaWarps = 4;                        // consumer warps
constexpr int kPaCons = kPaWarps * 32;
constexpr int kPaThreads = kPaCons + 32;           // + the producer warp
constexpr int kPaF32Warps = 3;                     // of them take tiles in the fp32 kernel: one a stage, in turn
constexpr int kPaRing = 96 * 1024;                 // bytes of the ring
constexpr int kPaPerSm = 2;                        // resident CTAs a SM
constexpr int kPaMaxGrid = 512;
constexpr int kPaSnap = 8;                         // tiles of the longest sequence up to which none is split
constexpr int kPaPieces = 64;                      // pieces of a sequence that small launches aim at, at most
constexpr uint64_t kPaWaitNs = 2000000000ull;

template <typename T, int D>
struct PaCfg {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int TE = BF ? 64 : 32;        // entries of a tile
    static constexpr int NB = D * (int)sizeof(T) / 128;          // 128-byte column boxes of a row
    static constexpr int TB = NB * TE * 128;       // bytes of a tile's keys
    static constexpr int NST = kPaRing / (2 * TB); // stages
    static constexpr int MIN = BF ? 2 : 1;         // tiles of a run at least
    static_assert(NST >= 3 && NST <= 12 && (BF || NST % kPaF32Warps == 0), "ring");
};

struct PaArgs {
    Paged c;
    int S;                      // B G
    const int32_t *lens, *table;                   // of the layer
    const void *q;
    void *out;
    float *part;                // [2 grid][part floats]
    int *cnt;                   // [grid] pieces finished of the sequence that begins in a CTA and leaves it
    int *status;
    int box;                    // rows of a box
    float scale;                // log2(e) / sqrt(d)
};

template <int NST, int TE>
struct PaSmem {
    uint64_t full[NST], empty[NST];
    alignas(16) float lm[NST][TE];
    int count[NST];             // valid entries of the stage's tile
    unsigned units[NST];        // its boxes that were read
    long long first, total;     // the CTA's first sequence: prefix of tiles before it; all tiles
    int s_first;
    int abort, last;
    long long wsum[kPaThreads / 32];
    int wmax[kPaThreads / 32];
    float m[kPaWarps][8], z[kPaWarps][8], M[8], Z[8];
};

constexpr int pa_part_floats(int D) { return 8 * D + 16; }

__device__ __forceinline__ void pa_ldsm4(uint32_t addr, uint32_t a[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr));
}
__device__ __forceinline__ void pa_ldsm4t(uint32_t addr, uint32_t a[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr));
}
__device__ __forceinline__ void pa_mma(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pa_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void pa_bulk(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void pa_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kPaCons) : "memory"); }

// Bounded wait; gives up at once when another thread has.
template <typename SM>
__device__ __forceinline__ bool pa_wait(uint32_t bar, uint32_t parity, SM &sm, int *status) {
    if (tc::mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t it = 0;; it++) {
        if (tc::mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 63u) {
            if (*(volatile int *)&sm.abort) return false;
            if (tc::globaltimer_ns() - t0 > kPaWaitNs) {
                atomicOr(status, kStTimeout);
                atomicExch(&sm.abort, 1);
                return false;
            }
        }
    }
}

// Entries of sequence s that are followed.
__device__ __forceinline__ int pa_len(const PaArgs &a, int s) {
    return max(0, min(a.lens[s], a.c.page_size * a.c.max_pages));
}
// `total` tiles are cut into nc runs [c total / nc, (c + 1) total / nc): where run c begins, and the run of tile i.
// Up to kPaNarrow tiles the products fit 32 bits (nc <= kPaMaxGrid); a 64-bit division costs about 0.1 us, and
// five of them lie on the way of a call that reads little.
constexpr long long kPaNarrow = 1 << 22;
__device__ __forceinline__ long long pa_run_first(int c, long long total, int nc) {
    return total <= kPaNarrow ? (uint32_t)c * (uint32_t)total / (uint32_t)nc : c * total / nc;
}
__device__ __forceinline__ int pa_run_of(long long i, long long total, int nc) {
    return total <= kPaNarrow ? (int)((((uint32_t)i + 1) * (uint32_t)nc + (uint32_t)total - 1) / (uint32_t)total) - 1
                              : (int)(((i + 1) * nc + total - 1) / total - 1);
}

// log m in base 2: finite values stay finite, the others what they are.
__device__ __forceinline__ float pa_lm2(float lm) {
    return fabsf(lm) <= FLT_MAX ? fminf(fmaxf(lm * kLog2e, -FLT_MAX), FLT_MAX) : lm;
}
__device__ __forceinline__ float pa_shift(float m) { return m == -INFINITY ? 0.f : m; }

// ---------------------------------------------------------------- consumers
// bf16: this warp's 16 entries of every tile of [t0, t1).
template <int D>
struct PaBf {
    using C = PaCfg<__nv_bfloat16, D>;
    uint32_t qa[D / 16][2];     // the queries as 16 x 16 row operands: rows 0-7 (8-15 the same)
    float acc[D / 8][4];        // rows hq: weights' first part, rows hq + 8: second part; columns of 8 channels
    float m, z;                 // of head hq; z: this lane's share

    __device__ __forceinline__ void begin(const PaArgs &a, int s, int gq) {
        const int lane = threadIdx.x & 31, hq = lane >> 2, tq = lane & 3;
        const uint32_t *q = reinterpret_cast<const uint32_t *>(
            static_cast<const __nv_bfloat16 *>(a.q) + ((size_t)s * gq + (hq < gq ? hq : 0)) * D);
#pragma unroll
        for (int kk = 0; kk < D / 16; kk++) {
            qa[kk][0] = hq < gq ? q[kk * 8 + tq] : 0u;
            qa[kk][1] = hq < gq ? q[kk * 8 + 4 + tq] : 0u;
        }
#pragma unroll
        for (int i = 0; i < D / 8; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = 0.f;
        m = -INFINITY;
        z = 0.f;
    }

    // Offset of the 16-byte chunk `ch` of row r of a tile.
    static __device__ __forceinline__ uint32_t at(int r, int ch) {
        return (uint32_t)((ch >> 3) * (C::TE * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
    }

    __device__ __forceinline__ void tile(uint32_t kst, uint32_t vst, const float *lm, int count, unsigned units, int box,
                                         float scale, bool has_lm) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tq = lane & 3;
        const int r0 = warp * 16;
        const int nv = min(16, count - r0);                       // valid entries of the slice
        if (nv <= 0 || !((units >> (r0 / box)) & 1u)) return;
        float x[2][4];
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) x[n][j] = 0.f;
        // matrices of a load: entries 0-7 / 8-15 x channels 0-7 / 8-15 of the step
        const int mi = lane >> 3, ri = lane & 7;
#pragma unroll
        for (int kk = 0; kk < D / 16; kk++) {
            uint32_t b[4];
            pa_ldsm4(kst + at(r0 + ri + (mi >> 1) * 8, kk * 2 + (mi & 1)), b);
            pa_mma(x[0], qa[kk][0], qa[kk][0], qa[kk][1], qa[kk][1], b[0], b[1]);
            pa_mma(x[1], qa[kk][0], qa[kk][0], qa[kk][1], qa[kk][1], b[2], b[3]);
        }
        // x[n][j]: head hq, entry 8 n + 2 tq + j (j < 2; j >= 2 repeats it)
        float y[2][2], mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const int e = n * 8 + 2 * tq + j;
                float v = x[n][j] * scale;
                if (has_lm) v += pa_lm2(lm[r0 + e]);
                y[n][j] = e < nv ? v : -INFINITY;
                mx = fmaxf(mx, y[n][j]);
            }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (__any_sync(0xffffffffu, mx > m)) {
            const float mn = fmaxf(m, mx), w = tc::ex2(m - pa_shift(mn));     // 0 from no entry so far
            m = mn;
            z *= w;
#pragma unroll
            for (int i = 0; i < D / 8; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] *= w;
        }
        const float sh = pa_shift(m);
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int n = 0; n < 2; n++) {
            const float p0 = tc::ex2(y[n][0] - sh), p1 = tc::ex2(y[n][1] - sh);
            z += p0 + p1;
            hi[n] = pa_bf16x2(p0, p1);
            lo[n] = pa_bf16x2(p0 - __uint_as_float(hi[n] << 16), p1 - __uint_as_float(hi[n] & 0xffff0000u));
        }
        // value rows past the length hold anything: 0 in the operand (words of entries 2 tq, 2 tq + 1 and + 8)
        uint32_t keep0 = ~0u, keep1 = ~0u;
        if (nv < 16) {
            keep0 = (2 * tq < nv ? 0xffffu : 0u) | (2 * tq + 1 < nv ? 0xffff0000u : 0u);
            keep1 = (2 * tq + 8 < nv ? 0xffffu : 0u) | (2 * tq + 9 < nv ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int i = 0; i < D / 16; i++) {
            uint32_t b[4];      // entries 0-7, 8-15 of channels 16 i .. + 7, then of + 8 .. + 15
            pa_ldsm4t(vst + at(r0 + ri + (mi & 1) * 8, i * 2 + (mi >> 1)), b);
            pa_mma(acc[2 * i], hi[0], lo[0], hi[1], lo[1], b[0] & keep0, b[1] & keep1);
            pa_mma(acc[2 * i + 1], hi[0], lo[0], hi[1], lo[1], b[2] & keep0, b[3] & keep1);
        }
    }

    // Maximum and sum of every head of this warp into shared memory.
    __device__ __forceinline__ void stats(float *ms, float *zs) {
        const int lane = threadIdx.x & 31;
        z += __shfl_xor_sync(0xffffffffu, z, 1);
        z += __shfl_xor_sync(0xffffffffu, z, 2);
        if ((lane & 3) == 0) { ms[lane >> 2] = m; zs[lane >> 2] = z; }
    }
    // Adds this warp's sums, scaled to the maxima M, into [8][D].
    __device__ __forceinline__ void add(float *sum, const float *M, int gq, bool first) {
        const int lane = threadIdx.x & 31, hq = lane >> 2, tq = lane & 3;
        if (hq >= gq) return;
        const float w = tc::ex2(m - pa_shift(M[hq]));
#pragma unroll
        for (int i = 0; i < D / 8; i++) {
            float2 *p = reinterpret_cast<float2 *>(sum + hq * D + i * 8 + 2 * tq);
            float2 v = first ? make_float2(0.f, 0.f) : *p;
            v.x += w * (acc[i][0] + acc[i][2]);
            v.y += w * (acc[i][1] + acc[i][3]);
            *p = v;
        }
    }
};

// fp32: whole tiles of 32 entries, one warp each.
template <int D, int GQ>
struct PaF32 {
    using C = PaCfg<float, D>;
    static constexpr int E = D / 32;           // channels of a lane
    float2 acc[GQ][E / 2];
    float m[GQ], z[GQ];                        // z: this lane's share
    float *qs, *ps;                            // shared: [GQ][D] queries (scaled), this warp's [GQ][32] weights

    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int h = 0; h < GQ; h++) {
#pragma unroll
            for (int e = 0; e < E / 2; e++) acc[h][e] = make_float2(0.f, 0.f);
            m[h] = -INFINITY;
            z[h] = 0.f;
        }
    }

    __device__ __forceinline__ void tile(const unsigned char *kst, const unsigned char *vst, const float *lm, int count,
                                         unsigned units, int box, bool has_lm) {
        const int lane = threadIdx.x & 31;
        const bool in = lane < count && ((units >> (lane / box)) & 1u);
        float2 x[GQ];
#pragma unroll
        for (int h = 0; h < GQ; h++) x[h] = make_float2(0.f, 0.f);
#pragma unroll 8
        for (int ch = 0; ch < D / 4; ch++) {
            const float4 k = *reinterpret_cast<const float4 *>(kst + (ch >> 3) * (C::TE * 128) + lane * 128 +
                                                               (((ch & 7) ^ (lane & 7)) << 4));
#pragma unroll
            for (int h = 0; h < GQ; h++) {
                const float4 q = *reinterpret_cast<const float4 *>(qs + h * D + ch * 4);
                x[h] = __ffma2_rn(make_float2(q.x, q.y), make_float2(k.x, k.y), x[h]);
                x[h] = __ffma2_rn(make_float2(q.z, q.w), make_float2(k.z, k.w), x[h]);
            }
        }
        const float l2 = has_lm ? pa_lm2(lm[lane]) : 0.f;
#pragma unroll
        for (int h = 0; h < GQ; h++) {
            const float y = in ? x[h].x + x[h].y + l2 : -INFINITY;
            float mx = y;
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            if (mx > m[h]) {                    // the same in every lane
                const float w = tc::ex2(m[h] - mx);
                m[h] = mx;
                z[h] *= w;
#pragma unroll
                for (int e = 0; e < E / 2; e++) { acc[h][e].x *= w; acc[h][e].y *= w; }
            }
            const float p = tc::ex2(y - pa_shift(m[h]));
            z[h] += p;
            ps[h * 32 + lane] = p;
        }
        __syncwarp();
        const unsigned ok = __ballot_sync(0xffffffffu, in);
        // lane's channels: E consecutive ones
        const int ch = lane * E / 4;
        const int off = (ch >> 3) * (C::TE * 128) + (E == 2 ? (lane & 1) * 8 : 0);
#pragma unroll 2
        for (int e0 = 0; e0 < 32; e0 += 4) {
            if (!((ok >> e0) & 15u)) continue;
            float4 p[GQ];
#pragma unroll
            for (int h = 0; h < GQ; h++) p[h] = *reinterpret_cast<const float4 *>(ps + h * 32 + e0);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int e = e0 + j;
                float2 v[E / 2];
                const unsigned char *r = vst + off + e * 128 + (((ch & 7) ^ (e & 7)) << 4);
#pragma unroll
                for (int i = 0; i < E / 2; i++) v[i] = *reinterpret_cast<const float2 *>(r + i * 8);
                if (!((ok >> e) & 1u)) {
#pragma unroll
                    for (int i = 0; i < E / 2; i++) v[i] = make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int h = 0; h < GQ; h++) {
                    const float w = j == 0 ? p[h].x : j == 1 ? p[h].y : j == 2 ? p[h].z : p[h].w;
#pragma unroll
                    for (int i = 0; i < E / 2; i++) acc[h][i] = __ffma2_rn(make_float2(w, w), v[i], acc[h][i]);
                }
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void stats(float *ms, float *zs) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < GQ; h++) {
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) z[h] += __shfl_xor_sync(0xffffffffu, z[h], o);
            if (lane == 0) { ms[h] = m[h]; zs[h] = z[h]; }
        }
    }
    __device__ __forceinline__ void add(float *sum, const float *M, int gq, bool first) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < GQ; h++) {
            if (h >= gq) break;
            const float w = tc::ex2(m[h] - pa_shift(M[h]));
#pragma unroll
            for (int i = 0; i < E / 2; i++) {
                float2 *p = reinterpret_cast<float2 *>(sum + h * D + lane * E + 2 * i);
                float2 v = first ? make_float2(0.f, 0.f) : *p;
                v.x += w * acc[h][i].x;
                v.y += w * acc[h][i].y;
                *p = v;
            }
        }
    }
};

// ------------------------------------------------------------------ kernel
template <typename T, int D, int GQ>
__global__ void __launch_bounds__(kPaThreads, kPaPerSm)
    paged_attention_kernel(const PaArgs a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV) {
    using C = PaCfg<T, D>;
    using SM = PaSmem<C::NST, C::TE>;
    extern __shared__ __align__(1024) unsigned char dsm[];
    unsigned char *ring = dsm;                                   // [NST][keys, values]
    float *sum = reinterpret_cast<float *>(dsm + C::NST * 2 * C::TB);        // [8][D]
    float *qs = sum + 8 * D;                                     // fp32: [GQ][D] queries, then [4][GQ][32] weights
    __shared__ SM sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int gq = a.c.Hq / a.c.G, S = a.S;

    next_may_start();
    if (tid == 0) {
        for (int i = 0; i < C::NST; i++) {
            tc::mbar_init(tc::smem_u32(&sm.full[i]), 1);
            tc::mbar_init(tc::smem_u32(&sm.empty[i]), C::BF ? kPaWarps : 1);
        }
        sm.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == kPaWarps && lane == 0) {
        tc::tma_prefetch_desc(&mapK);
        tc::tma_prefetch_desc(&mapV);
    }
    after_previous();

    // ---- the CTA's run: tiles of all sequences, and where its own begin
    const int seg = (S + kPaThreads - 1) / kPaThreads;
    long long mine = 0;
    int most = 0;
    for (int s = tid * seg; s < min(S, (tid + 1) * seg); s++) {
        const int n = pa_len(a, s);
        if (n < a.lens[s]) atomicOr(a.status, kStRange);
        mine += (n + C::TE - 1) / C::TE;
        most = max(most, (n + C::TE - 1) / C::TE);
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane == 0) sm.wmax[warp] = most;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sm.wsum[warp] = incl;
    __syncthreads();
    long long before = incl - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kPaThreads / 32; w++) {
        if (w < warp) before += sm.wsum[w];
        total += sm.wsum[w];
        most = max(most, sm.wmax[w]);
    }
    const bool snap = most <= kPaSnap;
    // A run holds MIN tiles at least, and as many as leave the longest sequence kPaPieces pieces: one CTA
    // joins them, eight or sixteen at a time.  (16000 entries of 2 sequences: 14.9 us with runs of 2 or 4
    // tiles, 16.4 of 8; 60000 entries of one head: 22.4 us in 64 pieces, 24.7 in 128; 2000 entries of 8
    // sequences: 11.0 of 2 tiles, 11.8 of 4, 14.4 of 8; fp32, 1000 entries of 10 in tiles of 32: 11.5 of 1,
    // 12.7 of 2, 14.0 of 4.)
    const int least = max(C::MIN, (most + kPaPieces - 1) / kPaPieces);
    const int nc = total <= kPaNarrow ? min((int)gridDim.x, (int)(((uint32_t)total + least - 1) / (uint32_t)least))
                                      : (int)min((long long)gridDim.x, (total + least - 1) / least);
    const long long lo = (int)blockIdx.x < nc ? pa_run_first(blockIdx.x, total, nc) : total;
    const long long hi = (int)blockIdx.x < nc ? pa_run_first(blockIdx.x + 1, total, nc) : total;
    if (lo < hi && lo >= before && lo < before + mine) {
        int s = tid * seg;
        for (;; s++) {
            const int n = (pa_len(a, s) + C::TE - 1) / C::TE;
            if (lo < before + n) break;
            before += n;
        }
        if (snap && lo > before) before += (pa_len(a, s++) + C::TE - 1) / C::TE;
        sm.s_first = s;
        sm.first = before;
    }
    // sequences without an entry
    for (int s = blockIdx.x; s < S; s += gridDim.x)
        if (a.lens[s] <= 0)
            for (int i = tid; i < gq * D; i += kPaThreads) put(static_cast<T *>(a.out) + (size_t)s * gq * D + i, 0.f);
    __syncthreads();
    if (lo >= hi) return;

    if (warp == kPaWarps) {
        // ---------------- producer ----------------
        const int per_tile = C::TE / min(a.box, C::TE), box = min(a.box, C::TE);
        uint32_t it = 0;
        bool ok = true;
        long long vs = sm.first;
        for (int s = sm.s_first; ok && s < S && vs < hi; s++) {
            const int n = pa_len(a, s), nt = (n + C::TE - 1) / C::TE;
            const int t0 = snap ? 0 : (int)(max(lo, vs) - vs), t1 = snap ? nt : (int)(min(hi, vs + nt) - vs);
            vs += nt;
            int held0 = 0, held = 0;                 // boxes [held0, held0 + held) looked up, one a lane
            int row = -1;
            for (int t = t0; ok && t < t1; t++, it++) {
                if (t * per_tile + per_tile > held0 + held || t == t0) {
                    held0 = t * per_tile;
                    held = 32;
                    const int e = (held0 + lane) * box;
                    row = -1;
                    if (e < n && held0 + lane < t1 * per_tile) {
                        const int64_t r = entry_row(Paged{nullptr, nullptr, nullptr, a.table, nullptr, 0, 0, 0, 0,
                                                          a.c.page_size, a.c.max_pages, a.c.n_pages}, s, e, a.status);
                        row = (int)r;
                    }
                }
                const int st = it % C::NST;
                ok = !*(volatile int *)&sm.abort &&
                     pa_wait(tc::smem_u32(&sm.empty[st]), ((it / C::NST) & 1) ^ 1, sm, a.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                // lane u < per_tile: box u of the tile
                const int u = lane;
                const int r = __shfl_sync(0xffffffffu, row, (t * per_tile - held0 + u) & 31);
                const bool have = u < per_tile && r >= 0;
                const unsigned units = __ballot_sync(0xffffffffu, have);
                const uint32_t fb = tc::smem_u32(&sm.full[st]);
                const uint32_t bytes = (uint32_t)(2 * C::NB * box * 128 + (a.c.log_m ? box * 4 : 0));
                if (lane == 0) {
                    sm.count[st] = min(C::TE, n - t * C::TE);
                    sm.units[st] = units;
                    if (units) tc::mbar_expect_tx(fb, bytes * __popc(units));
                    else tc::mbar_arrive(fb);
                }
                __syncwarp();
                if (have) {
                    const uint32_t kb = tc::smem_u32(ring + st * 2 * C::TB) + (uint32_t)(u * box * 128);
#pragma unroll
                    for (int b = 0; b < C::NB; b++) {
                        tc::tma_load_2d(kb + (uint32_t)(b * C::TE * 128), &mapK, b * (128 / (int)sizeof(T)), r, fb);
                        tc::tma_load_2d(kb + (uint32_t)(C::TB + b * C::TE * 128), &mapV, b * (128 / (int)sizeof(T)), r, fb);
                    }
                    if (a.c.log_m) pa_bulk(tc::smem_u32(&sm.lm[st][u * box]), a.c.log_m + r, (uint32_t)(box * 4), fb);
                }
            }
        }
        // the copies still in flight land before the block exits
        if (lane == 0)
            for (uint32_t i = it > C::NST ? it - C::NST : 0; i < it; i++)
                tc::mbar_wait(tc::smem_u32(&sm.full[i % C::NST]), (i / C::NST) & 1, kPaWaitNs);
        return;
    }

    // ---------------- consumers ----------------
    typename std::conditional<C::BF, PaBf<D>, PaF32<D, GQ>>::type w;
    if constexpr (!C::BF) {
        w.qs = qs;
        w.ps = qs + GQ * D + warp * GQ * 32;
    }
    uint32_t it = 0;
    long long vs = sm.first;
    for (int s = sm.s_first; s < S && vs < hi; s++) {
        const int n = pa_len(a, s), nt = (n + C::TE - 1) / C::TE;
        if (nt == 0) continue;
        const long long ve = vs + nt;
        const int t0 = snap ? 0 : (int)(max(lo, vs) - vs), t1 = snap ? nt : (int)(min(hi, ve) - vs);
        if constexpr (C::BF) {
            w.begin(a, s, gq);
        } else {
            for (int i = tid; i < GQ * D; i += kPaCons)
                qs[i] = i < gq * D ? static_cast<const float *>(a.q)[(size_t)s * gq * D + i] * a.scale : 0.f;
            w.begin();
            pa_sync();
        }
        for (int t = t0; t < t1; t++, it++) {
            const int st = it % C::NST;
            if (!C::BF && st % kPaF32Warps != warp) continue;        // a stage has one reader, which sees its every phase
            if (!pa_wait(tc::smem_u32(&sm.full[st]), (it / C::NST) & 1, sm, a.status)) continue;
            unsigned char *base = ring + st * 2 * C::TB;
            const int box = min(a.box, C::TE);
            if constexpr (C::BF)
                w.tile(tc::smem_u32(base), tc::smem_u32(base + C::TB), sm.lm[st], sm.count[st], sm.units[st], box, a.scale,
                       a.c.log_m != nullptr);
            else
                w.tile(base, base + C::TB, sm.lm[st], sm.count[st], sm.units[st], box, a.c.log_m != nullptr);
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sm.empty[st]));
        }
        // ---- the piece: the warps' maxima, then their sums in order
        w.stats(sm.m[warp], sm.z[warp]);
        pa_sync();
        if (tid < gq) {
            float M = -INFINITY, Z = 0.f;
            for (int i = 0; i < kPaWarps; i++) M = fmaxf(M, sm.m[i][tid]);
            for (int i = 0; i < kPaWarps; i++) Z += sm.z[i][tid] * tc::ex2(sm.m[i][tid] - pa_shift(M));
            sm.M[tid] = M;
            sm.Z[tid] = Z;
        }
        pa_sync();
        // fp32: only the warps that had one of the piece's tiles, from its first stage on
        const int adds = C::BF ? kPaWarps : min(kPaF32Warps, t1 - t0), from = C::BF ? 0 : (int)((it - (t1 - t0)) % kPaF32Warps);
        for (int i = 0; i < adds; i++) {
            if (warp == (C::BF ? i : (from + i) % kPaF32Warps)) w.add(sum, sm.M, gq, i == 0);
            pa_sync();
        }
        T *out = static_cast<T *>(a.out) + (size_t)s * gq * D;
        const int c_lo = pa_run_of(vs, total, nc), c_hi = pa_run_of(ve - 1, total, nc);
        if (snap || c_lo == c_hi) {
            for (int i = tid; i < gq * D; i += kPaCons) {
                const float Z = sm.Z[i / D];
                put(out + i, Z == 0.f ? 0.f : sum[i] / Z);               // a NaN stays
            }
        } else {
            // slot 2 c: the sequence the CTA continues, 2 c + 1: the one it begins and leaves
            constexpr int PF = pa_part_floats(D);
            float *pp = a.part + (size_t)(2 * blockIdx.x + ((int)blockIdx.x == c_lo)) * PF;
            for (int i = tid; i < gq * D; i += kPaCons) pp[i] = sum[i];
            if (tid < gq) { pp[8 * D + tid] = sm.M[tid]; pp[8 * D + 8 + tid] = sm.Z[tid]; }
            __threadfence();
            pa_sync();
            if (tid == 0) sm.last = atomicAdd(a.cnt + c_lo, 1) == c_hi - c_lo;
            pa_sync();
            if (sm.last) {
                __threadfence();
                const int np = c_hi - c_lo + 1;
                auto piece = [&](int p) { return a.part + (size_t)(2 * (c_lo + p) + (p == 0)) * PF; };
                // four channels a thread, over the pieces in order, N loads in flight: a batch is the latency of a
                // read (0.8 us), so 16 where there are more than 8 pieces
                auto join = [&](auto batch) {
                    constexpr int N = decltype(batch)::value;
                    for (int i = tid * 4; i < gq * D; i += kPaCons * 4) {
                        const int h = i / D;
                        float M = -INFINITY, Z = 0.f;
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int p0 = 0; p0 < np; p0 += N) {
                            float m[N], z[N], mx = M;
                            float4 x[N];
#pragma unroll
                            for (int p = 0; p < N; p++) {
                                // past the last piece: the last one again, with no weight
                                const float *q = piece(min(p0 + p, np - 1));
                                m[p] = __ldcg(q + 8 * D + h);
                                z[p] = __ldcg(q + 8 * D + 8 + h);
                                x[p] = __ldcg(reinterpret_cast<const float4 *>(q + i));
                            }
#pragma unroll
                            for (int p = 0; p < N; p++) {
                                if (p0 + p >= np) m[p] = -INFINITY;
                                mx = fmaxf(mx, m[p]);
                            }
                            const float sh = pa_shift(mx), f = tc::ex2(M - sh);
                            M = mx;
                            Z *= f;
                            v.x *= f; v.y *= f; v.z *= f; v.w *= f;
#pragma unroll
                            for (int p = 0; p < N; p++) {
                                const float g = tc::ex2(m[p] - sh);
                                Z += g * z[p];
                                v.x += g * x[p].x; v.y += g * x[p].y; v.z += g * x[p].z; v.w += g * x[p].w;
                            }
                        }
                        const float r = Z == 0.f ? 0.f : 1.f / Z;                // a NaN stays
                        put4(out + i, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
                    }
                };
                if (np > 8) join(std::integral_constant<int, 16>()); else join(std::integral_constant<int, 8>());
                if (tid == 0) a.cnt[c_lo] = 0;
            }
        }
        vs = ve;
        pa_sync();                          // sums, queries and head words are used again
    }
}

// [rows][D] rows, boxes of [box][128 bytes], 128-byte swizzle.
template <typename T>
bool pa_map(CUtensorMap *m, const void *p, int64_t rows, int d, int box) {
    auto enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t gdim[2] = {(cuuint64_t)d, (cuuint64_t)rows};
    cuuint64_t gstr[1] = {(cuuint64_t)d * sizeof(T)};
    cuuint32_t bx[2] = {128 / (cuuint32_t)sizeof(T), (cuuint32_t)box};
    cuuint32_t es[2] = {1, 1};
    return enc(m, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
               const_cast<void *>(p), gdim, gstr, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}


template <typename T, int D, int GQ>
cudaError_t pa_launch(PaArgs a, cudaStream_t s) {
    using C = PaCfg<T, D>;
    static std::atomic<int> grid_of[kMaxDevices];
    const auto kern = paged_attention_kernel<T, D, GQ>;
    const size_t smem = (size_t)C::NST * 2 * C::TB + 8 * D * sizeof(float) +
                        (C::BF ? 0 : (size_t)(GQ * D + kPaWarps * GQ * 32) * sizeof(float));
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    int grid = grid_of[dev].load(std::memory_order_relaxed);
    if (grid == 0) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        int per_sm = 1, sms = 1;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, kPaThreads, smem);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        grid = std::min(kPaMaxGrid, std::max(1, per_sm) * sms);
        grid_of[dev].store(grid, std::memory_order_relaxed);
    }
    CUtensorMap mk, mv;
    const int64_t rows = a.c.n_pages * a.c.page_size;
    const int box = std::min(a.box, C::TE);
    if (!pa_map<T>(&mk, a.c.K, rows, D, box) || !pa_map<T>(&mv, a.c.V, rows, D, box)) return cudaErrorNotSupported;
    return launch_overlapped(kern, grid, kPaThreads, smem, s, a, mk, mv);
}

template <int D>
cudaError_t pa_launch_f32(const PaArgs &a, int gq, cudaStream_t s) {
    return gq == 1 ? pa_launch<float, D, 1>(a, s) : gq == 2 ? pa_launch<float, D, 2>(a, s)
           : gq <= 4 ? pa_launch<float, D, 4>(a, s) : pa_launch<float, D, 8>(a, s);
}

constexpr size_t kPaCntBytes = kPaMaxGrid * sizeof(int);

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_paged_workspace_size(const gkv_paged_cache *c, size_t *bytes) {
    const gkv_status st = serve::check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = serve::kWsHead + kPaCntBytes + (size_t)2 * kPaMaxGrid * pa_part_floats(c->d) * sizeof(float);
    return GKV_OK;
}

extern "C" gkv_status gracekv_paged_attention(const gkv_paged_cache *c, int32_t l, const void *q, void *out,
                                              void *workspace, void *stream) {
    const gkv_status st = serve::check_paged(c);
    if (st != GKV_OK) return st;
    if (l < 0 || l >= c->L || !q || !out || !workspace) return GKV_EINVAL;
    if (!serve::al(q, 16) || !serve::al(out, 16) || !serve::al(workspace, 256)) return GKV_EINVAL;
    if (c->page_size % 16) return GKV_EUNSUPPORTED;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    PaArgs a;
    a.c = serve::paged_of(c);
    a.S = c->B * c->G;
    a.lens = c->lens + (int64_t)l * a.S;
    a.table = c->table + (int64_t)l * a.S * c->max_pages;
    a.q = q;
    a.out = out;
    a.status = reinterpret_cast<int *>(ws);
    a.cnt = reinterpret_cast<int *>(ws + serve::kWsHead);
    a.part = reinterpret_cast<float *>(ws + serve::kWsHead + kPaCntBytes);
    a.box = c->page_size % 64 == 0 ? 64 : c->page_size % 32 == 0 ? 32 : 16;
    a.scale = (float)(1.4426950408889634 / sqrt((double)c->d));
    const int gq = c->Hq / c->G;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (c->dtype == GKV_BF16)
        e = c->d == 128 ? pa_launch<__nv_bfloat16, 128, 8>(a, s) : pa_launch<__nv_bfloat16, 64, 8>(a, s);
    else
        e = c->d == 128 ? pa_launch_f32<128>(a, gq, s) : pa_launch_f32<64>(a, gq, s);
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}
