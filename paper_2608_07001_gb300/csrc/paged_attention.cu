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
// takes 8 to 11).  Quantised, half of the bytes: 59 us for those 1M entries (4.6 TB/s), 54 us
// for one request's, bound by the latency of the consumers' chain of a tile (about 2500 clocks
// for 128 entries, two CTAs of four such warps a SM) and not by HBM.
//
// Of a shared prefix's requests (SHARED) the same kernel leaves (maximum, sum, weighted
// sums) of the own entries, and one CTA more makes the plan of the prefix beside it.
//
// log m joins in base 2 with log m log2(e) held between the finite values, so
// that entries of the lowest or the largest log m keep equal weights; -inf stays
// no weight.  A logit that is NaN or +inf makes its head's output NaN: the
// quotient is 0 only where no weight at all was summed.
#include "paged.cuh"
#include "quant.cuh"
#include "shared_plan.cuh"
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
constexpr int kPaHeads = 4;                        // heads whose sums the warps leave at once
constexpr int kPaF32Warps = 3;                     // of them take tiles in the fp32 kernel: one a stage, in turn
constexpr int kPaRing = 96 * 1024;                 // bytes of the ring
constexpr int kPaPerSm = 2;                        // resident CTAs a SM
constexpr int kPaMaxGrid = 512;
constexpr int kPaSnap = 8;                         // tiles of the longest sequence up to which none is split
constexpr int kPaPieces = 64;                      // pieces of a sequence that small launches aim at, at most
constexpr uint64_t kPaWaitNs = 2000000000ull;

// T: rows of q and out; S: rows of the pools.
template <typename T, typename S, int D>
struct PaCfg {
    static constexpr bool BF = sizeof(T) == 2, QUANT = sizeof(S) == 1;
    static constexpr int TE = BF ? (QUANT ? 128 : 64) : 32;      // entries of a tile
    static constexpr int SNAP = kPaSnap * 64 / (BF ? TE : 64);   // kPaSnap in them (fp32: as it is)
    static constexpr int RB = D * (int)sizeof(S), BW = RB < 128 ? RB : 128;      // bytes of a row, of a column box's row
    static constexpr int NB = RB / BW;             // column boxes of a row
    static constexpr int TB = TE * RB;             // bytes of a tile's keys
    static constexpr int NST = kPaRing / (2 * TB) < 12 ? kPaRing / (2 * TB) : 12;      // stages
    // Offset of the 16-byte chunk `ch` of row r of a tile, swizzled over 128 or 64 bytes.
    static __device__ __forceinline__ uint32_t at(int r, int ch) {
        return BW == 128 ? (uint32_t)((ch >> 3) * (TE * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4))
                         : (uint32_t)(r * 64 + ((ch ^ ((r >> 1) & 3)) << 4));
    }
    static constexpr int MIN = BF && !QUANT ? 2 : 1;             // tiles of a run at least
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
    gkv_paged_scales scales;    // of quantised pools
};
struct PaSharedArgs : PaArgs {
    SharedArgs shared;
};
template <bool SHARED>
using PaArgsOf = typename std::conditional<SHARED, PaSharedArgs, PaArgs>::type;

template <int NST, int TE, bool QUANT>
struct PaSmem {
    uint64_t full[NST], empty[NST];
    alignas(16) float lm[NST][TE];
    alignas(16) uint8_t ks[QUANT ? NST : 1][TE], vs[QUANT ? NST : 1][TE];
    int count[NST];             // valid entries of the stage's tile
    unsigned units[NST];        // its boxes that were read
    long long first, total;     // the CTA's first sequence: prefix of tiles before it; all tiles
    int s_first;
    int abort, last;
    long long wsum[kPaThreads / 32];
    int wmax[kPaThreads / 32];
    float m[kPaWarps][8], z[kPaWarps][8], f[QUANT ? kPaWarps : 1][8], M[8], Z[8];
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
__device__ __forceinline__ void pa_zero16(uint32_t addr) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0) : "memory");
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

// log m in base 2, held within `most` (finite values stay finite), the others what they are.
__device__ __forceinline__ float pa_lm2(float lm, float most) {
    return fabsf(lm) <= FLT_MAX ? fminf(fmaxf(lm * kLog2e, -most), most) : lm;
}
__device__ __forceinline__ float pa_shift(float m) { return m == -INFINITY ? 0.f : m; }

// ---------------------------------------------------------------- consumers
// bf16: this warp's 16 entries of every tile of [t0, t1).
template <int D>
struct PaBf {
    using C = PaCfg<__nv_bfloat16, __nv_bfloat16, D>;
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

    __device__ __forceinline__ void tile(uint32_t kst, uint32_t vst, const uint8_t *, const uint8_t *, const float *lm,
                                         int count, unsigned units, int box, float scale, bool has_lm, float most) {
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
            pa_ldsm4(kst + C::at(r0 + ri + (mi >> 1) * 8, kk * 2 + (mi & 1)), b);
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
                if (has_lm) v += pa_lm2(lm[r0 + e], most);
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
            hi[n] = bf16x2_of(p0, p1);
            lo[n] = bf16x2_of(p0 - __uint_as_float(hi[n] << 16), p1 - __uint_as_float(hi[n] & 0xffff0000u));
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
            pa_ldsm4t(vst + C::at(r0 + ri + (mi & 1) * 8, i * 2 + (mi >> 1)), b);
            pa_mma(acc[2 * i], hi[0], lo[0], hi[1], lo[1], b[0] & keep0, b[1] & keep1);
            pa_mma(acc[2 * i + 1], hi[0], lo[0], hi[1], lo[1], b[2] & keep0, b[3] & keep1);
        }
    }

    // Maximum and sum of every head of this warp into shared memory.
    __device__ __forceinline__ void stats(float *ms, float *zs, float *) {
        const int lane = threadIdx.x & 31;
        z += __shfl_xor_sync(0xffffffffu, z, 1);
        z += __shfl_xor_sync(0xffffffffu, z, 2);
        if ((lane & 3) == 0) { ms[lane >> 2] = m; zs[lane >> 2] = z; }
    }
    // This warp's sums of heads h0 ... h0 + 3 into [4][D].
    __device__ __forceinline__ void leave(float *sum, int h0, int gq) {
        const int lane = threadIdx.x & 31, hq = lane >> 2, tq = lane & 3;
        if (hq < h0 || hq >= min(gq, h0 + kPaHeads)) return;
#pragma unroll
        for (int i = 0; i < D / 8; i++)
            *reinterpret_cast<float2 *>(sum + (hq - h0) * D + i * 8 + 2 * tq) = make_float2(acc[i][0] + acc[i][2], acc[i][1] + acc[i][3]);
    }
};

// The same over quantised pools.  The codes are exact in f16, and so are a head's
// queries times a power of two that brings its largest to 2^14 (down to 2^-38 of
// that), so the logits' products are those of the codes and both scales' exponents come after.  A
// thread's 4 bytes of an ldmatrix row are 4 neighbouring channels: they serve as
// channels 2 t, 2 t + 1 and + 8 of the product's step, which sums over them all, and
// the queries are laid out to match.  A transposed 16-bit word holds two channels, the
// even ones and the odd ones of 16 to a product.
// The values' scales 2^v_e go into the weights, P = p 2^(v_e - E + 14), E the power of two
// at or above the largest p 2^(v_e) so far, so that a value counts by its weight too; P
// as f16 and the remainder's 2^11 as f16, so to 2^-22 of a weight, or 2^-50 of the largest
// p 2^(v_e).  U is the largest log2 of that, E its integer above; both go by differences
// from the maximum, as beside logits of any size a scale's exponent would be lost.
// (Values as bf16 with their scales took 8 clocks for two codes instead of 2, and the
// kernel 73 us for 1M entries of d = 128.)
template <int D>
struct PaE4 {
    using C = PaCfg<__nv_bfloat16, E4m3, D>;
    uint32_t qa[D / 16][2];     // queries in f16, channels 16 i + 4 t .. + 3
    float acc[D / 8][4];        // as PaBf's, columns: the even, then the odd channels of 16
    float m, z, u;              // u: U
    int qe, ve;                 // the power of two taken from head hq's queries; E

    __device__ __forceinline__ void begin(const PaArgs &a, int s, int gq) {
        const int lane = threadIdx.x & 31, hq = lane >> 2, tq = lane & 3;
        const uint2 *q = reinterpret_cast<const uint2 *>(
            static_cast<const __nv_bfloat16 *>(a.q) + ((size_t)s * gq + (hq < gq ? hq : 0)) * D);
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; c++) {
            const uint2 u = hq < gq ? q[c * 4 + tq] : make_uint2(0, 0);
            qa[c][0] = u.x;
            qa[c][1] = u.y;
#pragma unroll
            for (int i = 0; i < 2; i++)
                top = fmaxf(top, fmaxf(finite_size(__uint_as_float(qa[c][i] << 16)), finite_size(__uint_as_float(qa[c][i] & 0xffff0000u))));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        qe = max((int)(__float_as_uint(top) >> 23) - 127 - 14, -100);
        const float f = __uint_as_float((uint32_t)(127 - qe) << 23);
#pragma unroll
        for (int c = 0; c < D / 16; c++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const __half2 h = __floats2half2_rn(__uint_as_float(qa[c][i] << 16) * f, __uint_as_float(qa[c][i] & 0xffff0000u) * f);
                qa[c][i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        ve = -120;
#pragma unroll
        for (int i = 0; i < D / 8; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = 0.f;
        m = u = -INFINITY;
        z = 0.f;
    }

    static __device__ __forceinline__ void mma_f16(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                   uint32_t b1) {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
            "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }

    // This warp's NG groups of 16 entries: their chains of products, exponentials and conversions run beside one another.
    static constexpr int NG = C::TE / 64;
    __device__ __forceinline__ void tile(uint32_t kst, uint32_t vst, const uint8_t *ks, const uint8_t *vs, const float *lm,
                                         int count, unsigned units, int box, float scale, bool has_lm, float most) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tq = lane & 3;
        const int mi = lane >> 3, ri = lane & 7;
        int nv[NG], some = 0;            // valid entries of a group
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const int r0 = (warp * NG + g) * 16;
            nv[g] = (units >> (r0 / box)) & 1u ? max(0, min(16, count - r0)) : 0;
            some |= nv[g];
        }
        if (!some) return;
        if (count < C::TE || units != (1u << (C::TE / box)) - 1) {
            // value rows that are not there hold anything: 0
#pragma unroll
            for (int g = 0; g < NG; g++)
                for (int i = lane; i < 16 * (D / 16); i += 32) {
                    const int r = (warp * NG + g) * 16 + i / (D / 16);
                    if (i / (D / 16) >= nv[g]) pa_zero16(vst + C::at(r, i % (D / 16)));
                }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // before the next copy into the stage
            __syncwarp();
        }
        float x[NG][2][4];
#pragma unroll
        for (int g = 0; g < NG; g++)
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int j = 0; j < 4; j++) x[g][n][j] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
#pragma unroll
            for (int g = 0; g < NG; g++) {
                uint32_t b[4];      // entries 0-7 of chunks c, c + 1, then entries 8-15
                pa_ldsm4(kst + C::at((warp * NG + g) * 16 + ri + (mi >> 1) * 8, c + (mi & 1)), b);
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int i = 0; i < 2; i++)
                        mma_f16(x[g][n], qa[c + i][0], qa[c + i][0], qa[c + i][1], qa[c + i][1], f16x2_codes(b[2 * n + i] & 0xffffu),
                                f16x2_codes(b[2 * n + i] >> 16));
            }
        }
        float y[NG][2][2], mx = -INFINITY;
        int we[NG][2][2];                // the values' scales
#pragma unroll
        for (int g = 0; g < NG; g++)
#pragma unroll
            for (int n = 0; n < 2; n++) {
                const int e0 = n * 8 + 2 * tq, at = (warp * NG + g) * 16 + e0;
                const uint32_t k2 = *reinterpret_cast<const uint16_t *>(ks + at), v2 = *reinterpret_cast<const uint16_t *>(vs + at);
                const float2 l2 = has_lm ? *reinterpret_cast<const float2 *>(lm + at) : make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const bool in = e0 + j < nv[g];
                    // 2^(q + k_e), where it is a number: the logit is next to nothing below, out of range above
                    const int t = min(max(qe + (int)((k2 >> (8 * j)) & 255), 1), 254);
                    float v = x[g][n][j] * scale * __uint_as_float((uint32_t)t << 23);
                    we[g][n][j] = (int)((v2 >> (8 * j)) & 255) - 127;
                    if (has_lm) v += pa_lm2(j ? l2.y : l2.x, most);
                    y[g][n][j] = in ? v : -INFINITY;
                    mx = fmaxf(mx, y[g][n][j]);
                }
            }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float mn = fmaxf(m, mx), sh = pa_shift(mn);
        float us = -INFINITY;
#pragma unroll
        for (int g = 0; g < NG; g++)
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    y[g][n][j] -= sh;
                    us = fmaxf(us, y[g][n][j] + (float)we[g][n][j]);
                }
        us = fmaxf(us, __shfl_xor_sync(0xffffffffu, us, 1));
        us = fmaxf(us, __shfl_xor_sync(0xffffffffu, us, 2));
        if (__any_sync(0xffffffffu, mn > m || us > u)) {
            const float by = m - sh;
            m = mn;
            u = fmaxf(u + by, us);
            const int top = u == -INFINITY ? ve : min(max(__float2int_ru(u), -120), 119);
            z *= tc::ex2(by);
            const float w = tc::ex2(by + (float)(ve - top));
            ve = top;
#pragma unroll
            for (int i = 0; i < D / 8; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] *= w;
        }
        uint32_t hi[NG][2], lo[NG][2];
#pragma unroll
        for (int g = 0; g < NG; g++) {
#pragma unroll
            for (int n = 0; n < 2; n++) {
                const float p0 = tc::ex2(y[g][n][0]), p1 = tc::ex2(y[g][n][1]);
                z += p0 + p1;
                // (2^(v_e - E) is a number where p is not 0)
                const float v0 = p0 * 0x1p14f * __uint_as_float((uint32_t)min(max(0, 127 + we[g][n][0] - ve), 254) << 23);
                const float v1 = p1 * 0x1p14f * __uint_as_float((uint32_t)min(max(0, 127 + we[g][n][1] - ve), 254) << 23);
                const __half2 h = __floats2half2_rn(v0, v1);
                const float2 f = __half22float2(h);
                const __half2 r = __floats2half2_rn((v0 - f.x) * 2048.f, (v1 - f.y) * 2048.f);
                hi[g][n] = *reinterpret_cast<const uint32_t *>(&h);
                lo[g][n] = *reinterpret_cast<const uint32_t *>(&r);
            }
        }
#pragma unroll
        for (int i = 0; i < D / 16; i += 2) {
#pragma unroll
            for (int g = 0; g < NG; g++) {
                uint32_t b[4];      // entries 0-7, 8-15 of chunk i, then of i + 1
                pa_ldsm4t(vst + C::at((warp * NG + g) * 16 + ri + (mi & 1) * 8, i + (mi >> 1)), b);
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    // bytes (entry 0, channels 0 1), (entry 1, channels 0 1) -> channel 0 of both, channel 1 of both
                    const uint32_t c0 = __byte_perm(b[2 * k], 0, 0x3120), c1 = __byte_perm(b[2 * k + 1], 0, 0x3120);
                    mma_f16(acc[2 * (i + k)], hi[g][0], lo[g][0], hi[g][1], lo[g][1], f16x2_codes(c0 & 0xffffu), f16x2_codes(c1 & 0xffffu));
                    mma_f16(acc[2 * (i + k) + 1], hi[g][0], lo[g][0], hi[g][1], lo[g][1], f16x2_codes(c0 >> 16), f16x2_codes(c1 >> 16));
                }
            }
        }
    }

    // What the sums are to be multiplied by in the end, 2^(E - 14), goes in two steps that stay in range.
    __device__ __forceinline__ void stats(float *ms, float *zs, float *fs) {
        const int lane = threadIdx.x & 31;
        z += __shfl_xor_sync(0xffffffffu, z, 1);
        z += __shfl_xor_sync(0xffffffffu, z, 2);
        if ((lane & 3) == 0) {
            ms[lane >> 2] = m;
            zs[lane >> 2] = z;
            fs[lane >> 2] = __uint_as_float((uint32_t)(127 + ve - 14 - ((ve - 14) >> 1)) << 23);
        }
    }
    __device__ __forceinline__ void leave(float *sum, int h0, int gq) {
        const int lane = threadIdx.x & 31, hq = lane >> 2, tq = lane & 3;
        if (hq < h0 || hq >= min(gq, h0 + kPaHeads)) return;
        const float f = __uint_as_float((uint32_t)(127 + ((ve - 14) >> 1)) << 23);
#pragma unroll
        for (int c = 0; c < D / 16; c++)
            *reinterpret_cast<float4 *>(sum + (hq - h0) * D + c * 16 + 4 * tq) =
                make_float4((acc[2 * c][0] + acc[2 * c][2] * 0x1p-11f) * f, (acc[2 * c + 1][0] + acc[2 * c + 1][2] * 0x1p-11f) * f,
                            (acc[2 * c][1] + acc[2 * c][3] * 0x1p-11f) * f, (acc[2 * c + 1][1] + acc[2 * c + 1][3] * 0x1p-11f) * f);
    }
};

// fp32: whole tiles of 32 entries, one warp each.  Over quantised pools the key's scale
// multiplies the logit and the value's the weight.
template <typename S, int D, int GQ>
struct PaF32 {
    using C = PaCfg<float, S, D>;
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

    __device__ __forceinline__ void tile(const unsigned char *kst, const unsigned char *vst, const uint8_t *ks,
                                         const uint8_t *vs, const float *lm, int count, unsigned units, int box, bool has_lm,
                                         float most) {
        const int lane = threadIdx.x & 31;
        const bool in = lane < count && ((units >> (lane / box)) & 1u);
        float2 x[GQ];
#pragma unroll
        for (int h = 0; h < GQ; h++) x[h] = make_float2(0.f, 0.f);
        auto product = [&](int c4, float4 k) {
#pragma unroll
            for (int h = 0; h < GQ; h++) {
                const float4 q = *reinterpret_cast<const float4 *>(qs + h * D + c4 * 4);
                x[h] = __ffma2_rn(make_float2(q.x, q.y), make_float2(k.x, k.y), x[h]);
                x[h] = __ffma2_rn(make_float2(q.z, q.w), make_float2(k.z, k.w), x[h]);
            }
        };
        float kscale = 1.f, vscale = 1.f;
        if constexpr (C::QUANT) {
            kscale = in ? scale_of(ks[lane]) : 0.f;
            vscale = in ? scale_of(vs[lane]) : 0.f;
#pragma unroll 2
            for (int ch = 0; ch < D / 16; ch++) {
                const uint4 u = *reinterpret_cast<const uint4 *>(kst + C::at(lane, ch));
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 k0 = values2(w[i] & 0xffffu), k1 = values2(w[i] >> 16);
                    product(ch * 4 + i, make_float4(k0.x, k0.y, k1.x, k1.y));
                }
            }
        } else {
#pragma unroll 8
            for (int ch = 0; ch < D / 4; ch++) product(ch, *reinterpret_cast<const float4 *>(kst + C::at(lane, ch)));
        }
        const float l2 = has_lm ? pa_lm2(lm[lane], most) : 0.f;
#pragma unroll
        for (int h = 0; h < GQ; h++) {
            const float y = in ? (C::QUANT ? (x[h].x + x[h].y) * kscale : x[h].x + x[h].y) + l2 : -INFINITY;
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
            ps[h * 32 + lane] = C::QUANT ? p * vscale : p;
        }
        __syncwarp();
        const unsigned ok = __ballot_sync(0xffffffffu, in);
        // lane's channels: E consecutive ones
        const int ch = lane * E / (16 / (int)sizeof(S)), in_chunk = lane * E * (int)sizeof(S) & 15;
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
                const unsigned char *r = vst + C::at(e, ch) + in_chunk;
                if constexpr (C::QUANT) {
#pragma unroll
                    for (int i = 0; i < E / 2; i++) v[i] = values2(*reinterpret_cast<const uint16_t *>(r + i * 2));
                } else {
#pragma unroll
                    for (int i = 0; i < E / 2; i++) v[i] = *reinterpret_cast<const float2 *>(r + i * 8);
                }
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
// SHARED: the plan of a shared prefix is made by the first block, and sequences leave parts to be joined with it.
template <typename T, typename S_, int D, int GQ, bool SHARED>
__global__ void __launch_bounds__(kPaThreads, kPaPerSm)
    paged_attention_kernel(const PaArgsOf<SHARED> a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV) {
    using C = PaCfg<T, S_, D>;
    using SM = PaSmem<C::NST, C::TE, C::QUANT>;
    extern __shared__ __align__(1024) unsigned char dsm[];
    unsigned char *ring = dsm;                                   // [NST][keys, values]
    float *sum = reinterpret_cast<float *>(dsm + C::NST * 2 * C::TB);        // bf16: [warps][kPaHeads][D]; fp32: [8][D]
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
    const int nblocks = (int)gridDim.x - SHARED, block = (int)blockIdx.x - SHARED;
    if constexpr (SHARED) {
        static_assert(sizeof(PlanSmem<kPaThreads>) <= kPaRing / 2, "plan");
        if (block < 0) {
            make_plan<kPaThreads>(a.shared, *reinterpret_cast<PlanSmem<kPaThreads> *>(dsm));
            return;
        }
    }

    // ---- the CTA's run: tiles of all sequences, and where its own begin.  On the line that is cut a sequence has LEAD
    // places in front of its tiles: it begins and ends in the time of about 128 entries.  (256 requests of about 100
    // entries in 8 heads: without, the last CTA is done after 51 us, of 12 sequences, the first after 26, of one; the whole
    // with 0 / 128 / 192 / 256 entries 85.7 / 82.2 / 83.5 / 85.6 us.)
    constexpr int LEAD = SHARED || C::QUANT ? 128 / C::TE : 0;
    auto places = [&](int n) { return n > 0 ? (n + C::TE - 1) / C::TE + LEAD : 0; };
    const int seg = (S + kPaThreads - 1) / kPaThreads;
    long long mine = 0;
    int most = 0;
    for (int s = tid * seg; s < min(S, (tid + 1) * seg); s++) {
        const int n = pa_len(a, s);
        if (n < a.lens[s]) atomicOr(a.status, kStRange);
        mine += places(n);
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
    const bool snap = most <= C::SNAP;
    // A run holds MIN tiles at least, and as many as leave the longest sequence kPaPieces pieces: one CTA
    // joins them, eight or sixteen at a time.  (16000 entries of 2 sequences: 14.9 us with runs of 2 or 4
    // tiles, 16.4 of 8; 60000 entries of one head: 22.4 us in 64 pieces, 24.7 in 128; 2000 entries of 8
    // sequences: 11.0 of 2 tiles, 11.8 of 4, 14.4 of 8; fp32, 1000 entries of 10 in tiles of 32: 11.5 of 1,
    // 12.7 of 2, 14.0 of 4.)
    const int least = max(C::MIN, (most + kPaPieces - 1) / kPaPieces);
    const int nc = total <= kPaNarrow ? min(nblocks, (int)(((uint32_t)total + least - 1) / (uint32_t)least))
                                      : (int)min((long long)nblocks, (total + least - 1) / least);
    // short sequences and a CTA for each: no CTA gets two (32 x 8 sequences of 200 entries: 13 us with two in some, 9 so)
    const bool each = (SHARED || C::QUANT) && snap && S <= nblocks, one = each && block < S && pa_len(a, block) > 0;
    const long long lo = each ? (one ? 0 : total) : block < nc ? pa_run_first(block, total, nc) : total;
    const long long hi = each ? (one ? 1 : total) : block < nc ? pa_run_first(block + 1, total, nc) : total;
    if (each) {
        if (tid == 0) {
            sm.s_first = block;
            sm.first = 0;
        }
    } else if (lo < hi && lo >= before && lo < before + mine) {
        int s = tid * seg;
        for (;; s++) {
            const int n = places(pa_len(a, s));
            if (lo < before + n) break;
            before += n;
        }
        if (snap && lo > before) before += places(pa_len(a, s++));
        sm.s_first = s;
        sm.first = before;
    }
    // sequences without an entry
    for (int s = block; s < S; s += nblocks)
        if (a.lens[s] <= 0) {
            if constexpr (SHARED) {
                if (tid < gq) a.shared.plan.own_mz[(size_t)s * gq + tid] = make_float2(-INFINITY, 0.f);
            } else {
                for (int i = tid; i < gq * D; i += kPaThreads) put(static_cast<T *>(a.out) + (size_t)s * gq * D + i, 0.f);
            }
        }
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
            const int t0 = snap ? 0 : (int)max(lo - vs - LEAD, 0ll), t1 = snap ? nt : (int)min(hi - vs - LEAD, (long long)nt);
            vs += places(n);
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
                const uint32_t bytes = (uint32_t)(2 * C::NB * box * C::BW + (a.c.log_m ? box * 4 : 0) + (C::QUANT ? 2 * box : 0));
                if (lane == 0) {
                    sm.count[st] = min(C::TE, n - t * C::TE);
                    sm.units[st] = units;
                    if (units) tc::mbar_expect_tx(fb, bytes * __popc(units));
                    else tc::mbar_arrive(fb);
                }
                __syncwarp();
                if (have) {
                    const uint32_t kb = tc::smem_u32(ring + st * 2 * C::TB) + (uint32_t)(u * box * C::BW);
#pragma unroll
                    for (int b = 0; b < C::NB; b++) {
                        tc::tma_load_2d(kb + (uint32_t)(b * C::TE * C::BW), &mapK, b * (C::BW / (int)sizeof(S_)), r, fb);
                        tc::tma_load_2d(kb + (uint32_t)(C::TB + b * C::TE * C::BW), &mapV, b * (C::BW / (int)sizeof(S_)), r, fb);
                    }
                    if constexpr (C::QUANT) {
                        pa_bulk(tc::smem_u32(&sm.ks[st][u * box]), a.scales.k + r, (uint32_t)box, fb);
                        pa_bulk(tc::smem_u32(&sm.vs[st][u * box]), a.scales.v + r, (uint32_t)box, fb);
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
    typename std::conditional<C::BF, typename std::conditional<C::QUANT, PaE4<D>, PaBf<D>>::type, PaF32<S_, D, GQ>>::type w;
    if constexpr (!C::BF) {
        w.qs = qs;
        w.ps = qs + GQ * D + warp * GQ * 32;
    }
    constexpr float kMost = SHARED ? kShMost : FLT_MAX;      // masks meet those of a shared prefix
    uint32_t it = 0;
    long long vs = sm.first;
    for (int s = sm.s_first; s < S && vs < hi; s++) {
        const int n = pa_len(a, s), nt = (n + C::TE - 1) / C::TE;
        if (nt == 0) continue;
        const long long ve = vs + nt + LEAD;
        const int t0 = snap ? 0 : (int)max(lo - vs - LEAD, 0ll), t1 = snap ? nt : (int)min(hi - vs - LEAD, (long long)nt);
        if (t0 >= t1) { vs = ve; continue; }             // its tiles begin in the next run
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
            const uint8_t *ks = sm.ks[C::QUANT ? st : 0], *vsc = sm.vs[C::QUANT ? st : 0];
            if constexpr (C::BF)
                w.tile(tc::smem_u32(base), tc::smem_u32(base + C::TB), ks, vsc, sm.lm[st], sm.count[st], sm.units[st], box,
                       a.scale, a.c.log_m != nullptr, kMost);
            else
                w.tile(base, base + C::TB, ks, vsc, sm.lm[st], sm.count[st], sm.units[st], box, a.c.log_m != nullptr, kMost);
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sm.empty[st]));
        }
        // ---- the piece: the warps' maxima, then their sums in order
        T *out = static_cast<T *>(a.out) + (size_t)s * gq * D;
        const int c_lo = snap ? 0 : pa_run_of(vs + LEAD, total, nc), c_hi = snap ? 0 : pa_run_of(ve - 1, total, nc);
        // slot 2 c: the sequence the CTA continues, 2 c + 1: the one it begins and leaves
        constexpr int PF = pa_part_floats(D);
        float *pp = a.part + (size_t)(2 * block + (block == c_lo)) * PF;
        // four channels of head h, of all heads' from i on
        auto finish = [&](int i, int h, float M, float Z, float4 v) {
            if (c_lo != c_hi) {
                *reinterpret_cast<float4 *>(pp + i) = v;
                if (i % D == 0) { pp[8 * D + h] = M; pp[8 * D + 8 + h] = Z; }
            } else if constexpr (SHARED) {
                *reinterpret_cast<float4 *>(a.shared.plan.own + (size_t)s * gq * D + i) = v;
                if (i % D == 0) a.shared.plan.own_mz[(size_t)s * gq + h] = make_float2(M, Z);
            } else if (Z == 0.f) {                                           // a NaN stays
                put4(out + i, make_float4(0.f, 0.f, 0.f, 0.f));
            } else {
                put4(out + i, make_float4(v.x / Z, v.y / Z, v.z / Z, v.w / Z));
            }
        };
        if constexpr (C::BF) {
            // Every warp leaves its sums, four heads at a time, and every thread joins four channels of them: two meetings
            // a piece.  (Each warp adding to one sum in turn is six, and 1500 of the 5000 clocks that a sequence of 64
            // entries took; 256 requests of about 100 entries in 8 heads on a prefix: 95 us so, 90 this way.)
            w.stats(sm.m[warp], sm.z[warp], sm.f[C::QUANT ? warp : 0]);
            for (int h0 = 0; h0 < gq; h0 += kPaHeads) {
                if (h0) pa_sync();
                w.leave(sum + warp * kPaHeads * D, h0, gq);
                pa_sync();
                const int i = tid * 4, h = h0 + i / D;
                if (h < min(gq, h0 + kPaHeads)) {
                    float M = -INFINITY, Z = 0.f;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < kPaWarps; k++) M = fmaxf(M, sm.m[k][h]);
#pragma unroll
                    for (int k = 0; k < kPaWarps; k++) {
                        const float g = tc::ex2(sm.m[k][h] - pa_shift(M)), f = C::QUANT ? sm.f[C::QUANT ? k : 0][h] : 1.f;
                        const float4 x = *reinterpret_cast<const float4 *>(sum + k * kPaHeads * D + i);
                        Z += sm.z[k][h] * g;
                        if (C::QUANT) {
                            v.x += g * x.x * f; v.y += g * x.y * f; v.z += g * x.z * f; v.w += g * x.w * f;
                        } else {
                            v.x += g * x.x; v.y += g * x.y; v.z += g * x.z; v.w += g * x.w;
                        }
                    }
                    finish(h0 * D + i, h, M, Z, v);
                }
            }
        } else {
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
            // only the warps that had one of the piece's tiles, from its first stage on
            const int adds = min(kPaF32Warps, t1 - t0), from = (int)((it - (t1 - t0)) % kPaF32Warps);
            for (int i = 0; i < adds; i++) {
                if (warp == (from + i) % kPaF32Warps) w.add(sum, sm.M, gq, i == 0);
                pa_sync();
            }
            for (int i = tid * 4; i < gq * D; i += kPaCons * 4)
                finish(i, i / D, sm.M[i / D], sm.Z[i / D], *reinterpret_cast<const float4 *>(sum + i));
        }
        if (c_lo != c_hi) {
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
                        if constexpr (SHARED) {
                            *reinterpret_cast<float4 *>(a.shared.plan.own + (size_t)s * gq * D + i) = v;
                            if (i % D == 0) a.shared.plan.own_mz[(size_t)s * gq + h] = make_float2(M, Z);
                        } else {
                            const float r = Z == 0.f ? 0.f : 1.f / Z;            // a NaN stays
                            put4(out + i, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
                        }
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

// [rows][D] rows, boxes of [box][128 or 64 bytes] with a swizzle as wide.
template <typename C, typename S>
bool pa_map(CUtensorMap *m, const void *p, int64_t rows, int d, int box) {
    auto enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t gdim[2] = {(cuuint64_t)d, (cuuint64_t)rows};
    cuuint64_t gstr[1] = {(cuuint64_t)d * sizeof(S)};
    cuuint32_t bx[2] = {C::BW / (cuuint32_t)sizeof(S), (cuuint32_t)box};
    cuuint32_t es[2] = {1, 1};
    return enc(m, C::QUANT ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : C::BF ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32,
               2, const_cast<void *>(p), gdim, gstr, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               C::BW == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, typename S, int D, int GQ, bool SHARED>
cudaError_t pa_launch(const PaArgsOf<SHARED> &a, cudaStream_t s) {
    using C = PaCfg<T, S, D>;
    static std::atomic<int> grid_of[kMaxDevices];
    const auto kern = paged_attention_kernel<T, S, D, GQ, SHARED>;
    const size_t smem = (size_t)C::NST * 2 * C::TB + (C::BF ? kPaWarps * kPaHeads : 8) * D * sizeof(float) +
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
    if (!pa_map<C, S>(&mk, a.c.K, rows, D, box) || !pa_map<C, S>(&mv, a.c.V, rows, D, box)) return cudaErrorNotSupported;
    return launch_overlapped(kern, grid, kPaThreads, smem, s, a, mk, mv);
}

template <typename S, int D, bool SHARED>
cudaError_t pa_launch_f32(const PaArgsOf<SHARED> &a, int gq, cudaStream_t s) {
    return gq == 1 ? pa_launch<float, S, D, 1, SHARED>(a, s) : gq == 2 ? pa_launch<float, S, D, 2, SHARED>(a, s)
           : gq <= 4 ? pa_launch<float, S, D, 4, SHARED>(a, s) : pa_launch<float, S, D, 8, SHARED>(a, s);
}

template <bool SHARED>
cudaError_t pa_launch_any(const PaArgsOf<SHARED> &a, const gkv_paged_cache *c, bool quant, cudaStream_t s) {
    const int gq = c->Hq / c->G;
    if (c->dtype == GKV_BF16) {
        if (quant)
            return c->d == 128 ? pa_launch<__nv_bfloat16, E4m3, 128, 8, SHARED>(a, s) : pa_launch<__nv_bfloat16, E4m3, 64, 8, SHARED>(a, s);
        return c->d == 128 ? pa_launch<__nv_bfloat16, __nv_bfloat16, 128, 8, SHARED>(a, s)
                           : pa_launch<__nv_bfloat16, __nv_bfloat16, 64, 8, SHARED>(a, s);
    }
    if (quant) return c->d == 128 ? pa_launch_f32<E4m3, 128, SHARED>(a, gq, s) : pa_launch_f32<E4m3, 64, SHARED>(a, gq, s);
    return c->d == 128 ? pa_launch_f32<float, 128, SHARED>(a, gq, s) : pa_launch_f32<float, 64, SHARED>(a, gq, s);
}

constexpr size_t kPaCntBytes = kPaMaxGrid * sizeof(int);

}  // namespace

namespace serve {

size_t paged_scratch_bytes(int d) { return kPaCntBytes + (size_t)2 * kPaMaxGrid * pa_part_floats(d) * sizeof(float); }

gkv_status paged_attention_call(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l, const void *q, void *out,
                                int *status, void *scratch, const SharedArgs *shared, cudaStream_t s) {
    if (l < 0 || l >= c->L || !q || !out || !al(q, 16) || !al(out, 16)) return GKV_EINVAL;
    if (c->page_size % 16) return GKV_EUNSUPPORTED;
    unsigned char *ws = static_cast<unsigned char *>(scratch);
    PaSharedArgs a{};
    a.c = paged_of(c);
    a.S = c->B * c->G;
    a.lens = c->lens + (int64_t)l * a.S;
    a.table = c->table + (int64_t)l * a.S * c->max_pages;
    a.q = q;
    a.out = out;
    a.status = status;
    a.cnt = reinterpret_cast<int *>(ws);
    a.part = reinterpret_cast<float *>(ws + kPaCntBytes);
    a.box = c->page_size % 64 == 0 ? 64 : c->page_size % 32 == 0 ? 32 : 16;
    a.scale = (float)(1.4426950408889634 / sqrt((double)c->d));
    if (scales) a.scales = *scales;
    if (shared) a.shared = *shared;
    const cudaError_t e = shared ? pa_launch_any<true>(a, c, scales, s) : pa_launch_any<false>(a, c, scales, s);
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

}  // namespace serve
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_paged_workspace_size(const gkv_paged_cache *c, size_t *bytes) {
    const gkv_status st = serve::check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = serve::kWsHead + serve::paged_scratch_bytes(c->d);
    return GKV_OK;
}

extern "C" gkv_status gracekv_paged_attention(const gkv_paged_cache *c, int32_t l, const void *q, void *out,
                                              void *workspace, void *stream) {
    const gkv_status st = serve::check_paged(c);
    if (st != GKV_OK) return st;
    if (!workspace || !serve::al(workspace, 256)) return GKV_EINVAL;
    return serve::paged_attention_call(c, nullptr, l, q, out, static_cast<int *>(workspace),
                                       static_cast<unsigned char *>(workspace) + serve::kWsHead, nullptr,
                                       static_cast<cudaStream_t>(stream));
}

extern "C" gkv_status gracekv_quant_attention(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l, const void *q,
                                              void *out, void *workspace, void *stream) {
    const gkv_status st = serve::check_quant(c, scales);
    if (st != GKV_OK) return st;
    if (!workspace || !serve::al(workspace, 256)) return GKV_EINVAL;
    return serve::paged_attention_call(c, scales, l, q, out, static_cast<int *>(workspace),
                                       static_cast<unsigned char *>(workspace) + serve::kWsHead, nullptr,
                                       static_cast<cudaStream_t>(stream));
}
