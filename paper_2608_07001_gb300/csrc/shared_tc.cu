// shared_tc.cu -- the entries of a shared prefix attended for all its requests
// at once: bf16 rows, on tcgen05 (shared_attention.cu has the whole).
//
// A CTA takes a piece: the gq query heads of up to `tok` requests (two row tiles
// of 128) over a run of key tiles of 128 entries of one (slot, KV head).  For a row
// tile
//   S = Q K^T + sqrt(d) log m (fp32 in TMEM), y = S c, c = log2(e) / sqrt(d),
//   P = 2^(y - M), Z += sum P, O += P V,
// with M a reference that follows the running maximum only when that has grown by
// more than 2^kLazy, so that O is rescaled in TMEM a few times instead of once a
// tile; (M, Z, O) of every row leave as the piece's parts.
// log m joins as one more K step of the product, 1 1 1 against its three bf16 parts
// (24 bits), and so does -inf for what no length or page covers: the softmax of a
// thread, which has a row, would otherwise read 128 words of shared memory a tile
// and find the maximum by hand (1650 clocks of 3400), where the load from TMEM
// returns it.
// Two row tiles take every key tile, each with its own softmax warps.  Where the
// requests fill one row tile at most, both warpgroups work on it, each with every
// other key tile and sums of its own, which are two parts.
//
// Few requests: bound by reading the prefix, 64 KB a key tile of d = 128 against two
// products of 128^3; many: by the chain product, exponentials, product of a row tile, of
// which TMEM holds two.  us a key tile and SM, pages of 64 entries, log m; in L2 / from HBM:
//                      one row tile     two row tiles
//   bf16       d = 64  0.96 / 1.07      1.73 / 1.76
//              d = 128 1.32 / 1.60      2.22 / 2.28       (64 KB in 1.60 us: 6.2 TB/s of all SMs)
//   quantised  d = 64  0.99 / 1.10      1.77 / 1.81
//              d = 128 1.40 / 1.55      2.17 / 2.52
// Pages of 16 entries, each box of which is a copy of its own: 1.3 to 1.4, 2.1 to 2.4 (bf16, d = 128) and as above.
// A piece takes about 10 us beside its tiles.
//
// Warps: 0-3 and 4-7 softmax (a thread a row), 8 looks pages up and issues TMA
// (boxes of up to 64 entries that do not cross a page; K and V tiles through a ring)
// and zeroes rows of entries that are not there, which are stale memory (0 times
// what is not finite is NaN), 9 and 10 issue the MMAs of row tile 0 and 1, 11 makes
// the K step of log m.
// A and B of a product have one type, so P goes as its bf16 part and the remainder's, two
// parts (2^-16 of a weight, as the own entries'), each half of them in the columns of its own
// scores.  Rounded once, a key tile of two row tiles took 1.54 us instead of 2.2 (d = 128) and
// 1.44 instead of 1.7 (d = 64), of one 1.19 instead of 1.32 and 0.79 instead of 0.96, from HBM
// 1.59 as it does; but outputs were 2.2 to 2.4e-3 from 64 bits, where rounding them
// makes 1.65e-3.
//
// Quantised pages: codes come through a ring of their own, and two warpgroups more
// (12-15 keys, 16-19 values) write the tiles as f16, 3 clocks for two codes (as bf16 with their scale 8,
// which bounded a tile: 2700 of 5100 clocks).  With k_e, v_e the scales' exponents,
//   K' = code 2^(k_e - k),  V' = code 2^(v_e - E),  y = S 2^q 2^k c,  O 2^E in the end,
// k the largest k_e of the tile, E the largest v_e so far, of entries that have a
// weight at all (no -inf, nor the lowest log m where there is another), q the power of
// two that brings a row's queries into f16 (its largest to 2^14, exact down to 2^-38 of
// that).  Codes stay exact down to 2^-15 of the largest scale and go to 0 at 2^-33 of the
// largest value.  P = 2^(y - M), rounded once, has 11 bits, at most 2^15 and exact to
// 2^-29 of that, its last bit 2^-39 of it.  (A remainder's part beside it, as of bf16: 75
// requests of five contexts 135.6 us instead of 111.3, for a rounding an eighth of the
// output's.)
// Where that would cost keys their bits (k_e that lie further apart in a tile) or log m beside
// q and k is no number (they are beyond 2^30 and 2^40), K' = code and the softmax warps make
// y = S 2^q 2^(k_e) c + log m from the scores themselves, with 128 reads of shared memory.
#include "quant.cuh"
#include "shared.cuh"
#include "tc.cuh"

#include <math.h>

#include <algorithm>
#include <atomic>

namespace gkv {
namespace serve {
namespace {

constexpr int kWarpTma = 8, kWarpMma = 9, kWarpBias = 11, kWarpConv = 12;
constexpr float kLazy = 8.f;                               // log2 of the growth a reference lets pass
constexpr float kHead = 7.f;                               // f16: log2 of where the weights start
constexpr int kNoScale = -120;                             // E before any entry
constexpr int kLeastQ = -100;                              // least q
// How large q and k may be for log m to join in the product: kShMost 2^-q 2^-k is a number and its last bits are too.
// kSpread: how far a key's scale may be below the tile's largest, its code exact in f16 (a key of zeros has the least
// scale there is, and its tile goes the longer way).
constexpr int kMostQ = 30, kMostK = 40, kSpread = 15;
constexpr int kOwn = -127;                                 // k of a tile whose keys keep their own scales (a number's exponent, of 0)
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr uint32_t kNapNs = 20000;                         // a look at a barrier may last that long
constexpr int NK = kShKeysTc;                              // keys of a tile
constexpr int kAhead = 4;                                  // tiles that the words beside the rows are fetched ahead: a window at most
constexpr int NBIAS = 4;                                   // slots of the K step of log m
constexpr uint32_t AUG = NK * 32;                          // its bytes: 16 elements a key
constexpr int NFIX = 8;                                    // more than the tiles that a ring holds
constexpr int kBiased = 1, kSpecial = 2, kFar = 4;         // of a tile: log m; entries that are not there; k = kOwn
constexpr int kGone = 255;                                 // scale byte of an entry that is not there: one that no row has
constexpr int kLowest = 1, kLargest = 2;                   // of a piece: every log m at -kShMost; some at kShMost

template <int D, bool QUANT>
struct Cfg {
    static constexpr int NB = D / 64;                      // 64-channel blocks of a 16-bit row
    static constexpr uint32_t TILE = NB * 128 * 128;       // bytes of a 128-row 16-bit tile
    static constexpr uint32_t RAW = 128 * D;               // bytes of a tile of codes
    // ring slots, 16-bit, of key and of value tiles
    static constexpr int KS = QUANT ? (D == 128 ? 1 : 3) : (D == 128 ? 2 : 5), VS = QUANT && D == 128 ? 2 : KS;
    // ring slots of codes, of either kind, beside two row tiles of queries; one row tile leaves room for one more of each
    static constexpr int NR = QUANT ? (D == 128 ? 1 : 3) : 0;
    static constexpr int PW = QUANT ? 32 : 64;             // TMEM columns of 64 keys' weights: one part or two
    static constexpr int NQA = QUANT ? 2 : 1;              // left sides of the K step: by row, or the same for all
    static constexpr size_t SMEM = (2 + KS + VS) * (size_t)TILE + (NBIAS + NQA) * (size_t)AUG + 2 * NR * (size_t)RAW;
    static constexpr int THREADS = QUANT ? 640 : 384;
    static_assert(KS < NFIX && VS < NFIX && KS + 4 < 2 * NFIX, "fixed tiles");
};

template <int KS, int VS, int NR, bool QUANT>
struct Bars {
    uint64_t kfull[KS], kempty[KS], vfull[VS], vempty[VS], krfull[NR + 1], krempty[NR + 1], vrfull[NR + 1], vrempty[NR + 1], qfull[2], qready[2], sfull[2], pfull[2][2], odone[2];
    uint64_t bfull[NBIAS], bempty[NBIAS], kfix[NFIX], vfix[NFIX], turn[2], fin;
    alignas(16) float lm[QUANT ? NBIAS : 1][QUANT ? NK : 4];             // sqrt(d) log m, -inf for what is not there
    alignas(16) uint8_t ke[QUANT ? NBIAS : 1][QUANT ? NK : 16], ve[QUANT ? NBIAS : 1][QUANT ? NK : 16];       // scale bytes
    float qscale[2][QUANT ? 128 : 1];  // 2^q
    int kind[NBIAS], ktop[NBIAS], vtop[NBIAS];             // k, E
    int far[2];                        // of a row tile: q of some row is beyond kMostQ
    int limit;                         // of the piece
    uint32_t tbase;
    int abort;
};

// Bounded.  What a wait does beyond its first look is a call: inlined, two dozen of them were half of the kernel's code,
// and its roles, which run beside one another, spent most of their time on fetching theirs.
__device__ __forceinline__ bool try_wait_for(uint32_t bar, uint32_t parity, uint32_t ns) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(ns)
        : "memory");
    return ok != 0;
}
__device__ __noinline__ bool wait_long(uint32_t addr, uint32_t parity, int *abort, int *status) {
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t it = 1; !try_wait_for(addr, parity, kNapNs); it++)
        if (!(it & 3u)) {
            if (*(volatile int *)abort) return false;
            if (tc::globaltimer_ns() - t0 > kWaitNs) {
                atomicOr(status, kStTimeout);
                atomicExch(abort, 1);
                return false;
            }
        }
    return true;
}
template <class B>
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, B &b, int *status) {
    const uint32_t addr = tc::smem_u32(bar);
    return tc::mbar_try_wait(addr, parity) || wait_long(addr, parity, &b.abort, status);
}
__device__ __noinline__ int pool_row(const SharedArgs &a, int64_t seq, int64_t e) {
    const Paged look{nullptr, nullptr, nullptr, a.table, nullptr, 0, 0, 0, 0, a.c.page_size, a.c.max_pages, a.c.n_pages};
    return (int)entry_row(look, seq, (int)e, a.status);
}

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two codes as f16 times a scale.
__device__ __forceinline__ uint32_t half2_of(uint32_t c, __half2 s) {
    const uint32_t h = f16x2_codes(c);
    const __half2 x = __hmul2(*reinterpret_cast<const __half2 *>(&h), s);
    return *reinterpret_cast<const uint32_t *>(&x);
}
// 2^e in f16, e <= 0; 0 below its smallest.
__device__ __forceinline__ __half half_pow2(int e) {
    return __ushort_as_half((unsigned short)(e >= -14 ? (e + 15) << 10 : e >= -24 ? 1 << (e + 24) : 0));
}
// Three bf16 parts of x, packed: x = lo(a) + hi(a) + lo(b), to 24 bits; what is not finite in the first.
__device__ __forceinline__ uint2 three_parts(float x) {
    const uint32_t a = bf16x2_of(x, 0.f);
    if (!(fabsf(x) <= FLT_MAX)) return make_uint2(a, 0u);
    const float r = x - __uint_as_float(a << 16);
    const uint32_t b = bf16x2_of(r, 0.f);
    return make_uint2(a | (b << 16), bf16x2_of(r - __uint_as_float(b << 16), 0.f));
}
// The order in which a piece's tiles are taken: L key tiles, then V(j) and K(j + L) in turn; keys and values so far.
__device__ __forceinline__ bool next_is_key(int keys, int values, int L, int n) { return keys < n && keys < values + L; }
// A ring's slot that comes next and its phase.
struct Turn {
    int at = 0;
    uint32_t ph;
    __device__ __forceinline__ explicit Turn(uint32_t first) : ph(first) {}
    __device__ __forceinline__ void step(int slots) {
        if (++at == slots) { at = 0; ph ^= 1; }
    }
};
// Shared-memory descriptors of the K step's operands: rows of 32 bytes, 32-byte swizzle (bit 4 of an address by bit 7).
__device__ __forceinline__ uint64_t aug_desc(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(256 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)6 << 61);
}
// Row r of such an operand: three elements, the others 0.
__device__ __forceinline__ void put_aug(unsigned char *base, int r, uint2 v) {
    const int flip = (r >> 2) & 1;
    *reinterpret_cast<uint4 *>(base + r * 32 + flip * 16) = make_uint4(v.x, v.y, 0u, 0u);
    *reinterpret_cast<uint4 *>(base + r * 32 + (flip ^ 1) * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// The scores of a row (TMEM, 128 columns) become base-2 logits in place: those of which log m could not be a part of the
// product, with each key's own scale (kOwn) or the tile's.  As the attention over quantised pages makes them: 2^(q + k_e)
// where it is a number.
__device__ __noinline__ void far_logits(uint32_t ts, const float *lm, const uint8_t *ke, int kt, float two_q, float c) {
    const int qe = (int)(__float_as_uint(two_q) >> 23) - 127;
#pragma unroll 1
    for (int h = 0; h < NK / 32; h++) {
        uint32_t x[32];
        tc::tmem_ld32_async(ts + 32 * h, x);
        tc::tmem_wait_ld(x);
#pragma unroll
        for (int e = 0; e < 32; e++) {
            const int t = min(max(qe + (kt == kOwn ? (int)ke[32 * h + e] : kt + 127), 1), 254);
            x[e] = __float_as_uint(__uint_as_float(x[e]) * c * __uint_as_float((uint32_t)t << 23) + lm[32 * h + e] * c);
        }
        tc::tmem_st(ts + 32 * h, x);
    }
    tc::tmem_wait_st();
}

template <int D, bool QUANT>
__global__ void __launch_bounds__(Cfg<D, QUANT>::THREADS, 1)
    shared_tc_kernel(const SharedArgs a, const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                     const __grid_constant__ CUtensorMap mapV) {
    using C = Cfg<D, QUANT>;
    // first row tile of queries, key slots, value slots, K steps, second row tile, codes (where there is no second row tile, from its place on)
    extern __shared__ __align__(1024) unsigned char Qs[];
    unsigned char *kring = Qs + C::TILE, *vring = kring + C::KS * C::TILE, *aug = vring + C::VS * C::TILE, *qaug = aug + NBIAS * AUG, *Qs1 = qaug + C::NQA * AUG;
    __shared__ Bars<C::KS, C::VS, C::NR, QUANT> b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    next_may_start();
    if (warp == kWarpMma) {
        tc::tmem_alloc(tc::smem_u32(&b.tbase), 512);
        tc::tmem_relinquish();
    }
    if (warp == kWarpTma && lane == 0) {
        tc::tma_prefetch_desc(&mapQ);
        tc::tma_prefetch_desc(&mapK);
        tc::tma_prefetch_desc(&mapV);
    }
    if (!QUANT && warp == kWarpBias) {                   // 1 1 1 in every row
        for (int r = lane; r < 128; r += 32) put_aug(qaug, r, make_uint2(0x3f803f80u, 0x3f80u));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    after_previous();
    // ---- the piece
    int4 w0 = a.plan.piece[2 * blockIdx.x], w1 = a.plan.piece[2 * blockIdx.x + 1];        // (of a block without one: anything)
    const bool idle = (int)blockIdx.x >= *a.plan.pieces;
    const int gq = a.c.Hq / a.c.G, tpt = a.tok / 2;
    if (idle) w0 = w1 = make_int4(0, 0, 0, 0);
    const int b0 = w0.y, nb = w0.z, len = w0.w, g = w1.x, j0 = w1.y, n = w1.z - w1.y;
    const bool two = nb > tpt;                           // two row tiles
    const int step = two ? 1 : 2, L = step;              // key tiles of a warpgroup; keys ahead of their values
    const int64_t seq = (int64_t)w0.x * a.c.G + g;
    const int box = a.box, per_tile = NK / box;
    const int nr = C::NR + (two ? 0 : 1);                // slots of codes, of either kind
    unsigned char *codes = two ? Qs1 + C::TILE : Qs1;

    if (warp == kWarpTma && lane == 0) {                 // the thread that uses them first
        for (int i = 0; i < C::KS; i++) {
            tc::mbar_init(tc::smem_u32(&b.kfull[i]), QUANT ? 4 : 1);
            tc::mbar_init(tc::smem_u32(&b.kempty[i]), 2);
        }
        for (int i = 0; i < C::VS; i++) {
            tc::mbar_init(tc::smem_u32(&b.vfull[i]), QUANT ? 4 : 1);
            tc::mbar_init(tc::smem_u32(&b.vempty[i]), 2);
        }
        for (int i = 0; i < C::NR + 1; i++) {
            tc::mbar_init(tc::smem_u32(&b.krfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.krempty[i]), 4);
            tc::mbar_init(tc::smem_u32(&b.vrfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.vrempty[i]), 4);
        }
        for (int i = 0; i < 2; i++) {
            tc::mbar_init(tc::smem_u32(&b.qfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.qready[i]), 4);
            tc::mbar_init(tc::smem_u32(&b.sfull[i]), 1);
            for (int k = 0; k < 2; k++) tc::mbar_init(tc::smem_u32(&b.pfull[i][k]), 4);
            tc::mbar_init(tc::smem_u32(&b.odone[i]), 1);
        }
        for (int i = 0; i < NBIAS; i++) {
            tc::mbar_init(tc::smem_u32(&b.bfull[i]), 1);
            // read by the products, and of quantised tiles by the conversion and the softmax warps
            tc::mbar_init(tc::smem_u32(&b.bempty[i]), 2 + (QUANT ? 4 + (two ? 8 : 4) : 0));
        }
        for (int i = 0; i < NFIX; i++) {
            tc::mbar_init(tc::smem_u32(&b.kfix[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.vfix[i]), 1);
        }
        for (int i = 0; i < 2; i++) tc::mbar_init(tc::smem_u32(&b.turn[i]), 1);
        tc::mbar_init(tc::smem_u32(&b.fin), 2);
        b.abort = b.far[0] = b.far[1] = 0;
        tc::fence_barrier_init();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    // pages are looked up before the block meets: boxes of tiles, in windows of 32, one a lane, the next window on its
    // way
    auto box_rows = [&](int w) {
        const int u = w * 32 + lane;
        const int64_t e = (int64_t)j0 * NK + (int64_t)u * box;
        return u < n * per_tile && e < len ? pool_row(a, seq, e) : -1;
    };
    int now = -1, after = -1;
    if (warp == kWarpTma || warp == kWarpBias) {
        now = box_rows(0);
        after = box_rows(1);
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tb = b.tbase;
    if (idle) {
        if (warp == kWarpMma) tc::tmem_dealloc(tb, 512);
        return;
    }

    if (warp < 8) {
        // ---------------- softmax: one thread a row ----------------
        const int i = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const int tk = r / gq, first = two ? i * tpt : 0;
        const bool live = tk < tpt && first + tk < nb;
        const bool work = __any_sync(0xffffffffu, live);
        const uint32_t ts = tb + ((uint32_t)(q * 32) << 16) + i * NK, to = tb + ((uint32_t)(q * 32) << 16) + 2 * NK + i * D;
        const int start = two ? 0 : i;
        float c = a.scale;
        bool far = false;
        int ve = kNoScale;                               // E
        float m = -INFINITY, z = 0.f;                    // the reference and the sum of the weights
        bool ok = true, any = false;
        // A wait that gave up leaves nothing to rely on, but the warp goes on together to the end: every later
        // wait gives up at once, and nothing is written.
        uint32_t ph = 0;
        for (int j = start; j < n; j += step, ph ^= 1) {
            const int sl = j % NBIAS;
            ok = wait(&b.sfull[i], ph, b, a.status) && ok;
            float cs = c;                                // what a score is to be scaled by
            int ve_new = kNoScale;
            if (QUANT) {
                ok = wait(&b.bfull[sl], (j / NBIAS) & 1, b, a.status) && ok;
                if (j == start) {
                    c *= b.qscale[two ? i : 0][QUANT ? r : 0];
                    far = b.far[two ? i : 0];
                }
                const int kt = b.ktop[sl];
                cs = c * __uint_as_float((uint32_t)(127 + kt) << 23);
                ve_new = b.vtop[sl];
                if (work && (far || kt == kOwn)) {
                    tc::tc_fence_after();
                    far_logits(ts, b.lm[sl], b.ke[sl], kt, b.qscale[two ? i : 0][QUANT ? r : 0], a.scale);
                    cs = 1.f;
                }
            }
            __syncwarp();
            if (QUANT && lane == 0) tc::mbar_arrive(tc::smem_u32(&b.bempty[sl]));
            tc::tc_fence_after();
            auto hand = [&](int k) {
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.pfull[i][k]));
            };
            if (work) {
                // Scores are read twice: for their maximum, which the load returns, and, in halves, for the weights.
                uint32_t x[2][32];
                float top = -INFINITY;
#pragma unroll 1
                for (int h = 0; h < 2; h++) {
                    float mx[2];
                    tc::tmem_ld32_max_async(ts + 64 * h, x[0], mx[0]);
                    tc::tmem_ld32_max_async(ts + 64 * h + 32, x[1], mx[1]);
                    tc::tmem_wait_ld(x[0]);
                    tc::tmem_loaded(x[1]);
                    tc::tmem_loaded(mx[0]);
                    tc::tmem_loaded(mx[1]);
                    top = max3(top, mx[0], mx[1]);
                }
                top = __fadd_rn(__fmul_rn(top, cs), QUANT ? -kHead : 0.f);
                const bool grow = m != -INFINITY && top > m + kLazy;
                if (m == -INFINITY) m = top;             // no weight so far
                if (__any_sync(0xffffffffu, grow) || (QUANT && ve_new != ve)) {
                    // S(j) was issued after the last product into O, so that one is done
                    float w = grow ? tc::ex2(m - top) : 1.f;
                    z *= w;
                    if (grow) m = top;
                    if (QUANT) {
                        w *= __uint_as_float((uint32_t)min(max(0, 127 + ve - ve_new), 254) << 23);       // (E falls beside w = 0 alone)
                        ve = ve_new;
                    }
                    if (any) {
#pragma unroll 1
                        for (int k = 0; k < D / 32; k++) {
                            tc::tmem_ld32_async(to + 32 * k, x[0]);
                            tc::tmem_wait_ld(x[0]);
#pragma unroll
                            for (int e = 0; e < 32; e++) x[0][e] = __float_as_uint(__uint_as_float(x[0][e]) * w);
                            tc::tmem_st(to + 32 * k, x[0]);
                        }
                    }
                }
                const float sh = m == -INFINITY ? 0.f : -m;
                float2 acc = make_float2(0.f, 0.f);
                uint32_t pk[32], rest[QUANT ? 1 : 32];
#pragma unroll 1
                for (int h = 0; h < 2; h++) {
                    tc::tmem_ld32_async(ts + 64 * h, x[0]);
                    tc::tmem_ld32_async(ts + 64 * h + 32, x[1]);
                    tc::tmem_wait_ld(x[0]);
                    tc::tmem_loaded(x[1]);
#pragma unroll
                    for (int e = 0; e < 32; e++) {
                        // scaled and shifted in two roundings, as the reference was: of scores of any size the largest gives 1
                        // (products and sums of pairs would be fused whatever they are called)
                        const float2 y = make_float2(__fadd_rn(__fmul_rn(__uint_as_float(x[e / 16][2 * e & 31]), cs), sh),
                                                     __fadd_rn(__fmul_rn(__uint_as_float(x[e / 16][(2 * e & 31) + 1]), cs), sh));
                        const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
                        acc = __fadd2_rn(acc, w);
                        if constexpr (QUANT) {
                            pk[e] = f16x2_of(w.x, w.y);
                        } else {
                            pk[e] = bf16x2_of(w.x, w.y);
                            const float2 r = __ffma2_rn(make_float2(__uint_as_float(pk[e] << 16), __uint_as_float(pk[e] & 0xffff0000u)),
                                                        make_float2(-1.f, -1.f), w);
                            rest[e] = bf16x2_of(r.x, r.y);
                        }
                    }
                    tc::tmem_st(ts + C::PW * h, pk);
                    if constexpr (!QUANT) tc::tmem_st(ts + C::PW * h + 32, rest);
                    hand(h);
                }
                z += acc.x + acc.y;
            } else {
                hand(0);
                hand(1);
            }
            any = true;
        }
        if (any) ok = wait(&b.odone[i], 0, b, a.status) && ok;
        ok = __all_sync(0xffffffffu, ok);
        tc::tc_fence_after();
        // a part: [D / 4][rows] sums of 4 channels, then [rows] references, [rows] sums of weights
        float *pp = a.plan.part + (2 * (size_t)blockIdx.x + i) * shared_part_floats(true, D);
        if (ok && work) {
            if (any) {
#pragma unroll 1
                for (int k = 0; k < D / 32; k += 2) {
                    uint32_t u[2][32];
                    tc::tmem_ld32_async(to + 32 * k, u[0]);
                    tc::tmem_ld32_async(to + 32 * k + 32, u[1]);
                    tc::tmem_wait_ld(u[0]);
                    tc::tmem_loaded(u[1]);
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        if constexpr (QUANT) {           // O 2^E, in two steps that stay in range
                            const int h = ve >> 1;
                            const float f0 = __uint_as_float((uint32_t)(127 + h) << 23), f1 = __uint_as_float((uint32_t)(127 + ve - h) << 23);
#pragma unroll
                            for (int e = 0; e < 32; e++) u[x][e] = __float_as_uint(__uint_as_float(u[x][e]) * f0 * f1);
                        }
                        if (live) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<uint4 *>(pp + ((size_t)((k + x) * 8 + e / 4) * kShRowsTc + r) * 4) =
                                    make_uint4(u[x][e], u[x][e + 1], u[x][e + 2], u[x][e + 3]);
                        }
                    }
                }
            }
            if (live) {
                // log m at the limit has come through the product, its scale and back: off by a few last bits, which are
                // 2^17 there.  The reference becomes what the own entries and the other parts have; of other logits, of
                // any size, it stays as it is.
                if ((b.limit & (m < 0.f ? kLowest : kLargest)) && fabsf(fabsf(m) - kShMost) <= kShMost * 0x1p-20f) m = copysignf(kShMost, m);
                pp[(size_t)kShRowsTc * D + r] = m;
                pp[(size_t)kShRowsTc * (D + 1) + r] = z;
            }
        }
    } else if (warp < kWarpConv) {
        const bool one = tc::elect_one();
        bool ok = true;
        if (warp == kWarpTma) {
            // ---------------- copies of key and value tiles ----------------
            if (lane == 0) {
                for (int i = 0; i < (two ? 2 : 1); i++) {
                    const uint32_t qb = tc::smem_u32(&b.qfull[i]);
                    tc::mbar_expect_tx(qb, (uint32_t)(C::NB * tpt * gq * 128));
#pragma unroll
                    for (int cb = 0; cb < C::NB; cb++)
                        tc::tma_load_3d(tc::smem_u32((i ? Qs1 : Qs) + cb * 128 * 128), &mapQ, cb * 64, g * gq, b0 + i * tpt, qb);
                }
            }
            __syncwarp();
            const int lp = 31 - __clz(per_tile), ks = QUANT ? nr : C::KS, vs = QUANT ? nr : C::VS;       // per_tile = 2^lp
            const unsigned whole = (1u << per_tile) - 1;
            const uint32_t bytes = (uint32_t)(box * D * (QUANT ? 1 : 2)), stepb = (uint32_t)(box * (QUANT ? D : 128));
            const uint32_t slot = QUANT ? C::RAW : C::TILE, kbase = tc::smem_u32(QUANT ? codes : kring),
                           vbase = tc::smem_u32(QUANT ? codes + nr * C::RAW : vring);
            uint64_t *const kf = QUANT ? b.krfull : b.kfull, *const vf = QUANT ? b.vrfull : b.vfull;
            uint64_t *const ke = QUANT ? b.krempty : b.kempty, *const ve = QUANT ? b.vrempty : b.vempty;
            // rows of this window, the one before it and the one after it, and which of them are there
            int before = -1, window = 0, jk = 0, jv = 0;
            unsigned v_before = 0, v_now = __ballot_sync(0xffffffffu, now >= 0);
            Turn kt(1), vt(1);
            // d = 64: a round takes V(j) and K(j + L), lane 0 sees to the key tile's barriers, lane 1 to the value tile's, as
            // it is the steps of this one warp that bound a piece of few rows (a tile at a time 2100 clocks a key tile, so
            // 1500 to 1800).  At d = 128 a tile a round: with rings of two each, waiting for both slots at once loses more
            // (16 requests on 131072 entries 132 us instead of 114).
            constexpr bool PAIR = D == 64;
            while (ok && jv < n) {
                const bool is_key = next_is_key(jk, jv, L, n);
                const bool has_k = PAIR ? jk < n : is_key, has_v = PAIR ? jk >= L || jk == n : !is_key;
                const int wk = jk >> (5 - lp), uk = (jk << lp) & 31, uv = (jv << lp) & 31;
                if (has_k && wk > window) {              // the first key tile of its window
                    before = now;
                    v_before = v_now;
                    now = after;
                    v_now = __ballot_sync(0xffffffffu, now >= 0);
                    after = box_rows(++window + 1);
                }
                const bool v_old = (jv >> (5 - lp)) < window;
                const int rows = v_old ? before : now;   // of the value tile
                const unsigned k_units = has_k ? (v_now >> uk) & whole : 0u, v_units = has_v ? ((v_old ? v_before : v_now) >> uv) & whole : 0u;
                const bool mine_v = lane & 1, has = mine_v ? has_v : has_k;
                ok = __all_sync(0xffffffffu, !has || wait(mine_v ? ve + vt.at : ke + kt.at, mine_v ? vt.ph : kt.ph, b, a.status));
                if (!ok) break;
                const uint32_t kb = tc::smem_u32(kf + kt.at), vb = tc::smem_u32(vf + vt.at);
                if (lane < 2 && has) {
                    const unsigned units = mine_v ? v_units : k_units;
                    if (units) tc::mbar_expect_tx(mine_v ? vb : kb, bytes * __popc(units));
                    else tc::mbar_arrive(mine_v ? vb : kb);
                }
                __syncwarp();
                // a box a lane: 0-7 of the key tile, 8-15 of the value tile (one lane with a loop over the boxes: pages of 16, quantised
                // d = 128 2.2 us a key tile instead of 1.5, bf16 2.3 instead of 2.0; pages of 64, bf16 1.27 instead of 1.19)
                {
                    const int u = lane & 7;
                    const bool v_lane = lane & 8;
                    const int k_row = __shfl_sync(0xffffffffu, now, (uk + u) & 31), v_row = __shfl_sync(0xffffffffu, rows, (uv + u) & 31);
                    if (lane < 16 && ((v_lane ? v_units : k_units) >> u) & 1u) {
                        const uint32_t to = (v_lane ? vbase + vt.at * slot : kbase + kt.at * slot) + u * stepb;
                        const CUtensorMap *map = v_lane ? &mapV : &mapK;
#pragma unroll
                        for (int cb = 0; cb < (QUANT ? 1 : C::NB); cb++) tc::tma_load_2d(to + cb * 128 * 128, map, cb * 64, v_lane ? v_row : k_row, v_lane ? vb : kb);
                    }
                }
                if (!QUANT) {
                    // Rows of entries that are not there become 0 once the tile has landed (which this warp, having waited
                    // for the slot's last use, is the one to see without mistaking the phase).
                    auto fixed = [&](int j, unsigned units, uint64_t *full, uint32_t parity, unsigned char *tile) {
                        const int count = len - (j0 + j) * NK;
                        if (count >= NK && units == whole) return;
                        ok = __all_sync(0xffffffffu, wait(full, parity, b, a.status)) && ok;
                        for (int i = lane; ok && i < NK * C::NB * 8; i += 32) {
                            const int r = i / (C::NB * 8), cb = i % (C::NB * 8);
                            if (r < count && ((units >> (r / box)) & 1u)) continue;
                            *reinterpret_cast<uint4 *>(tile + (cb >> 3) * (NK * 128) + r * 128 + (cb & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    };
                    if (has_v) fixed(jv, v_units, vf + vt.at, vt.ph ^ 1, vring + vt.at * C::TILE);
                    if (has_k) fixed(jk, k_units, kf + kt.at, kt.ph ^ 1, kring + kt.at * C::TILE);
                    if (lane < 2 && has) tc::mbar_arrive(tc::smem_u32(mine_v ? b.vfix + jv % NFIX : b.kfix + jk % NFIX));
                }
                if (has_k) {
                    jk++;
                    kt.step(ks);
                }
                if (has_v) {
                    jv++;
                    vt.step(vs);
                }
            }
            if (lane == 0) {                             // the copies still in flight land before the block exits
                for (int i = max(0, jk - ks); i < jk; i++) tc::mbar_wait(tc::smem_u32(kf + i % ks), (i / ks) & 1, kWaitNs);
                for (int i = max(0, jv - vs); i < jv; i++) tc::mbar_wait(tc::smem_u32(vf + i % vs), (i / vs) & 1, kWaitNs);
                for (int i = 0; i < (two ? 2 : 1); i++) tc::mbar_wait(tc::smem_u32(&b.qfull[i]), 0, kWaitNs);
            }
        } else if (warp == kWarpBias) {
            // ---------------- log m, masks, scales: four keys a lane ----------------
            struct Four { int row; float4 lm; uint32_t ks, vs; };
            auto load = [&](int row) {
                Four f{row, make_float4(0.f, 0.f, 0.f, 0.f), 0x7f7f7f7fu, 0x7f7f7f7fu};
                if (row >= 0) {
                    if (a.c.log_m) f.lm = *reinterpret_cast<const float4 *>(a.c.log_m + row);
                    if (QUANT) {
                        f.ks = *reinterpret_cast<const uint32_t *>(a.scales.k + row);
                        f.vs = *reinterpret_cast<const uint32_t *>(a.scales.v + row);
                    }
                }
                return f;
            };
            // The first of this lane's keys of tile j, which share a box: of this window or of the one after it.
            const int lp = 31 - __clz(per_tile), in_box = (lane * 4) & (box - 1);
            int window = 0;
            auto key_row = [&](int j) {
                const int src = (j << lp) >> 5 == window ? now : after;
                const int r = __shfl_sync(0xffffffffu, src, ((j << lp) + lane * 4 / box) & 31);
                return r < 0 ? -1 : r + in_box;
            };
            // Into L2 a few tiles ahead: from HBM these words take longer than a tile (d = 64, quantised, one row tile,
            // pages not in L2: 1.45 us a key tile without).
            auto fetch = [&](int row) {
                if (row < 0) return;
                if (a.c.log_m) prefetch_l2(a.c.log_m + row);
                if (QUANT) {
                    prefetch_l2(a.scales.k + row);
                    prefetch_l2(a.scales.v + row);
                }
            };
            const float unscale = kLog2e / a.scale, most = kShMost / a.scale;       // sqrt(d)
            int top_ve = kNoScale;
            float piece_top = -INFINITY;
            bool seen = false;
            // This warp alone sees to every tile's words, one after another, and where requests fill one row tile of d = 64
            // its steps are what bounds a tile: so rows are looked up once, and tiles all of whose entries count (ordinary)
            // pass by what the others need.
            Four cur = load(key_row(0));
            int next[kAhead - 1];                        // rows of the tiles from the next one on
#pragma unroll
            for (int i = 1; i < kAhead; i++) fetch(next[i - 1] = key_row(i));
            for (int j = 0; ok && j < n; j++) {
                const int sl = j % NBIAS;
                const Four f = cur;
                if (((j + 1) << lp) >> 5 > window) {
                    now = after;
                    after = box_rows(++window + 1);
                }
                cur = load(next[0]);                     // on its way: the next tile's words, a later one's into L2
#pragma unroll
                for (int i = 0; i < kAhead - 2; i++) next[i] = next[i + 1];
                fetch(next[kAhead - 2] = key_row(j + kAhead));
                ok = __all_sync(0xffffffffu, wait(&b.bempty[sl], ((j / NBIAS) & 1) ^ 1, b, a.status));
                if (!ok) break;
                const int count = f.row < 0 ? 0 : min(4, len - ((j0 + j) * NK + lane * 4));       // keys that are there
                const float lm[4] = {f.lm.x, f.lm.y, f.lm.z, f.lm.w};
                float v[4] = {f.lm.x * unscale, f.lm.y * unscale, f.lm.z * unscale, f.lm.w * unscale};
                const float low = fminf(fminf(v[0], v[1]), fminf(v[2], v[3]));
                float top = fmaxf(max3(v[0], v[1], v[2]), v[3]);
                const float any_nan = v[0] + v[1] + v[2] + v[3];
                const bool ordinary = __all_sync(0xffffffffu, count >= 4 && low > -most && top < most && any_nan == any_nan);
                bool special = false, far = false;
                uint32_t counts = ~0u, gone = 0;         // bytes: of entries that count, of those that are not there
                if (!ordinary) {
                    special = __any_sync(0xffffffffu, count < 4);
#pragma unroll
                    for (int i = 0; i < 4; i++) v[i] = i >= count ? -INFINITY : fabsf(lm[i]) <= FLT_MAX ? fminf(fmaxf(v[i], -most), most) : lm[i];
                    top = fmaxf(max3(v[0], v[1], v[2]), v[3]);
                    if (QUANT) {
                        // Beside an entry above the lowest log m those of it have no weight, nor a say in the scales; until
                        // there is one they are what there is.
                        const bool beside = seen || __any_sync(0xffffffffu, top > -most);
                        if (beside && !seen) top_ve = kNoScale;
                        seen = beside;
                        if (count < 4) gone = ~0u << 8 * max(count, 0);
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            if (seen && v[i] <= -most) v[i] = -INFINITY;
                            if (v[i] == -INFINITY) counts &= ~(255u << 8 * i);
                        }
                    }
                } else if (QUANT && !seen) {
                    seen = true;
                    top_ve = kNoScale;
                }
                // the piece's largest log m so far, by lane (of the softmax warps' two parts of one row tile together: an
                // entry above the lowest in one of them has all of the weight beside the other's lowest)
                piece_top = fmaxf(piece_top, top);
                if (j == n - 1)
                    b.limit = (__any_sync(0xffffffffu, piece_top > -most) ? 0 : kLowest) | (__any_sync(0xffffffffu, piece_top >= most) ? kLargest : 0);
                if constexpr (QUANT) {                   // the rows' threads make the rest of it
                    auto byte = [](uint32_t w, int i) { return (int)(w >> 8 * i & 255u); };
                    auto largest = [&](uint32_t w) { return max(max(byte(w, 0), byte(w, 1)), max(byte(w, 2), byte(w, 3))); };
                    const uint32_t kw = f.ks | ~counts;
                    const int least = min(min(byte(kw, 0), byte(kw, 1)), min(byte(kw, 2), byte(kw, 3)));
                    const int kb = (int)__reduce_max_sync(0xffffffffu, largest(f.ks & counts)), kt = min(kb, 246) - 127;
                    top_ve = max(top_ve, min((int)__reduce_max_sync(0xffffffffu, largest(f.vs & counts)), 246) - 127);
                    far = __any_sync(0xffffffffu, least < kb - kSpread) || abs(kt) > kMostK;
                    *reinterpret_cast<float4 *>(&b.lm[sl][lane * 4]) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<uint32_t *>(&b.ke[sl][lane * 4]) = f.ks | gone;
                    *reinterpret_cast<uint32_t *>(&b.ve[sl][lane * 4]) = f.vs | gone;
                    if (lane == 0) {
                        b.ktop[sl] = far ? kOwn : kt;
                        b.vtop[sl] = top_ve;
                    }
                } else if (a.c.log_m || special) {
#pragma unroll
                    for (int i = 0; i < 4; i++) put_aug(aug + sl * AUG, lane * 4 + i, three_parts(v[i]));
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                // (of keys with their own scales the rows' threads make that, too)
                if (lane == 0) b.kind[sl] = far ? kFar : (a.c.log_m ? kBiased : 0) | (special ? kSpecial : 0);
                // the key rows that are not there are 0 before the product
                if (special && !QUANT) ok = __all_sync(0xffffffffu, wait(&b.kfix[j % NFIX], (j / NFIX) & 1, b, a.status));
                __syncwarp();
                if (ok && lane == 0) tc::mbar_arrive(tc::smem_u32(&b.bfull[sl]));
            }
        } else {
            // ---------------- MMA issue: one warp a row tile, one lane issues ----------------
            // f16 operands where bf16's have a one: their type's field is 0
            constexpr uint32_t kTypes = tc::idesc_bf16_f32(0, 0) & ~(1u << 4), idA = tc::idesc_bf16_f32(128, NK);
            constexpr uint32_t idS = idA & (QUANT ? ~kTypes : ~0u);
            constexpr uint32_t idO = (tc::idesc_bf16_f32(128, D) & (QUANT ? ~kTypes : ~0u)) | tc::kIdescBmn;
            const int i = warp - kWarpMma, start = two ? 0 : i, qi = two ? i : 0;
            const uint32_t qd = (tc::smem_u32(qi ? Qs1 : Qs) >> 4) | (1u << 16);
            const uint32_t kd = (tc::smem_u32(kring) >> 4) | (1u << 16);
            const uint32_t vd = (tc::smem_u32(vring) >> 4) | ((NK * 128 >> 4) << 16);
            const uint64_t ad = aug_desc(tc::smem_u32(aug)), qad = aug_desc(tc::smem_u32(qaug + (QUANT ? qi : 0) * AUG));
            const uint32_t ts = tb + i * NK, to = tb + 2 * NK + i * D;
            ok = start >= n || wait(QUANT ? &b.qready[qi] : &b.qfull[qi], 0, b, a.status);
            const int joins = QUANT && b.far[qi] ? 0 : kBiased | kSpecial;       // kinds of tiles whose log m joins in the product
            // Both warps walk both rings in their order and release every slot, whoever uses it: a warp that passed over a
            // slot's phase could take the one after it for landed.
            Turn kt(0), vt(0);
            uint32_t pp = 0;                             // phase of the weights
            unsigned fixed = 0;                          // bit j % 32: tile j has rows that are not there
            auto mine = [&](int j) { return two || (j & 1) == i; };
            // Two row tiles: the warps issue O(j), S(j + 1) in turn, so that one row tile's exponentials run beside the
            // other's products.  Issued as they come, both wait for both: bf16 2.40 us a key tile of d = 128 instead of
            // 2.20, 1.95 of d = 64 instead of 1.72; quantised d = 64 1.88, 1.74.  Quantised d = 128 waits for its keys,
            // which have one slot: 2.41, in turn 2.50.
            uint32_t tp = i ^ 1;
            const bool turns = two && !(QUANT && D == 128);
            auto take_turn = [&] {
                if (!turns) return;
                ok = wait(&b.turn[i], tp, b, a.status) && ok;
                tp ^= 1;
            };
            auto pass_turn = [&] {
                if (turns && one) tc::mbar_arrive(tc::smem_u32(&b.turn[i ^ 1]));
            };
            for (int jk = 0, jv = 0; ok && jv < n;) {
                const bool is_key = next_is_key(jk, jv, L, n);
                const int j = is_key ? jk++ : jv++, at = is_key ? kt.at : vt.at;
                ok = wait(is_key ? &b.kfull[at] : &b.vfull[at], is_key ? kt.ph : vt.ph, b, a.status) && ok;
                if (is_key) {
                    const int sl = j % NBIAS;
                    kt.step(C::KS);
                    ok = wait(&b.bfull[sl], (j / NBIAS) & 1, b, a.status) && ok;
                    tc::tc_fence_after();
                    const int kind = b.kind[sl];
                    fixed = (fixed & ~(1u << (j & 31))) | (kind & kSpecial ? 1u << (j & 31) : 0u);
                    if (j == 0) take_turn();
                    if (!ok || !one) continue;
                    if (mine(j)) {
                        const uint32_t ka = kd + at * (C::TILE >> 4);
#pragma unroll
                        for (int cb = 0; cb < C::NB; cb++)
#pragma unroll
                            for (int x = 0; x < 4; x++)
                                tc::mma_bf16_lo(ts, qd + cb * (128 * 128 >> 4) + 2 * x, ka + cb * (NK * 128 >> 4) + 2 * x, idS, (cb | x) != 0);
                        if (kind & joins) tc::mma_bf16(ts, qad, ad + sl * (AUG >> 4), idA, 1);
                        tc::mma_commit(tc::smem_u32(&b.sfull[i]));
                        tc::mma_commit(tc::smem_u32(&b.kempty[at]));
                        tc::mma_commit(tc::smem_u32(&b.bempty[sl]));
                        pass_turn();
                    } else {
                        tc::mbar_arrive(tc::smem_u32(&b.kempty[at]));
                        tc::mbar_arrive(tc::smem_u32(&b.bempty[sl]));
                    }
                    continue;
                }
                vt.step(C::VS);
                if (mine(j)) {
                    const uint32_t va = vd + at * (C::TILE >> 4);
                    if (!QUANT && (fixed >> (j & 31)) & 1u) ok = wait(&b.vfix[j % NFIX], (j / NFIX) & 1, b, a.status) && ok;
#pragma unroll
                    for (int k = 0; k < 2; k++) {        // the weights come in halves
                        ok = wait(&b.pfull[i][k], pp, b, a.status) && ok;
                        if (k == 0) take_turn();
                        tc::tc_fence_after();
                        if (ok && one) {
#pragma unroll
                            for (int x = 0; x < C::PW / 8; x++)
                                tc::mma_bf16_ts_lo(to, ts + k * C::PW + x * 8, va + (k * 4 + x % 4) * (16 * 128 >> 4), idO, j != start || k + x != 0);
                        }
                    }
                    pp ^= 1;
                    if (ok && one) {
                        tc::mma_commit(tc::smem_u32(&b.vempty[at]));
                        if (j + step >= n) {
                            tc::mma_commit(tc::smem_u32(&b.odone[i]));
                            pass_turn();
                        }
                    }
                } else if (ok && one) {
                    tc::mbar_arrive(tc::smem_u32(&b.vempty[at]));
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok && lane == 0) {
                atomicOr(a.status, kStTimeout);
                atomicExch(&b.abort, 1);
            }
            // every operation issued is done before TMEM is freed: one more commit of each covers them
            if (one) tc::mma_commit(tc::smem_u32(&b.fin));
            __syncwarp();
            tc::mbar_wait(tc::smem_u32(&b.fin), 0, kWaitNs);
        }
    } else if constexpr (QUANT) {
        // ---------------- queries and codes to f16: one thread a row ----------------
        // the first warpgroup takes the keys, the second one the values and, as the first product waits for keys and queries,
        // the first row tile of queries
        const int r = (warp & 3) * 32 + lane, wg = (warp - kWarpConv) >> 2;
        for (int i = wg ^ 1; i < (two ? 2 : 1); i += 2) {
            if (!__all_sync(0xffffffffu, wait(&b.qfull[i], 0, b, a.status))) break;
            unsigned char *row = (i ? Qs1 : Qs) + r * 128;
            auto chunk = [&](int ch) { return reinterpret_cast<uint4 *>(row + (ch >> 3) * (128 * 128) + (((ch & 7) ^ (r & 7)) << 4)); };
            float top = 0.f;
            // (3650 clocks of the 19000 of a piece of one tile; 4400 with a chunk at a time)
#pragma unroll 4
            for (int ch = 0; ch < D / 8; ch++) {
                float x[8];
                unpack16(*chunk(ch), x);
                top = fmaxf(top, top_of(x));
            }
            const int qe = top > 0.f ? max((int)(__float_as_uint(top) >> 23) - 127 - 14, kLeastQ) : 0;
            const bool far = r / gq < tpt && (i * tpt + r / gq) < nb && abs(qe) > kMostQ;          // (the other rows may be anything)
            if (far) b.far[i] = 1;
            const float f = __uint_as_float((uint32_t)(127 - qe) << 23);
#pragma unroll 4
            for (int ch = 0; ch < D / 8; ch++) {
                float x[8];
                unpack16(*chunk(ch), x);
                *chunk(ch) = make_uint4(f16x2_of(x[0] * f, x[1] * f), f16x2_of(x[2] * f, x[3] * f), f16x2_of(x[4] * f, x[5] * f),
                                        f16x2_of(x[6] * f, x[7] * f));
            }
            b.qscale[i][r] = __uint_as_float((uint32_t)(127 + qe) << 23);
            const uint32_t ff = bf16x2_of(f, f);         // log m is scaled up with the row's scores
            put_aug(qaug + i * AUG, r, make_uint2(ff, ff & 0xffffu));
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.qready[i]));
        }
        Turn from(0), into(1);
        const bool keys = wg == 0;
        const int slots = keys ? C::KS : C::VS;
        unsigned char *const ring = keys ? kring : vring, *const raw = codes + (keys ? 0 : nr * C::RAW);
        bool ok = true;
        for (int j = 0; j < n; j++) {
            const int sl = j % NBIAS, at = from.at, to = into.at;
            ok = wait(keys ? &b.krfull[at] : &b.vrfull[at], from.ph, b, a.status) && ok;
            ok = wait(&b.bfull[sl], (j / NBIAS) & 1, b, a.status) && ok;
            ok = __all_sync(0xffffffffu, wait(keys ? &b.kempty[to] : &b.vempty[to], into.ph, b, a.status) && ok);
            if (!ok) break;
            from.step(nr);
            into.step(slots);
            // codes of entries that are not there may be anything, NaN too; those without a weight have a scale of 0, and a
            // NaN of theirs stays
            const float lm = b.lm[QUANT ? sl : 0][QUANT ? r : 0];
            const int top = keys ? b.ktop[sl] : b.vtop[sl], kind = b.kind[sl];
            const bool far = keys && (kind & kFar);      // codes as they are
            const int byte = (keys ? b.ke : b.ve)[QUANT ? sl : 0][QUANT ? r : 0], e = far ? 0 : min(byte - 127, 119) - top;
            const __half2 s = __half2half2(lm != -INFINITY ? half_pow2(e) : __ushort_as_half(0));
            const bool there = byte != kGone;
            if (keys && kind && !far) put_aug(aug + sl * AUG, r, three_parts(lm * __uint_as_float((uint32_t)(127 - top) << 23)));
            const unsigned char *src = raw + at * C::RAW + r * D;
            unsigned char *dst = ring + to * C::TILE + r * 128;
#pragma unroll
            for (int ch = 0; ch < D / 16; ch++) {
                const int c16 = D == 128 ? ch ^ (r & 7) : ch ^ ((r >> 1) & 3);
                uint4 u = *reinterpret_cast<const uint4 *>(src + c16 * 16);
                if (!there) u = make_uint4(0, 0, 0, 0);
                unsigned char *d = dst + (ch >> 2) * (128 * 128);
                const int c8 = (ch & 3) * 2;
                *reinterpret_cast<uint4 *>(d + ((c8 ^ (r & 7)) << 4)) =
                    make_uint4(half2_of(u.x & 0xffffu, s), half2_of(u.x >> 16, s), half2_of(u.y & 0xffffu, s), half2_of(u.y >> 16, s));
                *reinterpret_cast<uint4 *>(d + (((c8 + 1) ^ (r & 7)) << 4)) =
                    make_uint4(half2_of(u.z & 0xffffu, s), half2_of(u.z >> 16, s), half2_of(u.w & 0xffffu, s), half2_of(u.w >> 16, s));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(tc::smem_u32(keys ? &b.kfull[to] : &b.vfull[to]));
                tc::mbar_arrive(tc::smem_u32(keys ? &b.krempty[at] : &b.vrempty[at]));
                if (!keys) tc::mbar_arrive(tc::smem_u32(&b.bempty[sl]));
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        tc::tc_fence_after();
        tc::tmem_dealloc(tb, 512);
    }
}

// [B][Hq][D] queries: boxes of 64 channels x gq heads x tpt requests; [rows][D] pools: boxes of `box` entries.
bool map_q(CUtensorMap *m, const void *p, int B, int Hq, int d, int gq, int tpt) {
    auto enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t gdim[3] = {(cuuint64_t)d, (cuuint64_t)Hq, (cuuint64_t)B};
    cuuint64_t gstr[2] = {(cuuint64_t)d * 2, (cuuint64_t)Hq * d * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)gq, (cuuint32_t)tpt};
    cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), gdim, gstr, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <bool QUANT>
bool map_pool(CUtensorMap *m, const void *p, int64_t rows, int d, int box) {
    auto enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t gdim[2] = {(cuuint64_t)d, (cuuint64_t)rows};
    cuuint64_t gstr[1] = {(cuuint64_t)d * (QUANT ? 1 : 2)};
    cuuint32_t bx[2] = {QUANT ? (cuuint32_t)d : 64, (cuuint32_t)box};
    cuuint32_t es[2] = {1, 1};
    return enc(m, QUANT ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), gdim, gstr, bx,
               es, CU_TENSOR_MAP_INTERLEAVE_NONE, QUANT && d == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool QUANT>
cudaError_t launch(const SharedArgs &a, cudaStream_t s) {
    using C = Cfg<D, QUANT>;
    const auto kern = shared_tc_kernel<D, QUANT>;
    const int gq = a.c.Hq / a.c.G;
    const int64_t rows = a.c.n_pages * a.c.page_size;
    CUtensorMap mq, mk, mv;
    if (!map_q(&mq, a.q, a.B, a.c.Hq, D, gq, a.tok / 2) || !map_pool<QUANT>(&mk, a.c.K, rows, D, a.box) ||
        !map_pool<QUANT>(&mv, a.c.V, rows, D, a.box))
        return cudaErrorNotSupported;
    static std::atomic<int> ready[kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev].store(1, std::memory_order_relaxed);
    }
    return launch_overlapped(kern, dim3((unsigned)shared_pieces(true, a.blocks)), C::THREADS, C::SMEM, s, a, mq, mk, mv);
}

}  // namespace

cudaError_t launch_shared_tc(const SharedArgs &a, int d, bool quant, cudaStream_t s) {
    if (quant) return d == 128 ? launch<128, true>(a, s) : launch<64, true>(a, s);
    return d == 128 ? launch<128, false>(a, s) : launch<64, false>(a, s);
}

}  // namespace serve
}  // namespace gkv
