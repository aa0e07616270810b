// shared_tc.cu -- the entries of a shared prefix attended for all its requests
// at once: bf16 rows, on tcgen05 (shared_attention.cu has the whole).
//
// A CTA takes a piece: the gq query heads of up to `tok` requests (two row tiles
// of 128) over a run of key tiles of 128 entries of one (slot, KV head).  For a row
// tile
//   S = Q K^T (fp32 in TMEM), y = S c + log m log2(e), c = log2(e) / sqrt(d),
//   P = 2^(y - M), Z += sum P, O += P V,
// with M a reference that follows the running maximum only when that has grown by
// more than 2^kLazy, so that O is rescaled in TMEM a few times instead of once a
// tile; (M, Z, O) of every row leave as the piece's parts.
// Two row tiles take every key tile, each with its own softmax warps.  Where the
// requests fill one row tile at most, both warpgroups work on it, each with every
// other key tile and sums of its own, which are two parts.
//
// Few requests: bound by reading the prefix, 64 KB a key tile of d = 128 against two
// products of 128^3; many: by the tensor pipe and the 128^2 exponentials a tile.
//
// Warps: 0-3 and 4-7 softmax (a thread a row), 8 looks pages up and issues TMA
// (boxes of up to 64 entries that do not cross a page; K and V tiles through a ring,
// log m through a ring of its own) and zeroes V rows of entries that are not there,
// which are stale memory (0 times what is not finite is NaN), 9 and 10 issue the MMAs
// of row tile 0 and 1, 11 turns log m into base 2 and masks what no page or length
// covers.  Quantised pages: codes come through a ring of their own, and a
// warpgroup more (12-15) writes the tiles as bf16, code times scale, exactly: from
// there on nothing differs.
// P is rounded to bf16 once, as A and B of a product have one type; Z is not.
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
constexpr float kLazy = 8.f;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int NK = kShKeysTc;                              // keys of a tile
constexpr int NBIAS = 4;                                   // slots of log m

template <int D, bool QUANT>
struct Cfg {
    static constexpr int NB = D / 64;                      // 64-channel blocks of a bf16 row
    static constexpr uint32_t TILE = NB * 128 * 128;       // bytes of a 128-row bf16 tile
    static constexpr uint32_t RAW = 128 * D;               // bytes of a tile of codes
    static constexpr int NST = QUANT ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 10);       // ring slots, bf16
    static constexpr int NR = QUANT ? (D == 128 ? 3 : 6) : 1;                          // ring slots, codes
    static constexpr size_t SMEM = 2 * (size_t)TILE + NST * (size_t)TILE + (QUANT ? NR * (size_t)RAW : 0);
    static constexpr int THREADS = QUANT ? 512 : 384;
    // Registers a thread at launch, then of the softmax, issue and conversion warps; the sums agree.
    static constexpr int REGS = QUANT ? 128 : 168, RSOFT = QUANT ? 184 : 208, RISSUE = QUANT ? 64 : 88, RCONV = 80;
    static_assert(256 * RSOFT + 128 * RISSUE + (QUANT ? 128 * RCONV : 0) <= THREADS * REGS, "register split");
};

template <int NST, int NR>
struct Bars {
    uint64_t full[NST], empty[NST], rfull[NR], rempty[NR], qfull[2], sfull[2], pfull[2][2], odone[2];
    uint64_t lfull[NBIAS], bfull[NBIAS], bempty[NBIAS], vfix[NBIAS], fin;
    alignas(16) float bias[NBIAS][NK];
    alignas(16) uint8_t rscale[NR][NR > 1 ? NK : 16];
    unsigned units[NBIAS];             // boxes of the tile that were read
    int special[NBIAS];                // some key of the tile is not there
    unsigned runits[NR];
    int rcount[NR];                    // entries of the stage's tile up to the sequence's end
    uint32_t tbase;
    int abort;
};

template <class B>
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, B &b, int *status) {
    const uint32_t addr = tc::smem_u32(bar);
    uint64_t t0 = 0;
    for (uint32_t it = 1; !tc::mbar_try_wait(addr, parity); it++)
        if (!(it & 63u)) {
            const uint64_t t = tc::globaltimer_ns();
            if (t0 == 0) t0 = t;
            if (*(volatile int *)&b.abort) return false;
            if (t - t0 > kWaitNs) {
                atomicOr(status, kStTimeout);
                atomicExch(&b.abort, 1);
                return false;
            }
        }
    return true;
}

__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ void bulk(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
                 : "memory");
}
// log m in base 2: finite values stay finite, the others what they are.
__device__ __forceinline__ float log2_m(float lm) {
    return fabsf(lm) <= FLT_MAX ? fminf(fmaxf(lm * kLog2e, -FLT_MAX), FLT_MAX) : lm;
}

template <int D, bool QUANT>
__global__ void __launch_bounds__(Cfg<D, QUANT>::THREADS, 1)
    shared_tc_kernel(const SharedArgs a, const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                     const __grid_constant__ CUtensorMap mapV) {
    using C = Cfg<D, QUANT>;
    constexpr int NST = C::NST, NR = C::NR;
    extern __shared__ __align__(1024) unsigned char Qs[];
    unsigned char *ring = Qs + 2 * C::TILE, *codes = ring + NST * C::TILE;
    __shared__ Bars<NST, NR> b;
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
    after_previous();
    // ---- the piece
    const bool idle = (int)blockIdx.x >= *a.plan.pieces;
    const int gq = a.c.Hq / a.c.G, tpt = a.tok / 2;
    int4 w0 = make_int4(0, 0, 0, 0), w1 = w0;
    if (!idle) {
        w0 = a.plan.piece[2 * blockIdx.x];
        w1 = a.plan.piece[2 * blockIdx.x + 1];
    }
    const int p = w0.x, b0 = w0.y, nb = w0.z, len = w0.w, g = w1.x, j0 = w1.y, n = w1.z - w1.y;
    const bool two = nb > tpt;                           // two row tiles
    const int step = two ? 1 : 2, L = step;              // key tiles of a warpgroup; keys ahead of their values
    const int64_t seq = (int64_t)p * a.c.G + g;
    const int box = a.box, per_tile = NK / box;

    if (warp == kWarpTma && lane == 0) {                 // the thread that uses them first
        for (int i = 0; i < NST; i++) {
            tc::mbar_init(tc::smem_u32(&b.full[i]), QUANT ? 4 : 1);
            tc::mbar_init(tc::smem_u32(&b.empty[i]), 2);
        }
        for (int i = 0; i < NR; i++) {
            tc::mbar_init(tc::smem_u32(&b.rfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.rempty[i]), 4);
        }
        for (int i = 0; i < 2; i++) {
            tc::mbar_init(tc::smem_u32(&b.qfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.sfull[i]), 1);
            for (int k = 0; k < 2; k++) tc::mbar_init(tc::smem_u32(&b.pfull[i][k]), 4);
            tc::mbar_init(tc::smem_u32(&b.odone[i]), 1);
        }
        for (int i = 0; i < NBIAS; i++) {
            tc::mbar_init(tc::smem_u32(&b.lfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.bfull[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.vfix[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.bempty[i]), two ? 8 : 4);
        }
        tc::mbar_init(tc::smem_u32(&b.fin), 2);
        b.abort = 0;
        tc::fence_barrier_init();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
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
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::RSOFT));
        // ---------------- softmax: one thread a row ----------------
        const int i = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const int tk = r / gq, first = two ? i * tpt : 0;
        const bool live = tk < tpt && first + tk < nb;
        const bool work = __any_sync(0xffffffffu, live);
        const float c = a.scale;
        const uint32_t ts = tb + ((uint32_t)(q * 32) << 16) + i * NK, to = tb + ((uint32_t)(q * 32) << 16) + 2 * NK + i * D;
        const int start = two ? 0 : i;
        float m = -INFINITY, z = 0.f;                    // the reference and the sum of the weights
        bool ok = true, any = false;
        // A wait that gave up leaves nothing to rely on, but the warp goes on together to the end: every later
        // wait gives up at once, and nothing is written.
        uint32_t ph = 0;
        for (int j = start; j < n; j += step, ph ^= 1) {
            const int sl = j % NBIAS;
            ok = wait(&b.sfull[i], ph, b, a.status) && ok;
            ok = wait(&b.bfull[sl], (j / NBIAS) & 1, b, a.status) && ok;
            __syncwarp();
            tc::tc_fence_after();
            auto hand = [&](int k) {
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.pfull[i][k]));
            };
            if (work) {
                uint32_t x[4][32];
#pragma unroll
                for (int k = 0; k < 4; k++) tc::tmem_ld32_async(ts + 32 * k, x[k]);
                tc::tmem_wait_ld(x[0]);
#pragma unroll
                for (int k = 1; k < 4; k++) tc::tmem_loaded(x[k]);
                const float4 *bias = reinterpret_cast<const float4 *>(b.bias[sl]);
                float mx = -INFINITY;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const float2 c2 = make_float2(c, c);
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 u = bias[k * 8 + e / 4];
                        const float2 y0 = __ffma2_rn(make_float2(__uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1])), c2, make_float2(u.x, u.y));
                        const float2 y1 = __ffma2_rn(make_float2(__uint_as_float(x[k][e + 2]), __uint_as_float(x[k][e + 3])), c2, make_float2(u.z, u.w));
                        x[k][e] = __float_as_uint(y0.x);
                        x[k][e + 1] = __float_as_uint(y0.y);
                        x[k][e + 2] = __float_as_uint(y1.x);
                        x[k][e + 3] = __float_as_uint(y1.y);
                        if (e & 8) asm volatile("" ::: "memory");        // no more of log m in registers at once
                    }
                }
                if (b.special[sl]) {                     // keys that are not there: whatever their scores
#pragma unroll
                    for (int k = 0; k < 4; k++)
#pragma unroll
                        for (int e = 0; e < 32; e++) {
                            if (b.bias[sl][k * 32 + e] == -INFINITY) x[k][e] = 0xff800000u;
                            if ((e & 7) == 7) asm volatile("" ::: "memory");
                        }
                }
#pragma unroll
                for (int k = 0; k < 4; k++)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) mx = max3(mx, __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
                const bool grow = m != -INFINITY && mx > m + kLazy;
                if (m == -INFINITY) m = mx;              // no weight so far
                if (__any_sync(0xffffffffu, grow)) {
                    // S(j) was issued after the last product into O, so that one is done
                    const float w = grow ? tc::ex2(m - mx) : 1.f;
                    z *= w;
                    if (grow) m = mx;
                    if (any) {
#pragma unroll
                        for (int k = 0; k < D / 32; k++) {
                            uint32_t o[32];
                            tc::tmem_ld32_async(to + 32 * k, o);
                            tc::tmem_wait_ld(o);
#pragma unroll
                            for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * w);
                            tc::tmem_st(to + 32 * k, o);
                        }
                    }
                }
                const float sh = m == -INFINITY ? 0.f : -m;
                const float2 s2 = make_float2(sh, sh);
                float2 acc = make_float2(0.f, 0.f);
                uint32_t pk[32];
#pragma unroll
                for (int h = 0; h < 2; h++) {
#pragma unroll
                    for (int e = 0; e < 32; e++) {
                        const int at = h * 64 + 2 * e;
                        const float2 y = __fadd2_rn(make_float2(__uint_as_float(x[at / 32][at & 31]), __uint_as_float(x[at / 32][(at & 31) + 1])), s2);
                        const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
                        acc = __fadd2_rn(acc, w);
                        pk[e] = bf16x2_of(w.x, w.y);
                    }
                    tc::tmem_st(ts + 32 * h, pk);
                    hand(h);
                }
                z += acc.x + acc.y;
            } else {
                hand(0);
                hand(1);
            }
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.bempty[sl]));
            any = true;
        }
        if (any) ok = wait(&b.odone[i], 0, b, a.status) && ok;
        ok = __all_sync(0xffffffffu, ok);
        tc::tc_fence_after();
        // a part: [D / 4][rows] sums of 4 channels, then [rows] references, [rows] sums of weights
        float *pp = a.plan.part + (2 * (size_t)blockIdx.x + i) * shared_part_floats(true, D);
        if (ok && work) {
            if (any) {
#pragma unroll
                for (int k = 0; k < D / 32; k++) {
                    uint32_t u[32];
                    tc::tmem_ld32_async(to + 32 * k, u);
                    tc::tmem_wait_ld(u);
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<uint4 *>(pp + ((size_t)(k * 8 + e / 4) * kShRowsTc + r) * 4) =
                                make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                    }
                }
            }
            if (live) {
                pp[(size_t)kShRowsTc * D + r] = m;
                pp[(size_t)kShRowsTc * (D + 1) + r] = z;
            }
        }
    } else if (warp < kWarpConv) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::RISSUE));
        if (warp == kWarpTma) {
            // ---------------- producer ----------------
            if (lane == 0) {
                for (int i = 0; i < (two ? 2 : 1); i++) {
                    const uint32_t qb = tc::smem_u32(&b.qfull[i]);
                    tc::mbar_expect_tx(qb, (uint32_t)(C::NB * tpt * gq * 128));
#pragma unroll
                    for (int cb = 0; cb < C::NB; cb++)
                        tc::tma_load_3d(tc::smem_u32(Qs + i * C::TILE + cb * 128 * 128), &mapQ, cb * 64, g * gq, b0 + i * tpt, qb);
                }
            }
            struct Window { int held0 = 0, held = 0, row = -1; } win[2];          // boxes looked up, one a lane: of keys, of values
            const Paged look{nullptr, nullptr, nullptr, a.table, nullptr, 0, 0, 0, 0, a.c.page_size, a.c.max_pages, a.c.n_pages};
            // pool rows of tile j's boxes, in lanes 0 .. per_tile - 1
            auto rows_of = [&](Window &w, int j) {
                const int u0 = (j0 + j) * per_tile;
                if (u0 < w.held0 || u0 + per_tile > w.held0 + w.held) {
                    w.held0 = u0;
                    w.held = 32;
                    const int64_t e = (int64_t)(u0 + lane) * box;
                    w.row = e < len && u0 + lane < (j0 + n) * per_tile ? (int)entry_row(look, seq, (int)e, a.status) : -1;
                }
                return __shfl_sync(0xffffffffu, w.row, (u0 - w.held0 + lane) & 31);
            };
            int issued = 0;
            bool ok = true;
            auto next = [&](const CUtensorMap &map, Window &w, int j, const uint8_t *scales) {
                const int row = rows_of(w, j);
                const bool have = lane < per_tile && row >= 0;
                const unsigned units = __ballot_sync(0xffffffffu, have);
                const int st = issued % (QUANT ? NR : NST);
                const uint32_t par = ((issued / (QUANT ? NR : NST)) & 1) ^ 1;
                ok = __all_sync(0xffffffffu, !*(volatile int *)&b.abort && wait(QUANT ? &b.rempty[st] : &b.empty[st], par, b, a.status));
                if (!ok) return;
                const uint32_t fb = tc::smem_u32(QUANT ? &b.rfull[st] : &b.full[st]);
                const uint32_t bytes = QUANT ? (uint32_t)(box * (D + 1)) : (uint32_t)(C::NB * box * 128);
                if (lane == 0) {
                    if (QUANT) {
                        b.runits[st] = units;
                        b.rcount[st] = min(NK, len - (j0 + j) * NK);
                    }
                    if (units) tc::mbar_expect_tx(fb, bytes * __popc(units));
                    else tc::mbar_arrive(fb);
                }
                __syncwarp();
                if (have) {
                    if (QUANT) {
                        tc::tma_load_2d(tc::smem_u32(codes + st * C::RAW + lane * box * D), &map, 0, row, fb);
                        bulk(tc::smem_u32(&b.rscale[st][lane * box]), scales + row, (uint32_t)box, fb);
                    } else {
#pragma unroll
                        for (int cb = 0; cb < C::NB; cb++)
                            tc::tma_load_2d(tc::smem_u32(ring + st * C::TILE + cb * 128 * 128 + lane * box * 128), &map, cb * 64, row, fb);
                    }
                }
                issued++;
            };
            int biased = 0;
            auto key = [&](int j) {
                next(mapK, win[0], j, a.scales.k);
                if (!ok) return;
                // the tile's log m, and which of its keys are there
                const int row = rows_of(win[0], j), sl = j % NBIAS;
                const bool have = lane < per_tile && row >= 0;
                const unsigned units = __ballot_sync(0xffffffffu, have);
                ok = __all_sync(0xffffffffu, wait(&b.bempty[sl], ((j / NBIAS) & 1) ^ 1, b, a.status));
                if (!ok) return;
                const uint32_t lb = tc::smem_u32(&b.lfull[sl]);
                if (lane == 0) {
                    b.units[sl] = units;
                    if (units && a.c.log_m) tc::mbar_expect_tx(lb, (uint32_t)(box * 4 * __popc(units)));
                    else tc::mbar_arrive(lb);
                }
                __syncwarp();
                if (have && a.c.log_m) bulk(tc::smem_u32(&b.bias[sl][lane * box]), a.c.log_m + row, (uint32_t)(box * 4), lb);
                biased++;
            };
            for (int j = 0; ok && j < min(L, n); j++) key(j);
            for (int j = 0; ok && j < n; j++) {
                next(mapV, win[1], j, a.scales.v);
                if (ok && !QUANT) {
                    // V rows of entries that are not there: 0, once the tile has landed (which this warp, having waited
                    // for the slot's last use, is the one to see without mistaking the phase)
                    const int count = min(NK, len - (j0 + j) * NK), row = rows_of(win[1], j), st = (issued - 1) % NST;
                    const unsigned units = __ballot_sync(0xffffffffu, lane < per_tile && row >= 0);
                    if (count < NK || units != (1u << per_tile) - 1) {
                        ok = __all_sync(0xffffffffu, wait(&b.full[st], ((issued - 1) / NST) & 1, b, a.status));
                        if (!ok) break;
                        for (int i = lane; i < NK * C::NB * 8; i += 32) {
                            const int r = i / (C::NB * 8), cb = i % (C::NB * 8);
                            if (r < count && ((units >> (r / box)) & 1u)) continue;
                            *reinterpret_cast<uint4 *>(ring + st * C::TILE + (cb >> 3) * (NK * 128) + r * 128 + (cb & 7) * 16) =
                                make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.vfix[j % NBIAS]));
                }
                if (ok && j + L < n) key(j + L);
            }
            // the copies still in flight land before the block exits
            if (lane == 0) {
                constexpr int N = QUANT ? NR : NST;
                for (int i = max(0, issued - N); i < issued; i++)
                    tc::mbar_wait(tc::smem_u32(QUANT ? &b.rfull[i % N] : &b.full[i % N]), (i / N) & 1, kWaitNs);
                for (int i = max(0, biased - NBIAS); i < biased; i++)
                    tc::mbar_wait(tc::smem_u32(&b.lfull[i % NBIAS]), (i / NBIAS) & 1, kWaitNs);
                for (int i = 0; i < (two ? 2 : 1); i++) tc::mbar_wait(tc::smem_u32(&b.qfull[i]), 0, kWaitNs);
            }
        } else if (warp == kWarpBias) {
            // ---------------- log m, masks, stale values ----------------
            for (int j = 0; j < n; j++) {
                const int sl = j % NBIAS;
                if (!__all_sync(0xffffffffu, wait(&b.lfull[sl], (j / NBIAS) & 1, b, a.status))) break;
                const unsigned units = b.units[sl];
                const int count = min(NK, len - (j0 + j) * NK), k0 = lane * 4;
                const bool there = (units >> (k0 / box)) & 1u;                     // a box holds whole fours
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (a.c.log_m && there) {
                    v = *reinterpret_cast<const float4 *>(&b.bias[sl][k0]);
                    v = make_float4(log2_m(v.x), log2_m(v.y), log2_m(v.z), log2_m(v.w));
                }
                if (!there || k0 >= count) v.x = -INFINITY;
                if (!there || k0 + 1 >= count) v.y = -INFINITY;
                if (!there || k0 + 2 >= count) v.z = -INFINITY;
                if (!there || k0 + 3 >= count) v.w = -INFINITY;
                *reinterpret_cast<float4 *>(&b.bias[sl][k0]) = v;
                const bool special = __any_sync(0xffffffffu, !there || k0 + 3 >= count);
                if (lane == 0) b.special[sl] = special;
                // before the weights, and so before the product that they enter
                if (special && !QUANT && !__all_sync(0xffffffffu, wait(&b.vfix[sl], (j / NBIAS) & 1, b, a.status))) break;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.bfull[sl]));
            }
        } else {
            // ---------------- MMA issue: one warp a row tile, one lane issues ----------------
            constexpr uint32_t idS = tc::idesc_bf16_f32(128, NK), idO = tc::idesc_bf16_f32(128, D) | tc::kIdescBmn;
            const int i = warp - kWarpMma, start = two ? 0 : i, qi = two ? i : 0;
            const uint32_t qd = ((tc::smem_u32(Qs) >> 4) | (1u << 16)) + qi * (C::TILE >> 4);
            const uint32_t kd = (tc::smem_u32(ring) >> 4) | (1u << 16);
            const uint32_t vd = (tc::smem_u32(ring) >> 4) | ((NK * 128 >> 4) << 16);
            const uint32_t ts = tb + i * NK, to = tb + 2 * NK + i * D;
            const bool one = tc::elect_one();
            bool ok = start >= n || wait(&b.qfull[qi], 0, b, a.status);
            // Both warps walk the ring in its order and release every slot, whoever uses it: a warp that passed over a
            // slot's phase could take the one after it for landed.
            int st = 0;
            uint32_t ph = 0, pp = 0;                     // of the slot that comes next; of the weights
            auto arrived = [&] {
                ok = wait(&b.full[st], ph, b, a.status) && ok;
                tc::tc_fence_after();
                const int at = st;
                if (++st == NST) { st = 0; ph ^= 1; }
                return at;
            };
            auto mine = [&](int j) { return two || (j & 1) == i; };
            auto key = [&](int j) {
                const int at = arrived();
                if (!ok || !one) return;
                if (mine(j)) {
                    const uint32_t ka = kd + at * (C::TILE >> 4);
#pragma unroll
                    for (int cb = 0; cb < C::NB; cb++)
#pragma unroll
                        for (int x = 0; x < 4; x++)
                            tc::mma_bf16_lo(ts, qd + cb * (128 * 128 >> 4) + 2 * x, ka + cb * (NK * 128 >> 4) + 2 * x, idS, (cb | x) != 0);
                    tc::mma_commit(tc::smem_u32(&b.sfull[i]));
                    tc::mma_commit(tc::smem_u32(&b.empty[at]));
                } else {
                    tc::mbar_arrive(tc::smem_u32(&b.empty[at]));
                }
            };
            for (int j = 0; j < min(L, n); j++) key(j);
            for (int j = 0; ok && j < n; j++) {
                const int at = arrived();
                if (mine(j)) {
                    const uint32_t va = vd + at * (C::TILE >> 4);
#pragma unroll
                    for (int k = 0; k < 2; k++) {        // the weights come in halves
                        ok = wait(&b.pfull[i][k], pp, b, a.status) && ok;
                        tc::tc_fence_after();
                        if (ok && one) {
#pragma unroll
                            for (int x = k * 4; x < k * 4 + 4; x++)
                                tc::mma_bf16_ts_lo(to, ts + x * 8, va + x * (16 * 128 >> 4), idO, j != start || x != 0);
                        }
                    }
                    pp ^= 1;
                    if (ok && one) {
                        tc::mma_commit(tc::smem_u32(&b.empty[at]));
                        if (j + step >= n) tc::mma_commit(tc::smem_u32(&b.odone[i]));
                    }
                } else if (ok && one) {
                    tc::mbar_arrive(tc::smem_u32(&b.empty[at]));
                }
                if (ok && j + L < n) key(j + L);
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::RCONV));
        // ---------------- codes to bf16: one thread a row ----------------
        const int r = (warp - kWarpConv) * 32 + lane;
        for (int s = 0; s < 2 * n; s++) {
            const int rs = s % NR, st = s % NST;
            bool ok = wait(&b.rfull[rs], (s / NR) & 1, b, a.status);
            ok = wait(&b.empty[st], ((s / NST) & 1) ^ 1, b, a.status) && ok;
            if (!__all_sync(0xffffffffu, ok)) break;
            const bool there = r < b.rcount[rs] && ((b.runits[rs] >> (r / box)) & 1u);
            const float sc = there ? scale_of(b.rscale[rs][r]) : 0.f;
            const unsigned char *src = codes + rs * C::RAW + r * D;
            unsigned char *dst = ring + st * C::TILE + r * 128;
#pragma unroll
            for (int ch = 0; ch < D / 16; ch++) {
                const int from = D == 128 ? ch ^ (r & 7) : ch ^ ((r >> 1) & 3);
                uint4 u = *reinterpret_cast<const uint4 *>(src + from * 16);
                if (!there) u = make_uint4(0, 0, 0, 0);
                auto two_of = [&](uint32_t c) {
                    const float2 v = values2(c);
                    return bf16x2_of(v.x * sc, v.y * sc);
                };
                const uint4 lo = make_uint4(two_of(u.x & 0xffffu), two_of(u.x >> 16), two_of(u.y & 0xffffu), two_of(u.y >> 16));
                const uint4 hi = make_uint4(two_of(u.z & 0xffffu), two_of(u.z >> 16), two_of(u.w & 0xffffu), two_of(u.w >> 16));
                unsigned char *d = dst + (ch >> 2) * (128 * 128);
                const int at = (ch & 3) * 2;
                *reinterpret_cast<uint4 *>(d + ((at ^ (r & 7)) << 4)) = lo;
                *reinterpret_cast<uint4 *>(d + (((at + 1) ^ (r & 7)) << 4)) = hi;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(tc::smem_u32(&b.full[st]));
                tc::mbar_arrive(tc::smem_u32(&b.rempty[rs]));
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
        cudaFuncAttributes at;
        e = cudaFuncGetAttributes(&at, kern);
        if (e != cudaSuccess) return e;
        if (at.numRegs != C::REGS) return cudaErrorInvalidConfiguration;       // the register split would not add up
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev].store(1, std::memory_order_relaxed);
    }
    return launch_overlapped(kern, dim3((unsigned)shared_pieces(a.blocks)), C::THREADS, C::SMEM, s, a, mq, mk, mv);
}

}  // namespace

cudaError_t launch_shared_tc(const SharedArgs &a, int d, bool quant, cudaStream_t s) {
    if (quant) return d == 128 ? launch<128, true>(a, s) : launch<64, true>(a, s);
    return d == 128 ? launch<128, false>(a, s) : launch<64, false>(a, s);
}

}  // namespace serve
}  // namespace gkv
