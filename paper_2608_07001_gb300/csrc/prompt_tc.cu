// prompt_tc.cu -- the prompt's attention for bf16 on tcgen05.
//
// For the 256 rows of a CTA (two tiles of 128; a row is a query token and one
// of the gq heads that share a KV head, so a tile holds 128 / gq tokens and
// every key tile is read once for all gq heads):
//   S = Q K^T (fp32 in TMEM), P = 2^(S c - M c), c = log2(e) / sqrt(d),
//   O += P V, Z += sum P, out = O / Z, lse = M / sqrt(d) + ln Z.
// M is a row's reference, not its exact maximum: it follows the running maximum
// only when that has grown by more than 2^kLazy, so the accumulator in TMEM is
// rescaled a few times instead of once a key tile; P stays below 2^kLazy, and O
// and Z share the reference, so the quotient is the same.
//
// What bounds it: at d = 128 a 128 x 128 tile costs 2 x 128^3 MACs in each of
// the two products against 128^2 exponentials, so the tensor pipe; at d = 64
// the exponentials weigh twice as much.  The two row tiles alternate: while the
// tensor core works on one's S and PV, the other's warps take its softmax.
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1 (one thread a row, its 128 scores
// in registers), 8 TMA (Q once, then K and V tiles of 128 keys through a ring),
// 9 and 10 MMA issue of tile 0 and 1 (11 idle: registers are split by
// warpgroup).  TMEM: S0, S1 (128 columns each; P overlays the lower half of
// its S as packed bf16), O0, O1.  P is the A operand of its product from TMEM;
// V is the B operand as it lies in memory (rows of channels, "MN-major").
// tcgen05 operations of one thread complete in order, so the commit of S(j + 1)
// also tells that PV(j) is done: the rescaling needs no barrier of its own.
//
// Measured (32 / 8 heads): 16384 tokens of d = 128 1.24 to 1.36 ms by the power
// limit, 1.62 to 1.78 PFLOP/s of 1.88 that a plain matrix product reaches, the
// tensor pipe 72 % busy at 8192 tokens; 12000 tokens of d = 64 0.53 ms, 1.12
// PFLOP/s (0.56 ms with the maximum taken in registers: 64 instructions a tile,
// which tcgen05.ld.red, a load that also returns its largest value, saves).  Tried for d = 64 and slower: key tiles of 64 with two or three
// score buffers a row tile, four row tiles a CTA, two threads a row.
//
// Few blocks (a short chunk over a long cache) leave SMs idle: then a block's
// keys are split into parts (prompt.cuh) that prompt.cu joins.
//
// Masks: only the tiles that reach past a row's last key compare columns; the
// keys past a sequence's end get weight 0 that way, and their V rows, which
// may hold anything, are zeroed in shared memory before the product.
#include "prompt.cuh"
#include "tc.cuh"

#include <math.h>

#include <algorithm>
#include <atomic>

namespace gkv {
namespace serve {
namespace {

constexpr int kN = kKeysTc;
constexpr int kThreads = 384;                  // three warpgroups: two of softmax, one of TMA and MMA issue
// Registers a thread after the split; 256 x 208 + 128 x 88 = 384 x 168, the launch's own.
constexpr int kRegs = 168, kRegsSoftmax = 208, kRegsIssue = 88;
static_assert(256 * kRegsSoftmax + 128 * kRegsIssue <= kThreads * kRegs, "register split");
constexpr int kWarpTma = 8, kWarpMma = 9;      // MMA: warps 9 and 10, one a row tile
constexpr float kLazy = 8.f;                   // log2 of the growth a reference lets pass
constexpr uint64_t kWaitNs = 2000000000ull;

template <int D>
struct Cfg {
    static constexpr int NB = D / 64;                          // 64-channel blocks of a row
    static constexpr uint32_t TILE = NB * 128 * 128;           // bytes of a 128-row tile
    static constexpr int NST = (D == 128 ? 5 : 8);             // ring slots (K and V tiles in turn)
    static constexpr size_t SMEM = 1024 + (2 + NST) * (size_t)TILE;
};

struct Bars {
    uint64_t full[8], empty[8], qfull, sfull[2], pfull[2][2], odone[2], vfix, fin;
    uint32_t tbase;
    int abort, turn;           // turn: key tiles whose products row tile 0 has issued
};

struct Tc {
    int gq, tpt;               // heads of a KV head, tokens of a row tile
    int kh, vh;                // head coordinate step of k, v (0: one head for all)
};

__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, Bars &b, int *status) {
    const uint32_t addr = tc::smem_u32(bar);
    if (tc::mbar_try_wait(addr, parity)) return true;
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t it = 0;; it++) {
        if (tc::mbar_try_wait(addr, parity)) return true;
        if ((it & 63u) == 63u) {
            if (*(volatile int *)&b.abort) return false;
            if (tc::globaltimer_ns() - t0 > kWaitNs) {
                atomicOr(status, kStTimeout);
                atomicExch(&b.abort, 1);
                return false;
            }
        }
    }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_tc_kernel(const PromptArgs a, const Tc t, const __grid_constant__ CUtensorMap mapQ,
                     const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char raw[];
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) &
                                                            ~static_cast<uintptr_t>(1023));
    unsigned char *Qs = base, *ring = base + 2 * C::TILE;
    __shared__ Bars b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    next_may_start();
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::NST; i++) {
            tc::mbar_init(tc::smem_u32(&b.full[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.empty[i]), 2);
        }
        tc::mbar_init(tc::smem_u32(&b.qfull), 1);
        tc::mbar_init(tc::smem_u32(&b.vfix), 1);
        tc::mbar_init(tc::smem_u32(&b.fin), 2);
        for (int i = 0; i < 2; i++) {
            tc::mbar_init(tc::smem_u32(&b.sfull[i]), 1);
            for (int k = 0; k < 2; k++) tc::mbar_init(tc::smem_u32(&b.pfull[i][k]), 4);
            tc::mbar_init(tc::smem_u32(&b.odone[i]), 1);
        }
        b.abort = 0;
        b.turn = 0;
        tc::fence_barrier_init();
    }
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
    if (blockIdx.x == 0 && blockIdx.y == 0) check_bounds(a);
    // ---- the CTA's rows: heavy blocks (late tokens) first
    const int g = blockIdx.x % a.G;
    const int tok = 2 * t.tpt;
    const int64_t slot = prompt_slots(a.n_q, a.n_seqs, tok) - 1 - blockIdx.x / a.G;
    const int s = slot_seq(a.cu_q, a.n_seqs, slot, tok);
    int64_t q0, nq64, k0, nk64;
    const bool fits = seq_bounds(a, s, q0, nq64, k0, nk64);
    const int64_t t0_64 = (slot - (q0 / tok + s)) * tok;
    const int nq = (int)nq64, nk = (int)nk64, t0 = (int)t0_64;
    const int off = nk - nq;                             // query i sees keys <= i + off
    const int ntile = t0 + t.tpt < nq ? 2 : 1;
    // key tiles of each row tile, up to the last key its last token sees; of
    // them this part's: [j0, j0 + n)
    const int last0 = min(nq, t0 + t.tpt) - 1 + off, last1 = min(nq, t0 + 2 * t.tpt) - 1 + off;
    const int all0 = last0 >= 0 ? last0 / kN + 1 : 0, all1 = ntile > 1 && last1 >= 0 ? last1 / kN + 1 : 0;
    const int all = max(all0, all1), np = parts_of(all, a.split, kLeastTc);
    const int j0 = (int)((int64_t)blockIdx.y * all / np), j1 = (int)((int64_t)(blockIdx.y + 1) * all / np), n = j1 - j0;
    const int nkv0 = max(0, min(all0, j1) - j0), nkv1 = max(0, min(all1, j1) - j0);

    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tb = b.tbase;
    // nothing to do: a sequence that does not fit, a slot past its tokens, a part beyond the block's
    if (!fits || t0_64 < 0 || t0_64 >= nq64 || (int)blockIdx.y >= np) {
        if (warp == kWarpMma) tc::tmem_dealloc(tb, 512);
        return;
    }

    // the sequence's last key tile is partial and other rows follow it: their V rows are zeroed
    const int keep = nk - (j1 - 1) * kN;                  // keys of the sequence in the part's last tile, from it on
    const bool fix = n > 0 && keep < kN && k0 + nk < a.n_k;

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        // ---------------- softmax and epilogue: one thread a row ----------------
        const int i = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const int tk = r / t.gq, h = r - tk * t.gq;
        const int token = t0 + i * t.tpt + tk;
        const bool live = tk < t.tpt && token < nq;
        const int lim = live ? token + off : -1;         // last key the row sees
        const float c = a.scale * kLog2e;
        const uint32_t ts = tb + ((uint32_t)(q * 32) << 16) + (uint32_t)(i * kN), to = tb + ((uint32_t)(q * 32) << 16) + 2 * kN + i * D;
        // the first token of the tile sees the fewest keys: below its limit no mask is needed
        const int clear = t0 + i * t.tpt + off;
        float m = -INFINITY, z = 0.f;                    // m: the reference times c
        const int nj = i ? nkv1 : nkv0;
        bool ok = true;
        for (int j = 0; j < nj; j++) {
            ok = __all_sync(0xffffffffu, wait(&b.sfull[i], j & 1, b, a.status));
            if (!ok) break;
            tc::tc_fence_after();
            uint32_t x[4][32];
            float mx[4];
#pragma unroll
            for (int k = 0; k < 4; k++) tc::tmem_ld32_max_async(ts + 32 * k, x[k], mx[k]);
            tc::tmem_wait_ld(x[0]);
#pragma unroll
            for (int k = 1; k < 4; k++) tc::tmem_loaded(x[k]);
#pragma unroll
            for (int k = 0; k < 4; k++) tc::tmem_loaded(mx[k]);
            if ((j0 + j) * kN + kN - 1 > clear) {
                const int rel = lim - (j0 + j) * kN;
#pragma unroll
                for (int k = 0; k < 4; k++) {
#pragma unroll
                    for (int e = 0; e < 32; e++)
                        if (k * 32 + e > rel) x[k][e] = 0xff800000u;       // -inf
                    mx[k] = fmaxf(__uint_as_float(x[k][0]), __uint_as_float(x[k][1]));
#pragma unroll
                    for (int e = 2; e < 32; e += 2)
                        mx[k] = max3(mx[k], __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
                }
            }
            const float mn = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
            if (m == -INFINITY) m = mn;                  // nothing accumulated yet
            else if (__builtin_expect(mn > m + kLazy, 0)) z = -z;          // asks for a rescale (z > 0 marks none)
            if (__any_sync(0xffffffffu, z < 0.f)) {
                float w = 1.f;
                if (z < 0.f) {
                    w = tc::ex2(m - mn);
                    z = -z * w;
                    m = mn;
                }
#pragma unroll
                for (int k = 0; k < D / 32; k++) {
                    uint32_t o[32];
                    tc::tmem_ld32_async(to + 32 * k, o);
                    tc::tmem_wait_ld(o);
#pragma unroll
                    for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * w);
                    tc::tmem_st32(to + 32 * k, o);
                }
            }
            const float sh = m == -INFINITY ? 0.f : -m;
            const float2 c2 = make_float2(c, c), s2 = make_float2(sh, sh);
            float2 acc = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 2; k++) {
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; e++) {
                    const float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * k + e / 16][(2 * e) & 31]),
                                                            __uint_as_float(x[2 * k + e / 16][((2 * e) & 31) + 1])), c2, s2);
                    const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
                    acc = __fadd2_rn(acc, w);
                    p[e] = pack2(w.x, w.y);
                }
                tc::tmem_st32(ts + 32 * k, p);
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.pfull[i][k]));
            }
            z += acc.x + acc.y;
        }
        if (ok && nj > 0) ok = __all_sync(0xffffffffu, wait(&b.odone[i], 0, b, a.status));
        tc::tc_fence_after();
        const int64_t row = q0 + token;
        const int hq = g * t.gq + h;
        if (np == 1) {
            if (ok && i < ntile) {
                // A thread holds a row, and 32 rows a store are 32 memory sectors: the rows go through
                // shared memory (this warp's rows of Q, which no product reads any more; 16-byte chunks
                // permuted by row) and leave 512 bytes a store.
                constexpr int CH = D / 8;                    // chunks of a row
                const float inv = z > 0.f ? 1.f / z : z;     // no key: 0; a NaN stays
                const int64_t at = live ? row * a.o_ts + hq * a.o_hs : -1;
                unsigned char *stage = Qs + i * C::TILE + q * 32 * (D * 2);
#pragma unroll
                for (int k = 0; k < D / 32; k++) {
                    uint32_t u[32];
                    if (nj > 0) {
                        tc::tmem_ld32_async(to + 32 * k, u);
                        tc::tmem_wait_ld(u);
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (lim >= 0) {
                            v.x = pack2(__uint_as_float(u[e]) * inv, __uint_as_float(u[e + 1]) * inv);
                            v.y = pack2(__uint_as_float(u[e + 2]) * inv, __uint_as_float(u[e + 3]) * inv);
                            v.z = pack2(__uint_as_float(u[e + 4]) * inv, __uint_as_float(u[e + 5]) * inv);
                            v.w = pack2(__uint_as_float(u[e + 6]) * inv, __uint_as_float(u[e + 7]) * inv);
                        }
                        const int ch = k * 4 + e / 8;
                        if (nj > 0) *reinterpret_cast<uint4 *>(stage + lane * (D * 2) + ((ch ^ lane) & (CH - 1)) * 16) = v;
                        else if (live) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at + ch * 8) = v;
                    }
                }
                if (nj > 0) {
                    __syncwarp();
#pragma unroll 4
                    for (int x = 0; x < CH; x++) {
                        const int rr = x * (32 / CH) + lane / CH, ch = lane % CH;
                        const int64_t to_row = __shfl_sync(0xffffffffu, at, rr);
                        const uint4 v = *reinterpret_cast<const uint4 *>(stage + rr * (D * 2) + ((ch ^ rr) & (CH - 1)) * 16);
                        if (to_row >= 0) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + to_row + ch * 8) = v;
                    }
                }
                if (live && a.lse) a.lse[row * a.Hq + hq] = z == 0.f ? -INFINITY : (m + log2f(z)) * 0.6931471805599453f;
            }
        } else {
            // a part: [D / 4][rows] sums of 4 channels, then [rows] references, [rows] sums of weights
            float *pp = a.part + ((size_t)blockIdx.x * a.split + blockIdx.y) * part_floats(kRowsTc, D);
            const int pr = i * 128 + r;
            if (ok && i < ntile) {
#pragma unroll
                for (int k = 0; k < D / 32; k++) {
                    uint32_t u[32];
                    if (nj > 0) {
                        tc::tmem_ld32_async(to + 32 * k, u);
                        tc::tmem_wait_ld(u);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e++) u[e] = 0u;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4 *>(pp + ((size_t)(k * 8 + e / 4) * kRowsTc + pr) * 4) =
                            make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                }
                pp[(size_t)kRowsTc * D + pr] = m;
                pp[(size_t)kRowsTc * (D + 1) + pr] = z;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
        if (warp == kWarpTma) {
            // ---------------- producer ----------------
            int issued = 0;
            bool ok = n > 0;
            if (lane == 0 && ok) {
                const uint32_t qb = tc::smem_u32(&b.qfull);
                tc::mbar_expect_tx(qb, (uint32_t)(ntile * C::NB * t.tpt * t.gq * 128));
                for (int i = 0; i < ntile; i++)
    #pragma unroll
                    for (int c = 0; c < C::NB; c++)
                        tc::tma_load_3d(tc::smem_u32(Qs + i * C::TILE + c * 128 * 128), &mapQ, c * 64, g * t.gq,
                                        (int)(q0 + t0 + i * t.tpt), qb);
                for (int i = 0; i < 2 * n; i++) {
                    const int st = i % C::NST;
                    ok = !*(volatile int *)&b.abort && wait(&b.empty[st], ((i / C::NST) & 1) ^ 1, b, a.status);
                    if (!ok) break;
                    const uint32_t fb = tc::smem_u32(&b.full[st]);
                    tc::mbar_expect_tx(fb, C::TILE);
    #pragma unroll
                    for (int c = 0; c < C::NB; c++)
                        tc::tma_load_3d(tc::smem_u32(ring + st * C::TILE + c * 128 * 128), (i & 1) ? &mapV : &mapK, c * 64,
                                        g * ((i & 1) ? t.vh : t.kh), (int)(k0 + (j0 + (i >> 1)) * kN), fb);
                    issued++;
                }
            }
            issued = __shfl_sync(0xffffffffu, issued, 0);
            ok = issued == 2 * n && n > 0;
            if (fix && ok) {
                const int st = (2 * n - 1) % C::NST;
                if (wait(&b.full[st], ((2 * n - 1) / C::NST) & 1, b, a.status)) {
                    for (int i = lane; i < (kN - keep) * C::NB * 8; i += 32) {
                        const int r = keep + i / (C::NB * 8), c = i % (C::NB * 8);
                        *reinterpret_cast<uint4 *>(ring + st * C::TILE + (c >> 3) * (128 * 128) + r * 128 + (c & 7) * 16) =
                            make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&b.vfix));
                }
            }
            // the copies still in flight land before the block exits
            if (lane == 0 && n > 0) {
                for (int i = max(0, issued - C::NST); i < issued; i++)
                    tc::mbar_wait(tc::smem_u32(&b.full[i % C::NST]), (i / C::NST) & 1, kWaitNs);
                tc::mbar_wait(tc::smem_u32(&b.qfull), 0, kWaitNs);
            }
        } else if (warp <= kWarpMma + 1) {
            // ---------------- MMA issue: one warp a row tile, one lane issues ----------------
            if (n > 0) {
                constexpr uint32_t idS = tc::idesc_bf16_f32(128, kN), idO = tc::idesc_bf16_f32(128, D) | tc::kIdescBmn;
                const int i = warp - kWarpMma, ni = i ? nkv1 : nkv0;
                // descriptors: the start address (16-byte units) is the low word's low end, the rest is constant
                const uint32_t qd = ((tc::smem_u32(Qs) >> 4) | (1u << 16)) + i * (C::TILE >> 4);
                const uint32_t kd = (tc::smem_u32(ring) >> 4) | (1u << 16);
                const uint32_t vd = (tc::smem_u32(ring) >> 4) | ((128 * 128 >> 4) << 16);
                const uint32_t ts = tb + i * kN, to = tb + 2 * kN + i * D;
                const bool one = tc::elect_one();
                int st = 1;
                uint32_t ph = 0;                         // of the ring slot that comes next
                bool ok = wait(&b.qfull, 0, b, a.status) && wait(&b.full[0], 0, b, a.status);
                auto qk = [&](int slot) {                // S = Q K^T, K in the slot
                    const uint32_t ka = kd + slot * (C::TILE >> 4);
#pragma unroll
                    for (int c = 0; c < C::NB; c++)
#pragma unroll
                        for (int x = 0; x < 4; x++)
                            tc::mma_bf16_lo(ts, qd + c * (128 * 128 >> 4) + 2 * x, ka + c * (128 * 128 >> 4) + 2 * x, idS,
                                            (c | x) != 0);
                    tc::mma_commit(tc::smem_u32(&b.sfull[i]));
                };
                tc::tc_fence_after();
                if (ok && one) {
                    if (ni > 0) qk(0);
                    tc::mma_commit(tc::smem_u32(&b.empty[0]));
                }
                ok = __all_sync(0xffffffffu, ok);
                // the row tiles may end at different key tiles: both warps release every slot, in order
                for (int j = 0; ok && j < n; j++) {
                    const int vs = st;
                    const uint32_t vph = ph;
                    if (++st == C::NST) { st = 0; ph ^= 1; }
                    const int ks = st;
                    const uint32_t kph = ph;
                    const bool more = j + 1 < n;
                    ok = wait(&b.full[vs], vph, b, a.status);
                    if (more) {
                        ok = ok && wait(&b.full[ks], kph, b, a.status);
                        if (++st == C::NST) { st = 0; ph ^= 1; }
                    } else if (fix) {
                        ok = ok && wait(&b.vfix, 0, b, a.status);
                    }
                    // Tile 1 goes after tile 0.  Products of the two issued at once would run interleaved, end
                    // together and leave the tensor pipe idle while both tiles are in their softmax (d = 128,
                    // 16K tokens: 1250 us in turn, 1370 without; d = 64, where the softmax is the longer side,
                    // the same either way).  An order, not a dependence: the wait may run out.
                    if (i == 1)
                        for (int w = 0; w < 20000 && *(volatile int *)&b.turn <= j; w++) {}
                    if (j < ni) {
                        const uint32_t va = vd + vs * (C::TILE >> 4);
#pragma unroll
                        for (int k = 0; k < 2; k++) {            // the weights come in two halves
                            ok = ok && wait(&b.pfull[i][k], j & 1, b, a.status);
                            tc::tc_fence_after();
                            if (ok && one) {
#pragma unroll
                                for (int x = k * (kN / 32); x < (k + 1) * (kN / 32); x++)
                                    tc::mma_bf16_ts_lo(to, ts + x * 8, va + x * (16 * 128 >> 4), idO, (j | x) != 0);
                            }
                        }
                        if (ok && one) {
                            if (j + 1 < ni) qk(ks);
                            else tc::mma_commit(tc::smem_u32(&b.odone[i]));
                        }
                    }
                    if (i == 0 && one) *(volatile int *)&b.turn = j + 1;
                    if (ok && one) {
                        tc::mma_commit(tc::smem_u32(&b.empty[vs]));
                        if (more) tc::mma_commit(tc::smem_u32(&b.empty[ks]));
                    }
                    ok = __all_sync(0xffffffffu, ok);
                }
                if (!ok && lane == 0) {
                    atomicOr(a.status, kStTimeout);
                    atomicExch(&b.abort, 1);
                }
                // every operation issued is done before TMEM is freed: one more commit of each covers them
                if (one) tc::mma_commit(tc::smem_u32(&b.fin));
                __syncwarp();
                tc::mbar_wait(tc::smem_u32(&b.fin), 0, kWaitNs);
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

// [tokens][heads][d] rows with element strides ts, hs: boxes of 64 channels x
// box_h heads x box_t tokens, 128-byte swizzle.
bool make_map(CUtensorMap *m, const void *p, int64_t tokens, int heads, int d, int64_t ts, int64_t hs, int box_h, int box_t) {
    auto enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t gdim[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens};
    cuuint64_t gstr[2] = {(cuuint64_t)(heads > 1 ? hs : d) * 2, (cuuint64_t)(tokens > 1 ? ts : (int64_t)d * heads) * 2};
    if (gstr[0] == 0 || gstr[1] == 0) return false;
    cuuint32_t box[3] = {64, (cuuint32_t)box_h, (cuuint32_t)box_t};
    cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), gdim, gstr, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(PromptArgs a, cudaStream_t s) {
    Tc t;
    t.gq = a.Hq / a.G;
    t.tpt = 128 / t.gq;
    // a broadcast head (stride 0) is one head read for every group
    t.kh = a.k_hs != 0;
    t.vh = a.v_hs != 0;
    CUtensorMap mq, mk, mv;
    if (!make_map(&mq, a.q, a.n_q, a.Hq, D, a.q_ts, a.q_hs, t.gq, t.tpt)) return cudaErrorNotSupported;
    if (a.n_k == 0) {
        mk = mv = mq;
    } else if (!make_map(&mk, a.k, a.n_k, t.kh ? a.G : 1, D, a.k_ts, a.k_hs, 1, kN) ||
               !make_map(&mv, a.v, a.n_k, t.vh ? a.G : 1, D, a.v_ts, a.v_hs, 1, kN)) {
        return cudaErrorNotSupported;
    }
    const int64_t blocks = prompt_slots(a.n_q, a.n_seqs, 2 * t.tpt) * a.G;
    if (blocks >= (1LL << 31)) return cudaErrorNotSupported;
    static std::atomic<int> ready[kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        cudaFuncAttributes at;
        e = cudaFuncGetAttributes(&at, prompt_tc_kernel<D>);
        if (e != cudaSuccess) return e;
        if (at.numRegs != kRegs) return cudaErrorInvalidConfiguration;     // the register split would not add up
        e = cudaFuncSetAttribute(prompt_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev].store(1, std::memory_order_relaxed);
    }
    // fewer blocks than SMs: their keys are split over the others
    a.split = (int)std::max<int64_t>(1, std::min<int64_t>(kPartsTc / blocks, (a.n_k + kN - 1) / kN / kLeastTc));
    e = launch_overlapped(prompt_tc_kernel<D>, dim3((unsigned)blocks, (unsigned)a.split), kThreads, Cfg<D>::SMEM, s, a, t, mq,
                          mk, mv);
    return e == cudaSuccess && a.split > 1 ? launch_prompt_join(a, D, GKV_BF16, true, s) : e;
}

}  // namespace

cudaError_t launch_prompt_tc(const PromptArgs &a, int d, cudaStream_t s) {
    return d == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace serve
}  // namespace gkv
