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
// What bounds it: at d = 128 a 128 x 128 tile costs 128^3 MACs in each of the
// two products against 128^2 exponentials, so the tensor pipe; at d = 64
// the exponentials weigh twice as much, and the softmax warps bound it.  The two
// row tiles alternate: while the tensor core works on one's S and PV, the
// other's warps take its softmax.
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1 (one thread a row, its scores of a
// key tile in registers; the load from TMEM returns their maximum too), 8 TMA
// (Q once, then K and V tiles through a ring), 9 and 10 MMA issue of tile 0 and
// 1 (11 idle: registers are split by warpgroup).  P is the A operand of its
// product from TMEM, packed bf16 over the first half of its S; V is the B
// operand as it lies in memory (rows of channels, "MN-major").
// P is rounded to bf16 once, because A and B of a product have one type; its sum Z is
// not.  A weight moves by 2^-8 of itself at most, as each output does when it is
// rounded: outputs are 2.0 to 2.2e-3 from 64 bits where weights of 32 bits give 1.65e-3.
// A second bf16 part of P would take half as much tensor work again.
// TMEM, d = 128: S0, S1 of 128 keys, O0, O1.  tcgen05 operations of one thread
// complete in order, so the commit of S(j + 1) also tells that PV(j) is done.
// TMEM, d = 64: key tiles of 96, so that two S a row tile and O fill the 512
// columns: S(j + 1) is made under the softmax of j, and the round trip P, PV,
// QK, S (830 clocks and more) leaves the softmax warps' path.
// The issuing warp is a chain of waits and commits, about 110 clocks each: at
// d = 64 a ring slot holds V(j) and K(j + 2), one wait and one commit for both,
// and P is handed over at once.
//
// Measured (32 / 8 heads; GPU time): 16384 tokens of d = 128 1.17 to 1.38 ms by the
// power limit, 1.60 to 1.88 PFLOP/s of 1.88 that a plain matrix product reaches, the
// tensor pipe 75 % busy at 8192 tokens (316 us); 12000 tokens of d = 64 0.48 to 0.57
// ms by the power limit, 1.21
// PFLOP/s.  d = 64 step by step: 128-key tiles, one S 560 us, the maximum with
// the load 528, 96-key tiles and two S 532, one slot for V and K 511, P at once
// 509, a faster start and end of a block 497, no vote at a wait and the loop by
// two 480.  A loop of the softmax alone takes 1000 clocks for 96 keys of two
// warps a scheduler (770 of them exponentials), this kernel about 1370.  Tried for
// d = 64 and slower: two threads a row, no maximum but a check of the weights'
// sum, the next scores read under the last weights, P in columns of its own,
// key tiles of 64 with two or three S, four row tiles a CTA.
//
// Few blocks (a short chunk over a long cache) leave SMs idle: then a block's
// keys are split into parts (prompt.cuh) that prompt.cu joins.
//
// x c - m in one step keeps what rounding m left off, up to 2^-24 |m|, and so scales
// a row's weights, O and Z alike, by up to 2^64 at |m| = 2^30.  References stop there
// (kFar): a row of larger scores has infinite weights and gives NaN, one of nothing
// but scores further below has none and gives NaN too; scores that far below the
// others count 0.  Rounding x c as m was would lift the limit, but any look at m in
// the loop that is not there now costs 4 to 8 % of every call at d = 128.
//
// Masks: only the tiles that reach past a row's last key compare columns; the
// keys past a sequence's end get weight 0 that way, and their V rows, which
// may hold anything, are zeroed in shared memory before the product.
#include "prompt.cuh"
#include "tc.cuh"

#include <float.h>
#include <math.h>

#include <algorithm>
#include <atomic>

namespace gkv {
namespace serve {
namespace {

constexpr int kThreads = 384;                  // three warpgroups: two of softmax, one of TMA and MMA issue
// Registers a thread after the split; 256 x 208 + 128 x 88 = 384 x 168, the launch's own.
constexpr int kRegs = 168, kRegsSoftmax = 208, kRegsIssue = 88;
static_assert(256 * kRegsSoftmax + 128 * kRegsIssue <= kThreads * kRegs, "register split");
constexpr int kWarpTma = 8, kWarpMma = 9;      // MMA: warps 9 and 10, one a row tile
constexpr float kLazy = 8.f;                   // log2 of the growth a reference lets pass
constexpr float kFar = 1 << 30;                // size that a finite reference does not pass
constexpr uint64_t kWaitNs = 2000000000ull;

template <int D>
struct Cfg {
    static constexpr int NK = keys_tc(D);                      // keys of a tile
    static constexpr int SB = D == 128 ? 1 : 2;                // score buffers of a row tile
    static constexpr int SW = SB * NK;                         // TMEM columns of a row tile's scores
    static_assert(2 * (SW + D) <= 512 && NK % 32 == 0, "TMEM columns");
    static constexpr int NB = D / 64;                          // 64-channel blocks of a row
    static constexpr uint32_t TILE = NB * 128 * 128;           // bytes of a 128-row tile
    static constexpr uint32_t KT = NB * NK * 128;              // bytes of a key or value tile
    static constexpr bool PAIR = D == 64;                      // a ring slot holds V(j) and K(j + SB), or one of them
    static constexpr uint32_t SLOT = PAIR ? 2 * KT : KT;
    static constexpr int NST = D == 128 ? 5 : 8;               // ring slots
    static constexpr int HV = D == 128 ? 2 : 1;                // pieces in which P is handed over
    static constexpr size_t SMEM = 1024 + 2 * (size_t)TILE + NST * (size_t)SLOT;
};

struct Bars {
    uint64_t full[8], empty[8], qfull[2], sfull[2][2], pfull[2][2][2], vfix, fin;
    uint64_t odone[2], oprev[2];       // the last PV of a row tile is in O; the last but one (two score buffers)
    uint32_t tbase;
    int abort, turn;           // turn: key tiles whose products row tile 0 has issued
};

struct Tc {
    int gq, tpt;               // heads of a KV head, tokens of a row tile
    int kh, vh;                // head coordinate step of k, v (0: one head for all)
    int slots;                 // of prompt_slots
};

__device__ __forceinline__ bool wait(uint32_t addr, uint32_t parity, Bars &b, int *status) {
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
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, Bars &b, int *status) {
    return wait(tc::smem_u32(bar), parity, b, status);
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
    constexpr int NK = C::NK, SB = C::SB;
    extern __shared__ __align__(1024) unsigned char raw[];
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) &
                                                            ~static_cast<uintptr_t>(1023));
    unsigned char *Qs = base, *ring = base + 2 * C::TILE;
    __shared__ Bars b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    next_may_start();
    if (warp == kWarpTma && lane == 0) {                 // the thread that uses them first
        for (int i = 0; i < C::NST; i++) {
            tc::mbar_init(tc::smem_u32(&b.full[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.empty[i]), 2);
        }
        for (int i = 0; i < 2; i++) {
            tc::mbar_init(tc::smem_u32(&b.qfull[i]), 1);
            for (int k = 0; k < 2; k++) {
                tc::mbar_init(tc::smem_u32(&b.sfull[i][k]), 1);
                for (int x = 0; x < 2; x++) tc::mbar_init(tc::smem_u32(&b.pfull[i][k][x]), 4);
            }
            tc::mbar_init(tc::smem_u32(&b.odone[i]), 1);
            tc::mbar_init(tc::smem_u32(&b.oprev[i]), 1);
        }
        tc::mbar_init(tc::smem_u32(&b.vfix), 1);
        tc::mbar_init(tc::smem_u32(&b.fin), 2);
        b.abort = 0;
        b.turn = 0;
        tc::fence_barrier_init();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kWarpMma) {
        tc::tmem_alloc(tc::smem_u32(&b.tbase), 512);
        tc::tmem_relinquish();
    }
    after_previous();
    if (blockIdx.x == 0) check_bounds(a);
    // ---- the CTA's rows: heavy blocks (late tokens) first
    const int part = blockIdx.x % a.split, block = blockIdx.x / a.split, g = block % a.G;
    const int tok = 2 * t.tpt;
    const int slot = t.slots - 1 - block / a.G;
    int64_t q0, nq64, k0, nk64;
    int s;
    const bool fits = slot_rows(a, slot, tok, s, q0, nq64, k0, nk64);
    const int64_t t0_64 = ((int64_t)slot - ((int)q0 / tok + s)) * tok;
    const int nq = (int)nq64, nk = (int)nk64, t0 = (int)t0_64;
    const int off = nk - nq;                             // query i sees keys <= i + off
    const int ntile = t0 + t.tpt < nq ? 2 : 1;
    // key tiles of each row tile, up to the last key its last token sees; of
    // them this part's: [j0, j0 + n)
    const int last0 = min(nq, t0 + t.tpt) - 1 + off, last1 = min(nq, t0 + 2 * t.tpt) - 1 + off;
    const int all0 = last0 >= 0 ? last0 / NK + 1 : 0, all1 = ntile > 1 && last1 >= 0 ? last1 / NK + 1 : 0;
    const int all = max(all0, all1), np = parts_of(all, a.split, least_tc(D));
    const int j0 = part_first(all, np, part), j1 = part_first(all, np, part + 1), n = j1 - j0;
    const int nkv0 = max(0, min(all0, j1) - j0), nkv1 = max(0, min(all1, j1) - j0);

    // nothing to do: a sequence that does not fit, a slot past its tokens, a part beyond the block's
    const bool idle = !fits || t0_64 < 0 || t0_64 >= nq64 || part >= np;

    // ---- copies, by the producer's thread: the first ones leave before the block meets
    auto copy = [&](const CUtensorMap *map, int head, int j, uint32_t at, uint32_t fb) {
#pragma unroll
        for (int c = 0; c < C::NB; c++)
            tc::tma_load_3d(tc::smem_u32(ring + at + c * NK * 128), map, c * 64, head, (int)(k0 + (j0 + j) * NK), fb);
    };
    // a slot with V(jv), K(jk) or both; with neither (fewer key tiles than score buffers) it arrives empty
    auto fill = [&](int st, int jv, int jk) {
        const bool v = jv >= 0, k = jk >= 0 && jk < n;
        const uint32_t fb = tc::smem_u32(&b.full[st]);
        if (v || k) tc::mbar_expect_tx(fb, (v + k) * C::KT);
        else tc::mbar_arrive(fb);
        if (v) copy(&mapV, g * t.vh, jv, st * C::SLOT, fb);
        if (k) copy(&mapK, g * t.kh, jk, st * C::SLOT + (C::PAIR ? C::KT : 0), fb);
    };
    if (warp == kWarpTma && lane == 0 && !idle && n > 0) {
        for (int i = 0; i < ntile; i++) {
            const uint32_t qb = tc::smem_u32(&b.qfull[i]);
            tc::mbar_expect_tx(qb, (uint32_t)(C::NB * t.tpt * t.gq * 128));
#pragma unroll
            for (int c = 0; c < C::NB; c++)
                tc::tma_load_3d(tc::smem_u32(Qs + i * C::TILE + c * 128 * 128), &mapQ, c * 64, g * t.gq,
                                (int)(q0 + t0 + i * t.tpt), qb);
            if (i == 0)
                for (int k = 0; k < SB; k++) fill(k, -1, k);
        }
    }

    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tb = b.tbase;
    if (idle) {
        if (warp == kWarpMma) tc::tmem_dealloc(tb, 512);
        return;
    }

    // the sequence's last key tile is partial and other rows follow it: their V rows are zeroed
    const int keep = nk - (j1 - 1) * NK;                  // keys of the sequence in the part's last tile, from it on
    const bool fix = n > 0 && keep < NK && k0 + nk < a.n_k;

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        // ---------------- softmax and epilogue: one thread a row ----------------
        const int i = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const int tk = r / t.gq, h = r - tk * t.gq;
        const int token = t0 + i * t.tpt + tk;
        const bool live = tk < t.tpt && token < nq;
        const int lim = live ? token + off : -1;         // last key the row sees
        const float c = a.scale * kLog2e;
        const uint32_t lanes = tb + ((uint32_t)(q * 32) << 16);
        const uint32_t ts0 = lanes + (uint32_t)(i * C::SW), to = lanes + 2 * C::SW + i * D;
        // the first token of the tile sees the fewest keys: below its limit no mask is needed
        const int clear = t0 + i * t.tpt + off;
        float m = -INFINITY, z = 0.f;                    // m: the reference times c
        const int nj = i ? nkv1 : nkv0;
        bool ok = true;
        // A wait that gave up leaves nothing to rely on, but the warp goes on together to the end: every later
        // wait gives up at once, and nothing is written.
        const uint32_t bs = tc::smem_u32(&b.sfull[i][0]), bp = tc::smem_u32(&b.pfull[i][0][0]);
        uint32_t ph = 0;                                 // of the score buffers
        // d = 64: by two, so that a score buffer's addresses are constants (12000 tokens 485 -> 480 us)
#pragma unroll (SB)
        for (int j = 0; j < nj; j++) {
            const int sb = j % SB;
            const uint32_t ts = ts0 + (uint32_t)(sb * NK);
            ok = wait(bs + 8 * sb, ph, b, a.status) && ok;
            __syncwarp();
            tc::tc_fence_after();
            uint32_t x[NK / 32][32];
            float mx[NK / 32];
#pragma unroll
            for (int k = 0; k < NK / 32; k++) tc::tmem_ld32_max_async(ts + 32 * k, x[k], mx[k]);
            tc::tmem_wait_ld(x[0]);
#pragma unroll
            for (int k = 1; k < NK / 32; k++) tc::tmem_loaded(x[k]);
#pragma unroll
            for (int k = 0; k < NK / 32; k++) tc::tmem_loaded(mx[k]);
            if ((j0 + j) * NK + NK - 1 > clear) {
                const int rel = lim - (j0 + j) * NK;
#pragma unroll
                for (int k = 0; k < NK / 32; k++) {
#pragma unroll
                    for (int e = 0; e < 32; e++)
                        if (k * 32 + e > rel) x[k][e] = 0xff800000u;       // -inf
                    mx[k] = fmaxf(__uint_as_float(x[k][0]), __uint_as_float(x[k][1]));
#pragma unroll
                    for (int e = 2; e < 32; e += 2)
                        mx[k] = max3(mx[k], __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
                }
            }
#pragma unroll
            for (int k = 1; k < NK / 32; k++) mx[0] = fmaxf(mx[0], mx[k]);
            const float mn = mx[0] == -INFINITY ? -INFINITY : fminf(fmaxf(mx[0] * c, -kFar), kFar);
            if (m == -INFINITY) m = mn;                  // nothing accumulated yet
            else if (__builtin_expect(mn > m + kLazy, 0)) z = -FLT_MIN - z;        // asks for a rescale, by a sum of 0 too
            if (__any_sync(0xffffffffu, z < 0.f)) {
                // O is rescaled once PV(j - 1) is in it: with one score buffer S(j) came after it; with two
                // S(j + 1) does, and at the last tile a commit of its own tells
                if constexpr (SB == 2) {
                    ok = (j + 1 < nj ? wait(&b.sfull[i][(j + 1) & 1], ((j + 1) / 2) & 1, b, a.status)
                                     : wait(&b.oprev[i], 0, b, a.status)) && ok;
                    __syncwarp();
                    tc::tc_fence_after();
                }
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
                    tc::tmem_st(to + 32 * k, o);
                }
            }
            const float sh = m == -INFINITY ? 0.f : -m;
            const float2 c2 = make_float2(c, c), s2 = make_float2(sh, sh);
            float2 acc = make_float2(0.f, 0.f);
            auto weights = [&](uint32_t &p, int at) {
                const float2 y = __ffma2_rn(make_float2(__uint_as_float(x[at / 32][at & 31]),
                                                        __uint_as_float(x[at / 32][(at & 31) + 1])), c2, s2);
                const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
                acc = __fadd2_rn(acc, w);
                p = pack2(w.x, w.y);
            };
            auto hand = [&](int k) {
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(bp + 8 * (2 * sb + k));
            };
            uint32_t p0[32], p1[(NK - 64) / 2];
#pragma unroll
            for (int e = 0; e < 32; e++) weights(p0[e], 2 * e);
            tc::tmem_st(ts, p0);
            if (C::HV == 2) hand(0);
#pragma unroll
            for (int e = 0; e < (NK - 64) / 2; e++) weights(p1[e], 64 + 2 * e);
            tc::tmem_st(ts + 32, p1);
            hand(C::HV - 1);
            z += acc.x + acc.y;
            if (sb == SB - 1) ph ^= 1;
        }
        if (nj > 0) ok = __all_sync(0xffffffffu, wait(&b.odone[i], 0, b, a.status) && ok);
        tc::tc_fence_after();
        const int64_t row = q0 + token;
        const int hq = g * t.gq + h;
        if (np == 1) {
            if (ok && i < ntile) {
                // A thread holds a row, and 32 rows a store are 32 memory sectors: the rows go through
                // shared memory (this warp's rows of Q, which no product reads any more; 16-byte chunks
                // permuted by row) and leave 512 bytes a store.
                constexpr int CH = D / 8;                    // chunks of a row
                const float inv = row_scale(m, z);
                const int64_t at = live ? row * a.o_ts + hq * a.o_hs : -1;
                uint4 v[CH];
                if (nj > 0) {
                    unsigned char *stage = Qs + i * C::TILE + q * 32 * (D * 2);
                    uint32_t u[D / 32][32];
#pragma unroll
                    for (int k = 0; k < D / 32; k++) tc::tmem_ld32_async(to + 32 * k, u[k]);
                    tc::tmem_wait_ld(u[0]);
#pragma unroll
                    for (int k = 1; k < D / 32; k++) tc::tmem_loaded(u[k]);
#pragma unroll
                    for (int ch = 0; ch < CH; ch++) {
                        const uint32_t *w = &u[ch / 4][ch % 4 * 8];
                        uint4 y = make_uint4(0, 0, 0, 0);
                        if (lim >= 0) {
                            y.x = pack2(__uint_as_float(w[0]) * inv, __uint_as_float(w[1]) * inv);
                            y.y = pack2(__uint_as_float(w[2]) * inv, __uint_as_float(w[3]) * inv);
                            y.z = pack2(__uint_as_float(w[4]) * inv, __uint_as_float(w[5]) * inv);
                            y.w = pack2(__uint_as_float(w[6]) * inv, __uint_as_float(w[7]) * inv);
                        }
                        *reinterpret_cast<uint4 *>(stage + lane * (D * 2) + ((ch ^ lane) & (CH - 1)) * 16) = y;
                    }
                    __syncwarp();
                    // all loads, then all stores: in turns every load would wait for the store before it
#pragma unroll
                    for (int x = 0; x < CH; x++) {
                        const int rr = x * (32 / CH) + lane / CH, ch = lane % CH;
                        v[x] = *reinterpret_cast<const uint4 *>(stage + rr * (D * 2) + ((ch ^ rr) & (CH - 1)) * 16);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < CH; x++) v[x] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int x = 0; x < CH; x++) {
                    const int64_t to_row = __shfl_sync(0xffffffffu, at, x * (32 / CH) + lane / CH);
                    if (to_row >= 0) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + to_row + lane % CH * 8) = v[x];
                }
                if (live && a.lse) a.lse[row * a.Hq + hq] = row_lse(m, z);
            }
        } else {
            // a part: [D / 4][rows] sums of 4 channels, then [rows] references, [rows] sums of weights
            float *pp = a.part + ((size_t)block * a.split + part) * part_floats(kRowsTc, D);
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
            // keys SB tiles ahead of their values, as the products take them; the first SB key tiles are on their way
            int issued = n > 0 ? (C::PAIR ? SB : min(SB, n)) : 0;
            bool ok = n > 0;
            if (lane == 0) {
                auto next = [&](int jv, int jk) {
                    const int st = issued % C::NST;
                    ok = !*(volatile int *)&b.abort && wait(&b.empty[st], ((issued / C::NST) & 1) ^ 1, b, a.status);
                    if (!ok) return;
                    fill(st, jv, jk);
                    issued++;
                };
                for (int j = 0; ok && j < n; j++) {
                    if (C::PAIR) {
                        next(j, j + SB);
                    } else {
                        next(j, -1);
                        if (ok && j + SB < n) next(-1, j + SB);
                    }
                }
            }
            issued = __shfl_sync(0xffffffffu, issued, 0);
            const int slots = C::PAIR ? n + SB : 2 * n;
            ok = issued == slots && n > 0;
            if (fix && ok) {
                const int st = (slots - 1) % C::NST;
                if (wait(&b.full[st], ((slots - 1) / C::NST) & 1, b, a.status)) {
                    for (int i = lane; i < (NK - keep) * C::NB * 8; i += 32) {
                        const int r = keep + i / (C::NB * 8), c = i % (C::NB * 8);
                        *reinterpret_cast<uint4 *>(ring + st * C::SLOT + (c >> 3) * (NK * 128) + r * 128 + (c & 7) * 16) =
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
                for (int i = 0; i < ntile; i++) tc::mbar_wait(tc::smem_u32(&b.qfull[i]), 0, kWaitNs);
            }
        } else if (warp <= kWarpMma + 1) {
            // ---------------- MMA issue: one warp a row tile, one lane issues ----------------
            if (n > 0) {
                constexpr uint32_t idS = tc::idesc_bf16_f32(128, NK), idO = tc::idesc_bf16_f32(128, D) | tc::kIdescBmn;
                const int i = warp - kWarpMma, ni = i ? nkv1 : nkv0;
                // descriptors: the start address (16-byte units) is the low word's low end, the rest is constant
                const uint32_t qd = ((tc::smem_u32(Qs) >> 4) | (1u << 16)) + i * (C::TILE >> 4);
                const uint32_t kd = ((tc::smem_u32(ring) + (C::PAIR ? C::KT : 0)) >> 4) | (1u << 16);
                const uint32_t vd = (tc::smem_u32(ring) >> 4) | ((NK * 128 >> 4) << 16);
                const uint32_t ts = tb + i * C::SW, to = tb + 2 * C::SW + i * D;
                const bool one = tc::elect_one();
                int st = 0;
                uint32_t ph = 0;                         // of the ring slot that comes next
                bool ok = i >= ntile || wait(&b.qfull[i], 0, b, a.status);
                auto qk = [&](int slot, int sb) {        // S = Q K^T into score buffer sb, K in the slot
                    const uint32_t ka = kd + slot * (C::SLOT >> 4);
#pragma unroll
                    for (int c = 0; c < C::NB; c++)
#pragma unroll
                        for (int x = 0; x < 4; x++)
                            tc::mma_bf16_lo(ts + sb * NK, qd + c * (128 * 128 >> 4) + 2 * x, ka + c * (NK * 128 >> 4) + 2 * x,
                                            idS, (c | x) != 0);
                    tc::mma_commit(tc::smem_u32(&b.sfull[i][sb]));
                };
#pragma unroll
                for (int s0 = 0; s0 < SB; s0++) {
                    if (!C::PAIR && s0 >= n) break;
                    ok = wait(&b.full[st], ph, b, a.status) && ok;
                    tc::tc_fence_after();
                    if (ok && one) {
                        if (s0 < ni) qk(st, s0);
                        tc::mma_commit(tc::smem_u32(&b.empty[st]));
                    }
                    st++;
                }
                ok = __all_sync(0xffffffffu, ok);
                // the row tiles may end at different key tiles: both warps release every slot, in order
                const uint32_t bfull = tc::smem_u32(&b.full[0]), bempty = tc::smem_u32(&b.empty[0]);
                const uint32_t bp = tc::smem_u32(&b.pfull[i][0][0]);
                uint32_t pp = 0;                         // phase of the weights
                for (int jb = 0; ok && jb < n; jb += SB, pp ^= 1) {
#pragma unroll
                    for (int sb = 0; sb < SB; sb++) {
                        const int j = jb + sb;
                        if (SB > 1 && j >= n) break;
                        const int vs = st;
                        ok = wait(bfull + 8 * vs, ph, b, a.status) && ok;
                        if (++st == C::NST) { st = 0; ph ^= 1; }
                        int ks = vs;
                        const bool more = !C::PAIR && j + SB < n;
                        if (more) {
                            ks = st;
                            ok = wait(bfull + 8 * ks, ph, b, a.status) && ok;
                            if (++st == C::NST) { st = 0; ph ^= 1; }
                        }
                        if (fix && j + 1 == n) ok = wait(&b.vfix, 0, b, a.status) && ok;
                        // d = 128: tile 1 goes after tile 0.  Products of the two issued at once would run
                        // interleaved, end together and leave the tensor pipe idle while both tiles are in
                        // their softmax (16K tokens: 1250 us in turn, 1370 without).  At d = 64, where the
                        // softmax is the longer side, a turn only delays.  An order, not a dependence: the
                        // wait may run out.
                        if (D == 128 && i == 1)
                            for (int w = 0; w < 20000 && *(volatile int *)&b.turn <= j; w++) {}
                        if (j < ni) {
                            const uint32_t va = vd + vs * (C::SLOT >> 4);
#pragma unroll
                            for (int k = 0; k < C::HV; k++) {        // the weights come in pieces
                                ok = wait(bp + 8 * (2 * sb + k), pp, b, a.status) && ok;
                                tc::tc_fence_after();
                                if (one) {
#pragma unroll
                                    for (int x = k * 4; x < (k == C::HV - 1 ? NK / 16 : 4); x++)
                                        tc::mma_bf16_ts_lo(to, ts + sb * NK + x * 8, va + x * (16 * 128 >> 4), idO, (j | x) != 0);
                                    if (k == C::HV - 1) {
                                        if (j + SB < ni) qk(ks, sb);
                                        else tc::mma_commit(tc::smem_u32(j + 1 == ni ? &b.odone[i] : &b.oprev[i]));
                                    }
                                }
                            }
                        }
                        if (D == 128 && i == 0 && one) *(volatile int *)&b.turn = j + 1;
                        if (one) {
                            tc::mma_commit(bempty + 8 * vs);
                            if (more) tc::mma_commit(bempty + 8 * ks);
                        }
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

// Parts of a block.  Fewer blocks than SMs leave SMs idle, so their keys are split; parts and their join cost
// about 5 us and 0.15 us a block (0.26 MB written and read a part), a wave's start and end 6 us.  Blocks see
// `tiles` key tiles at most and, were the sequences' lengths within twice their mean, `some`.  Parts beyond one a
// SM, which run in waves, are taken on the latter's account only.  (d = 128, us unsplit / split: 600 queries over
// 30000 keys of 8 heads 354 / 230 in 3 parts, 2 waves; 120 over 30000 283 / 50 in 9, 71 in 19; 4000 of 2 heads
// 48 / 26 in 4; not split: 2000 of 2 heads of 4 queries 25 / 30, 1024 of 8 17 / 32.)
int split_of(int64_t blocks, int64_t tiles, int n_seqs, int d) {
    const double tile = d == 64 ? 0.75 : 1.2;            // us
    auto cost = [&](int64_t parts, int64_t n) {
        return (double)((blocks * parts + kSms - 1) / kSms) * (6. + (double)((n + parts - 1) / parts) * tile) +
               (parts > 1 ? 5. + 0.15 * (double)blocks : 0.);
    };
    const int64_t one = std::min<int64_t>(kSms / blocks, tiles / least_tc(d));
    int64_t best = one > 1 && cost(one, tiles) < cost(1, tiles) ? one : 1;
    const int64_t some = std::min<int64_t>(tiles, 2 * tiles / n_seqs);
    const int64_t most = std::min<int64_t>(kPartsTc / blocks, some / least_tc(d));
    for (int64_t p = best + 1; p <= most; p++)
        if (cost(p, some) < cost(best, some)) best = p;
    return (int)best;
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
    } else if (!make_map(&mk, a.k, a.n_k, t.kh ? a.G : 1, D, a.k_ts, a.k_hs, 1, Cfg<D>::NK) ||
               !make_map(&mv, a.v, a.n_k, t.vh ? a.G : 1, D, a.v_ts, a.v_hs, 1, Cfg<D>::NK)) {
        return cudaErrorNotSupported;
    }
    const int64_t slots = prompt_slots(a.n_q, a.n_seqs, 2 * t.tpt), blocks = slots * a.G;
    if (blocks >= (1LL << 31)) return cudaErrorNotSupported;
    t.slots = (int)slots;
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
    a.split = split_of(blocks, (a.n_k + Cfg<D>::NK - 1) / Cfg<D>::NK, a.n_seqs, D);
    e = launch_overlapped(prompt_tc_kernel<D>, dim3((unsigned)(blocks * a.split)), kThreads, Cfg<D>::SMEM, s, a, t, mq,
                          mk, mv);
    return e == cudaSuccess && a.split > 1 ? launch_prompt_join(a, D, GKV_BF16, true, s) : e;
}

}  // namespace

cudaError_t launch_prompt_tc(const PromptArgs &a, int d, cudaStream_t s) {
    return d == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace serve
}  // namespace gkv
