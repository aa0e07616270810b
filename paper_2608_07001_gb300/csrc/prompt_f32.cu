// prompt_f32.cu -- the prompt's attention on CUDA cores: fp32 inputs, which
// keep fp32 in both products, and bf16 tensors whose strides have no tensor
// map (a broadcast token or query axis).
//
// A block holds 64 rows (a row is a query token and one of the gq heads of a
// KV head, so a key tile is read once for them all) and walks tiles of 64 keys:
//   S = Q K^T / sqrt(d), the running maximum M and sum Z of a row,
//   P = exp(S - M) through shared memory, O = O exp(M_old - M) + P V.
// FMA-bound: 2 x 64 x 64 x d FMAs a tile against 16 KB (d = 64) or 32 KB of K
// and V each.  128 threads own 8 x 4 scores and 8 x d/16 outputs each, so that
// a shared-memory read feeds 8 (S) and 10 (PV) FMAs; packed fp32x2 FMA halves
// the issue slots, along the channels for S and across output columns for PV.
// K of the next tile arrives (cp.async) under PV, V under S.  Two blocks a SM.
// Measured: 52 TFLOP/s (32 / 8 heads of 128 at 4500 tokens; FMA pipe 67 % busy),
// 48 at d = 64 (46 with the products unrolled by 2 instead of 8), 25 us for 1024
// tokens of 2 heads: 13 us of a part's one tile, of which 3 issue its copies, 4
// of the join, the rest launches.  256 threads of 4 x 4 scores: 44 TFLOP/s.
//
// When a launch has fewer blocks than the GPU holds, a block's keys are split
// into parts (prompt.cuh) that prompt.cu joins.
#include "prompt.cuh"
#include "tc.cuh"

#include <math.h>

#include <algorithm>
#include <atomic>

namespace gkv {
namespace serve {
namespace {

constexpr int kR = kRowsF32, kK = kKeysF32, kThreads = 128;

template <int D>
struct Cfg {
    // Q, K, V, P without padding, so that two blocks fit a SM at d = 128 (2 x 112 KB); the 16-byte chunks of
    // a key are permuted by key % 8 instead, as 8 lanes read one chunk of 8 keys
    static constexpr int Q = kR * D, K = kK * D, V = kK * D, P = kR * kK;
    static constexpr size_t SMEM = (size_t)(Q + K + V + P) * sizeof(float);
};

__device__ __forceinline__ void copy16(float *dst, const float *src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// 4 channels into shared memory as fp32; zeros when off.
__device__ __forceinline__ void load4(float *dst, const float *src, bool on) { copy16(dst, src, on); }
__device__ __forceinline__ void load4(float *dst, const __nv_bfloat16 *src, bool on) {
    uint2 u = make_uint2(0, 0);
    if (on) u = *reinterpret_cast<const uint2 *>(src);
    *reinterpret_cast<float4 *>(dst) = make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u),
                                                   __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) prompt_f32_kernel(const PromptArgs a) {
    using C = Cfg<D>;
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = Qs + C::Q, *Vs = Ks + C::K, *Ps = Vs + C::V;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    next_may_start();
    after_previous();
    if (blockIdx.x == 0) check_bounds(a);

    // ---- the block: rows of one KV head, heavy blocks (late tokens) first, all parts of one before the next
    // (one after another by part, the last part's heavy blocks would start last: 3000 tokens of 2 heads 153 us,
    // 118 this way)
    const int part = blockIdx.x % a.split;
    const int gq = a.Hq / a.G, tok = kR / gq, block = blockIdx.x / a.split, g = block % a.G;
    const int slot = (int)prompt_slots(a.n_q, a.n_seqs, tok) - 1 - block / a.G;
    int s;
    int64_t q0, nq64, k0, nk64;
    if (!slot_rows(a, slot, tok, s, q0, nq64, k0, nk64)) return;
    const int64_t t0_64 = ((int64_t)slot - ((int)q0 / tok + s)) * tok;
    if (t0_64 < 0 || t0_64 >= nq64) return;
    const int nq = (int)nq64, nk = (int)nk64, t0 = (int)t0_64, off = nk - nq;
    const int last = min(nq, t0 + tok) - 1 + off;
    const int n = last >= 0 ? last / kK + 1 : 0;
    const int np = parts_of(n, a.split, kLeastF32);
    if (part >= np) return;
    const int j0 = part_first(n, np, part), j1 = part_first(n, np, part + 1);

    const T *K = static_cast<const T *>(a.k) + k0 * a.k_ts + g * a.k_hs;
    const T *V = static_cast<const T *>(a.v) + k0 * a.v_ts + g * a.v_hs;
    auto load_k = [&](int j) {
        for (int i = tid; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4), key = j * kK + r;
            load4(Ks + r * D + (c ^ (r & 7)) * 4, K + (key < nk ? key : 0) * a.k_ts + c * 4, key < nk);
        }
        copy_commit();
    };
    auto load_v = [&](int j) {
        for (int i = tid; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4), key = j * kK + r;
            load4(Vs + r * D + c * 4, V + (key < nk ? key : 0) * a.v_ts + c * 4, key < nk);
        }
        copy_commit();
    };
    if (n > 0) {
        load_k(j0);
        // a warp loads RW rows a step, N steps of STEP rows: each lane finds the offset of one of them
        constexpr int RW = 32 / (D / 4), STEP = kThreads / (D / 4), N = kR / STEP;
        const int lane = tid & 31, first = tid / 32 * RW, c = tid % (D / 4), rw = lane / (D / 4);
        const int mine = first + lane / N + lane % N * STEP, tk = mine / gq;
        const bool on = tk < tok && t0 + tk < nq;
        const int64_t at = on ? (q0 + t0 + tk) * a.q_ts + (g * gq + mine - tk * gq) * a.q_hs : -1;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int64_t from = __shfl_sync(0xffffffffu, at, rw * N + i);
            load4(Qs + (first + rw + i * STEP) * D + c * 4, static_cast<const T *>(a.q) + (from < 0 ? 0 : from) + c * 4, from >= 0);
        }
        copy_commit();
    }

    float2 o[8][D / 32];
    float m[8], z[8];
    int lim[8];                               // last key of the row (base 0), below 0: none
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma unroll
        for (int c = 0; c < D / 32; c++) o[i][c] = make_float2(0.f, 0.f);
        m[i] = -INFINITY;
        z[i] = 0.f;
        const int tk = (ty * 8 + i) / gq;
        lim[i] = tk < tok && t0 + tk < nq ? t0 + tk + off : -1;
    }
    const float sc = a.scale * kLog2e;

    for (int j = j0; j < j1; j++) {
        load_v(j);
        copy_wait<1>();                       // K of this tile (and Q)
        __syncthreads();
        float2 x[8][4];
#pragma unroll
        for (int i = 0; i < 8; i++)
#pragma unroll
            for (int c = 0; c < 4; c++) x[i][c] = make_float2(0.f, 0.f);
#pragma unroll 8
        for (int e = 0; e < D; e += 4) {
            float4 kf[4];
#pragma unroll
            for (int c = 0; c < 4; c++) kf[c] = *reinterpret_cast<const float4 *>(Ks + (tx + 16 * c) * D + ((e >> 2) ^ (tx & 7)) * 4);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float4 qf = *reinterpret_cast<const float4 *>(Qs + (ty * 8 + i) * D + e);
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    x[i][c] = __ffma2_rn(make_float2(qf.x, qf.y), make_float2(kf[c].x, kf[c].y), x[i][c]);
                    x[i][c] = __ffma2_rn(make_float2(qf.z, qf.w), make_float2(kf[c].z, kf[c].w), x[i][c]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float y[4], mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; c++) {
                y[c] = j * kK + tx + 16 * c <= lim[i] ? (x[i][c].x + x[i][c].y) * sc : -INFINITY;
                mx = fmaxf(mx, y[c]);
            }
#pragma unroll
            for (int w = 8; w >= 1; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            const float mn = fmaxf(m[i], mx), sh = mn == -INFINITY ? 0.f : mn, w = tc::ex2(m[i] - sh);
            m[i] = mn;
            z[i] *= w;
#pragma unroll
            for (int c = 0; c < D / 32; c++) { o[i][c].x *= w; o[i][c].y *= w; }
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const float p = tc::ex2(y[c] - sh);
                z[i] += p;
                Ps[(ty * 8 + i) * kK + tx + 16 * c] = p;
            }
        }
        __syncthreads();                      // all of K is read, all of P written
        if (j + 1 < j1) load_k(j + 1);
        if (j + 1 < j1) copy_wait<1>(); else copy_wait<0>();      // V of this tile
        __syncthreads();
#pragma unroll 8
        for (int e = 0; e < kK; e += 4) {
            float4 p[8];
#pragma unroll
            for (int i = 0; i < 8; i++) p[i] = *reinterpret_cast<const float4 *>(Ps + (ty * 8 + i) * kK + e);
#pragma unroll
            for (int f = 0; f < 4; f++) {
                float4 v[D / 64];
#pragma unroll
                for (int c = 0; c < D / 64; c++) v[c] = *reinterpret_cast<const float4 *>(Vs + (e + f) * D + c * 64 + tx * 4);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float w = f == 0 ? p[i].x : f == 1 ? p[i].y : f == 2 ? p[i].z : p[i].w;
#pragma unroll
                    for (int c = 0; c < D / 64; c++) {
                        o[i][2 * c] = __ffma2_rn(make_float2(w, w), make_float2(v[c].x, v[c].y), o[i][2 * c]);
                        o[i][2 * c + 1] = __ffma2_rn(make_float2(w, w), make_float2(v[c].z, v[c].w), o[i][2 * c + 1]);
                    }
                }
            }
        }
        __syncthreads();                      // V and P are read
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1) z[i] += __shfl_xor_sync(0xffffffffu, z[i], w);

    if (np > 1) {       // a part: [kR][D] sums, then [kR] maxima, [kR] sums of weights
        float *pp = a.part + ((size_t)block * a.split + part) * part_floats(kR, D);
#pragma unroll
        for (int i = 0; i < 8; i++) {
#pragma unroll
            for (int c = 0; c < D / 64; c++)
                *reinterpret_cast<float4 *>(pp + (ty * 8 + i) * D + c * 64 + tx * 4) =
                    make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
            if (tx == 0) { pp[kR * D + ty * 8 + i] = m[i]; pp[kR * (D + 1) + ty * 8 + i] = z[i]; }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int r = ty * 8 + i, tk = r / gq, t = t0 + tk, h = g * gq + r % gq;
        if (tk >= tok || t >= nq) continue;
        const float inv = z[i] > 0.f ? 1.f / z[i] : z[i];        // no key: 0; a NaN stays
        T *p = static_cast<T *>(a.out) + (q0 + t) * a.o_ts + h * a.o_hs + tx * 4;
#pragma unroll
        for (int c = 0; c < D / 64; c++)
            put4(p + c * 64, make_float4(o[i][2 * c].x * inv, o[i][2 * c].y * inv, o[i][2 * c + 1].x * inv,
                                         o[i][2 * c + 1].y * inv));
        if (tx == 0 && a.lse)
            a.lse[(q0 + t) * a.Hq + h] = z[i] == 0.f ? -INFINITY : (m[i] + log2f(z[i])) * 0.6931471805599453f;
    }
}

template <typename T, int D>
cudaError_t launch(PromptArgs a, int dtype, cudaStream_t s) {
    static std::atomic<int> ready[kMaxDevices];
    const size_t smem = Cfg<D>::SMEM;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(prompt_f32_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready[dev].store(1, std::memory_order_relaxed);
    }
    const int tok = kR / (a.Hq / a.G);
    const int64_t blocks = prompt_slots(a.n_q, a.n_seqs, tok) * a.G;
    if (blocks >= (1LL << 31)) return cudaErrorInvalidConfiguration;
    // as many parts as fit beside one another, none smaller than a key tile
    a.split = (int)std::max<int64_t>(1, std::min<int64_t>(kPartsF32 / blocks, (a.n_k + kK - 1) / kK));
    e = launch_overlapped(prompt_f32_kernel<T, D>, dim3((unsigned)(blocks * a.split)), kThreads, smem, s, a);
    return e == cudaSuccess && a.split > 1 ? launch_prompt_join(a, D, dtype, false, s) : e;
}

}  // namespace

cudaError_t launch_prompt_f32(const PromptArgs &a, int d, int dtype, cudaStream_t s) {
    if (dtype == GKV_BF16) return d == 128 ? launch<__nv_bfloat16, 128>(a, dtype, s) : launch<__nv_bfloat16, 64>(a, dtype, s);
    return d == 128 ? launch<float, 128>(a, dtype, s) : launch<float, 64>(a, dtype, s);
}

}  // namespace serve
}  // namespace gkv
