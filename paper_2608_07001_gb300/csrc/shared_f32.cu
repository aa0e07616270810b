// shared_f32.cu -- the entries of a shared prefix attended for all its requests
// at once: fp32 rows, on CUDA cores (shared_attention.cu has the whole).
//
// A block takes a piece: 64 rows (up to `tok` requests' gq query heads of one KV
// head) over a run of key tiles of 64 entries:
//   S = Q K^T log2(e) / sqrt(d) + log m log2(e), the running maximum M and sum Z
//   of a row, P = 2^(S - M) through shared memory, O = O 2^(M_old - M) + P V,
// fp32 throughout; quantised rows become fp32, code times scale, on their way into
// shared memory.  FMA-bound: 2 x 64 x 64 x d FMAs a tile whatever of the 64 rows
// are there: 48 TFLOP/s of 74 at d = 128, 45 at 64; quantised, whose codes every thread
// turns into fp32 between two products, 36 and 34.  128 threads own 8 x 4 scores and 8 x d / 16 sums each; packed fp32x2
// FMA.  K of the next tile arrives under PV, V under S.
#include "quant.cuh"
#include "shared.cuh"
#include "tc.cuh"

#include <math.h>

#include <atomic>

namespace gkv {
namespace serve {
namespace {

constexpr int kR = kShRowsF32, kK = kShKeysF32, kThreads = 128;

template <int D>
struct Cfg {
    static constexpr int Q = kR * D, K = kK * D, V = kK * D, P = kR * kK;
    static constexpr size_t SMEM = (size_t)(Q + K + V + P) * sizeof(float);
};

__device__ __forceinline__ void copy16(float *dst, const float *src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D, bool QUANT>
__global__ void __launch_bounds__(kThreads, 2) shared_f32_kernel(const SharedArgs a) {
    using C = Cfg<D>;
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = Qs + C::Q, *Vs = Ks + C::K, *Ps = Vs + C::V;
    __shared__ int row_s[2][kK];           // pool rows of a tile's entries, -1: not there
    __shared__ float bias_s[2][kK];        // log m, base 2
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    next_may_start();
    after_previous();
    const int4 w0 = a.plan.piece[2 * blockIdx.x], w1 = a.plan.piece[2 * blockIdx.x + 1];
    if ((int)blockIdx.x >= *a.plan.pieces) return;
    const int b0 = w0.y, nb = w0.z, len = w0.w, g = w1.x, j0 = w1.y, j1 = w1.z, gq = a.c.Hq / a.c.G;
    const int64_t seq = (int64_t)w0.x * a.c.G + g;

    // the entries of tile j, by the first 64 threads
    auto find = [&](int j) {
        if (tid < kK && j < j1) {
            const int e = j * kK + tid;
            const Paged look{nullptr, nullptr, nullptr, a.table, nullptr, 0, 0, 0, 0, a.c.page_size, a.c.max_pages, a.c.n_pages};
            const int row = e < len ? (int)entry_row(look, seq, e, a.status) : -1;
            float lm = row >= 0 && a.c.log_m ? a.c.log_m[row] : 0.f;
            if (fabsf(lm) <= FLT_MAX) lm = fminf(fmaxf(lm * kLog2e, -kShMost), kShMost);
            row_s[j & 1][tid] = row;
            bias_s[j & 1][tid] = lm;
        }
    };
    // four channels (c) of the entry in place r of tile j
    auto load4 = [&](float *dst, const char *pool, const uint8_t *scales, int j, int r, int c) {
        const int row = row_s[j & 1][r];
        if constexpr (QUANT) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row >= 0) {
                const uint32_t u = *reinterpret_cast<const uint32_t *>(pool + (int64_t)row * D + c * 4);
                const float s = scale_of(scales[row]);
                const float2 x = values2(u & 0xffffu), y = values2(u >> 16);
                v = make_float4(x.x * s, x.y * s, y.x * s, y.y * s);
            }
            *reinterpret_cast<float4 *>(dst) = v;
        } else {
            copy16(dst, reinterpret_cast<const float *>(pool) + (int64_t)(row < 0 ? 0 : row) * D + c * 4, row >= 0);
        }
    };
    // 16-byte chunks of a key are permuted by key % 8, as 8 lanes read one chunk of 8 keys
    auto load_k = [&](int j) {
        for (int i = tid; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4);
            load4(Ks + r * D + (c ^ (r & 7)) * 4, a.c.K, a.scales.k, j, r, c);
        }
        copy_commit();
    };
    auto load_v = [&](int j) {
        for (int i = tid; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4);
            load4(Vs + r * D + c * 4, a.c.V, a.scales.v, j, r, c);
        }
        copy_commit();
    };
    find(j0);
    __syncthreads();
    load_k(j0);
    for (int i = tid; i < kR * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4);
        const bool on = r / gq < nb;
        copy16(Qs + r * D + c * 4, static_cast<const float *>(a.q) + (on ? ((int64_t)(b0 + r / gq) * a.c.Hq + g * gq + r % gq) * D : 0) + c * 4, on);
    }
    copy_commit();

    float2 o[8][D / 32];
    float m[8], z[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma unroll
        for (int c = 0; c < D / 32; c++) o[i][c] = make_float2(0.f, 0.f);
        m[i] = -INFINITY;
        z[i] = 0.f;
    }
    const float sc = a.scale;

    for (int j = j0; j < j1; j++) {
        load_v(j);
        find(j + 1);
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
        float bias[4];
        bool there[4];
#pragma unroll
        for (int c = 0; c < 4; c++) {
            bias[c] = bias_s[j & 1][tx + 16 * c];
            there[c] = row_s[j & 1][tx + 16 * c] >= 0;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float y[4], mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; c++) {
                y[c] = there[c] ? (x[i][c].x + x[i][c].y) * sc + bias[c] : -INFINITY;
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
        __syncthreads();                      // all of K is read, all of P written, the next tile's rows found
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
    // a part: [rows][D] sums, then [rows] references, [rows] sums of weights
    float *pp = a.plan.part + (size_t)blockIdx.x * shared_part_floats(false, D);
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1) z[i] += __shfl_xor_sync(0xffffffffu, z[i], w);
        const int r = ty * 8 + i;
        if (r / gq >= nb) continue;
#pragma unroll
        for (int c = 0; c < D / 64; c++)
            *reinterpret_cast<float4 *>(pp + r * D + c * 64 + tx * 4) =
                make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
        if (tx == 0) { pp[kR * D + r] = m[i]; pp[kR * (D + 1) + r] = z[i]; }
    }
}

template <int D, bool QUANT>
cudaError_t launch(const SharedArgs &a, cudaStream_t s) {
    static std::atomic<int> ready[kMaxDevices];
    const auto kern = shared_f32_kernel<D, QUANT>;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev].store(1, std::memory_order_relaxed);
    }
    return launch_overlapped(kern, dim3((unsigned)shared_pieces(false, a.blocks)), kThreads, Cfg<D>::SMEM, s, a);
}

}  // namespace

cudaError_t launch_shared_f32(const SharedArgs &a, int d, bool quant, cudaStream_t s) {
    if (quant) return d == 128 ? launch<128, true>(a, s) : launch<64, true>(a, s);
    return d == 128 ? launch<128, false>(a, s) : launch<64, false>(a, s);
}

}  // namespace serve
}  // namespace gkv
