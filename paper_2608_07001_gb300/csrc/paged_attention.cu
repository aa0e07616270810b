// paged_attention.cu -- attention of one token per request over the paged
// cache (gracekv_paged_attention; App. A.3, Eq. app_decode_logit).
//
// For every (b, g) and its Hq / G query heads h, over its lens entries e:
//     x_e = q_h . k_e / sqrt(d) + log m_e,  out_h = sum_e softmax(x)_e v_e .
//
// This version: one CTA per (b, h); its warps take every 8th entry with a
// running maximum and sum each, lanes over the channels, and are joined in
// shared memory.
#include "paged.cuh"

#include <math.h>

namespace gkv {
namespace {

using namespace serve;

template <typename T, int D>
__global__ void __launch_bounds__(256) paged_rows_kernel(const Paged c, int l, const T *q, T *out, float scale, int *status) {
    constexpr int E = D / 32;
    __shared__ float sm[8], sz[8], sa[8][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / c.Hq, h = blockIdx.x % c.Hq, g = h / (c.Hq / c.G);
    const int64_t s = ((int64_t)l * c.B + b) * c.G + g;
    const int len = c.lens[s], n = max(0, min(len, c.page_size * c.max_pages));
    if (len > 0 && len > n && threadIdx.x == 0) atomicOr(status, kStRange);
    const T *K = reinterpret_cast<const T *>(c.K), *V = reinterpret_cast<const T *>(c.V);
    float qf[E], acc[E], m = -INFINITY, z = 0.f;
#pragma unroll
    for (int e = 0; e < E; e++) { qf[e] = to_f(q[(size_t)blockIdx.x * D + lane * E + e]); acc[e] = 0.f; }
    for (int j = warp; j < n; j += 8) {
        const int64_t row = entry_row(c, s, j, status);
        if (row < 0) continue;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; e++) x += qf[e] * to_f(K[row * D + lane * E + e]);
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        x = x * scale + (c.log_m ? c.log_m[row] : 0.f);
        if (x == -INFINITY) continue;              // multiplicity 0
        const float mn = fmaxf(m, x), w = __expf(m - mn), p = __expf(x - mn);
        m = mn;
        z = z * w + p;
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] = acc[e] * w + p * to_f(V[row * D + lane * E + e]);
    }
    if (lane == 0) { sm[warp] = m; sz[warp] = z; }
#pragma unroll
    for (int e = 0; e < E; e++) sa[warp][lane * E + e] = acc[e];
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += 256) {
        float M = -INFINITY, num = 0.f, den = 0.f;
        for (int w = 0; w < 8; w++) M = fmaxf(M, sm[w]);
        for (int w = 0; w < 8; w++) {
            const float f = sm[w] == -INFINITY ? 0.f : __expf(sm[w] - M);
            den += f * sz[w];
            num += f * sa[w][i];
        }
        put(out + (size_t)blockIdx.x * D + i, den > 0.f ? num / den : 0.f);
    }
}

template <typename T, int D>
cudaError_t launch(const Paged &c, int l, const void *q, void *out, int *status, cudaStream_t s) {
    paged_rows_kernel<T, D><<<c.B * c.Hq, 256, 0, s>>>(c, l, static_cast<const T *>(q), static_cast<T *>(out),
                                                       (float)(1.0 / sqrt((double)D)), status);
    return cudaGetLastError();
}

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_paged_workspace_size(const gkv_paged_cache *c, size_t *bytes) {
    const gkv_status st = serve::check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = serve::kWsHead;
    return GKV_OK;
}

extern "C" gkv_status gracekv_paged_attention(const gkv_paged_cache *c, int32_t l, const void *q, void *out,
                                              void *workspace, void *stream) {
    const gkv_status st = serve::check_paged(c);
    if (st != GKV_OK) return st;
    if (l < 0 || l >= c->L || !q || !out || !workspace) return GKV_EINVAL;
    if (!serve::al(q, 16) || !serve::al(out, 16) || !serve::al(workspace, 256)) return GKV_EINVAL;
    if (c->page_size % 16) return GKV_EUNSUPPORTED;
    const serve::Paged p = serve::paged_of(c);
    int *status = static_cast<int *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (c->dtype == GKV_BF16)
        e = c->d == 128 ? launch<__nv_bfloat16, 128>(p, l, q, out, status, s) : launch<__nv_bfloat16, 64>(p, l, q, out, status, s);
    else
        e = c->d == 128 ? launch<float, 128>(p, l, q, out, status, s) : launch<float, 64>(p, l, q, out, status, s);
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}
