// prompt.cu -- the prompt's attention: causal softmax attention of packed
// sequences with grouped heads (gracekv_prompt_*).
//
// For query i of a sequence with nq queries and nk keys, over its keys
// j <= i + nk - nq:  x_j = q . k_j / sqrt(d),  out = sum_j softmax(x)_j v_j,
// lse = log sum_j exp x_j.  One pass over the keys with the running maximum M
// and sum Z of the softmax: a new maximum M' scales the sums so far by
// exp(M - M').
//
// This version: one warp per (token, query head), lanes over the channels.
#include "prompt.cuh"

#include <math.h>

namespace gkv {
namespace {

using namespace serve;

template <typename T, int D>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const PromptArgs a) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    if (blockIdx.x == 0) check_bounds(a);
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (w >= a.n_q * a.Hq) return;
    const int64_t row = w / a.Hq;
    const int h = (int)(w % a.Hq), g = h / (a.Hq / a.G);
    const int s = seq_of(a.cu_q, a.n_seqs, row);
    int64_t q0, nq, k0, nk;
    if (!seq_bounds(a, s, q0, nq, k0, nk) || row < q0 || row >= q0 + nq) return;      // a row of no sequence
    const int64_t n = row - q0 + nk - nq + 1;      // keys it sees
    const T *q = static_cast<const T *>(a.q) + row * a.q_ts + h * a.q_hs + lane * E;
    const T *k = static_cast<const T *>(a.k) + k0 * a.k_ts + g * a.k_hs + lane * E;
    const T *v = static_cast<const T *>(a.v) + k0 * a.v_ts + g * a.v_hs + lane * E;
    float qf[E], acc[E], m = -INFINITY, z = 0.f;
#pragma unroll
    for (int e = 0; e < E; e++) { qf[e] = to_f(q[e]); acc[e] = 0.f; }
    for (int64_t j = 0; j < n; j++) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; e++) x += qf[e] * to_f(k[j * a.k_ts + e]);
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        x *= a.scale;
        const float mn = fmaxf(m, x), c = __expf(m - mn), p = __expf(x - mn);
        m = mn;
        z = z * c + p;
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] = acc[e] * c + p * to_f(v[j * a.v_ts + e]);
    }
    T *o = static_cast<T *>(a.out) + row * a.o_ts + h * a.o_hs + lane * E;
#pragma unroll
    for (int e = 0; e < E; e++) put(o + e, n > 0 ? acc[e] / z : 0.f);
    if (a.lse && lane == 0) a.lse[row * a.Hq + h] = n > 0 ? m + logf(z) : -INFINITY;
}

gkv_status check_geometry(const gkv_prompt *p) {
    if (!p || p->G <= 0 || p->Hq <= 0 || p->Hq % p->G) return GKV_EINVAL;
    if (p->dtype != GKV_F32 && p->dtype != GKV_BF16) return GKV_EINVAL;
    if ((p->d != 64 && p->d != 128) || p->Hq / p->G > 8) return GKV_EUNSUPPORTED;
    return GKV_OK;
}

gkv_status check_prompt(const gkv_prompt *p) {
    const gkv_status st = check_geometry(p);
    if (st != GKV_OK) return st;
    if (p->n_seqs < 0 || p->n_q < 0 || p->n_k < 0 || p->n_q >= (1LL << 31) || p->n_k >= (1LL << 31)) return GKV_EINVAL;
    if (!p->cu_q || !p->cu_k || !al(p->cu_q, 4) || !al(p->cu_k, 4) || !al(p->lse, 4)) return GKV_EINVAL;
    if (p->n_q > 0 && (!rows_ok(p->q, p->q_ts, p->q_hs, p->dtype) || !rows_ok(p->out, p->o_ts, p->o_hs, p->dtype)))
        return GKV_EINVAL;
    if (p->n_k > 0 && (!rows_ok(p->k, p->k_ts, p->k_hs, p->dtype) || !rows_ok(p->v, p->v_ts, p->v_hs, p->dtype)))
        return GKV_EINVAL;
    return GKV_OK;
}

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_prompt_workspace_size(const gkv_prompt *p, size_t *bytes) {
    const gkv_status st = check_geometry(p);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = serve::kWsHead;
    return GKV_OK;
}

extern "C" gkv_status gracekv_prompt_attention(const gkv_prompt *p, void *workspace, void *stream) {
    const gkv_status st = check_prompt(p);
    if (st != GKV_OK) return st;
    if (!workspace || !al(workspace, 256)) return GKV_EINVAL;
    if (p->n_seqs == 0 || p->n_q == 0) return GKV_OK;
    PromptArgs a{p->q, p->k, p->v, p->out, p->lse, p->cu_q, p->cu_k, p->n_seqs, p->G, p->Hq, p->n_q, p->n_k,
                 p->q_ts, p->q_hs, p->k_ts, p->k_hs, p->v_ts, p->v_hs, p->o_ts, p->o_hs,
                 (float)(1.0 / sqrt((double)p->d)), static_cast<int *>(workspace)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p->dtype == GKV_BF16) {
        const cudaError_t e = serve::launch_prompt_tc(a, p->d, s);
        if (e != cudaErrorNotSupported) return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
    }
    const int64_t blocks = (p->n_q * p->Hq + 7) / 8;
    if (blocks >= (1LL << 31)) return GKV_EUNSUPPORTED;
    const unsigned n = (unsigned)blocks;
    if (p->dtype == GKV_BF16) {
        if (p->d == 128) prompt_rows_kernel<__nv_bfloat16, 128><<<n, 256, 0, s>>>(a);
        else prompt_rows_kernel<__nv_bfloat16, 64><<<n, 256, 0, s>>>(a);
    } else {
        if (p->d == 128) prompt_rows_kernel<float, 128><<<n, 256, 0, s>>>(a);
        else prompt_rows_kernel<float, 64><<<n, 256, 0, s>>>(a);
    }
    return cudaGetLastError() == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

extern "C" gkv_status gracekv_prompt_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
