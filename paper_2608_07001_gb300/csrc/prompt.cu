// prompt.cu -- the prompt's attention: causal softmax attention of packed
// sequences with grouped heads (gracekv_prompt_*).
//
// For query i of a sequence with nq queries and nk keys, over its keys
// j <= i + nk - nq:  x_j = q . k_j / sqrt(d),  out = sum_j softmax(x)_j v_j,
// lse = log sum_j exp x_j.  One pass over the keys with the running maximum M
// and sum Z of the softmax: a new maximum M' scales the sums so far by
// exp(M - M').
//
// bf16 runs on tcgen05 (prompt_tc.cu), fp32 on CUDA cores (prompt_f32.cu).
// This file checks the arguments and lays out the workspace: the status word,
// the counters of split blocks, their parts.
#include "prompt.cuh"

#include <math.h>

namespace gkv {
namespace {

using namespace serve;

constexpr size_t kCntBytes = (serve::kPromptParts * sizeof(int) + 255) / 256 * 256;

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

namespace serve {
// The tcgen05 kernel's parts hold 256 rows, the fp32 kernel's 64.
size_t prompt_part_floats(int d, int dtype) { return (size_t)(dtype == GKV_BF16 ? 256 : kPromptF32Rows) * (d + 2); }
}  // namespace serve
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_prompt_workspace_size(const gkv_prompt *p, size_t *bytes) {
    const gkv_status st = check_geometry(p);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = serve::kWsHead + kCntBytes +
             (size_t)serve::kPromptParts * serve::prompt_part_floats(p->d, p->dtype) * sizeof(float);
    return GKV_OK;
}

extern "C" gkv_status gracekv_prompt_attention(const gkv_prompt *p, void *workspace, void *stream) {
    const gkv_status st = check_prompt(p);
    if (st != GKV_OK) return st;
    if (!workspace || !al(workspace, 256)) return GKV_EINVAL;
    if (p->n_seqs == 0 || p->n_q == 0) return GKV_OK;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    const serve::PromptArgs a{p->q, p->k, p->v, p->out, p->lse, p->cu_q, p->cu_k, p->n_seqs, p->G, p->Hq, p->n_q, p->n_k,
                              p->q_ts, p->q_hs, p->k_ts, p->k_hs, p->v_ts, p->v_hs, p->o_ts, p->o_hs,
                              (float)(1.0 / sqrt((double)p->d)), reinterpret_cast<int *>(ws),
                              reinterpret_cast<int *>(ws + serve::kWsHead),
                              reinterpret_cast<float *>(ws + serve::kWsHead + kCntBytes), 1};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaErrorNotSupported;
    if (p->dtype == GKV_BF16) e = serve::launch_prompt_tc(a, p->d, s);
    if (e == cudaErrorNotSupported) e = serve::launch_prompt_f32(a, p->d, p->dtype, s);
    return e == cudaSuccess ? GKV_OK : e == cudaErrorInvalidConfiguration ? GKV_EUNSUPPORTED : GKV_ECUDA;
}

extern "C" gkv_status gracekv_prompt_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
