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
// This file checks the arguments, lays out the workspace (the status word, the
// word on the bounds' order, the parts of split blocks) and joins the parts.
#include "prompt.cuh"
#include "tc.cuh"

#include <math.h>

#include <type_traits>

namespace gkv {
namespace {

using namespace serve;

// Joins some rows of a split block (32 of the tcgen05 kernel's, 8 of the fp32
// kernel's), four channels a thread, over the parts in order with eight loads in
// flight (16 for many fp32 parts): the latency of a read or two.  The
// tcgen05 kernel's parts are read across rows as they lie and turned in shared
// memory, so that rows leave whole.
constexpr int join_rows(bool tc) { return tc ? 32 : 8; }
template <typename T, int D, bool TC>
__global__ void __launch_bounds__(join_rows(TC) * D / 4) prompt_join_kernel(const PromptArgs a) {
    constexpr int ROWS = TC ? kRowsTc : kRowsF32, KEYS = TC ? keys_tc(D) : kKeysF32, LEAST = TC ? least_tc(D) : kLeastF32;
    constexpr int C4 = D / 4, LD = C4 + 1, RB = join_rows(TC);
    constexpr size_t PF = part_floats(ROWS, D);
    __shared__ float4 out_s[TC ? RB * LD : 1];
    __shared__ float m_s[RB], z_s[RB];
    next_may_start();
    after_previous();
    const int gq = a.Hq / a.G, half = TC ? kRowsTc / 2 : kRowsF32, tpt = half / gq, tok = TC ? 2 * tpt : tpt;
    const int g = blockIdx.x % a.G;
    const int slot = (int)prompt_slots(a.n_q, a.n_seqs, tok) - 1 - (int)(blockIdx.x / a.G);
    int s;
    int64_t q0, nq, k0, nk;
    if (!slot_rows(a, slot, tok, s, q0, nq, k0, nk)) return;
    const int64_t t0 = ((int64_t)slot - ((int)q0 / tok + s)) * tok;
    if (t0 < 0 || t0 >= nq) return;
    const int last = (int)((nq < t0 + tok ? nq : t0 + tok) - 1 + nk - nq);
    const int np = parts_of(last >= 0 ? last / KEYS + 1 : 0, a.split, LEAST);
    if (np == 1) return;
    const int r0 = blockIdx.y * RB, i = threadIdx.x;
    const float *p0 = a.part + (size_t)blockIdx.x * a.split * PF;
    const int rr = TC ? i % RB : i / C4, c = TC ? i / RB : i % C4, r = r0 + rr;
    const size_t at = TC ? (size_t)c * ROWS + r : (size_t)r * C4 + c;
    auto token = [&](int row) { return row % half / gq < tpt ? t0 + row / half * tpt + row % half / gq : nq; };
    auto write = [&](int row, int col, float4 v, float M, float Z) {
        const int64_t t = token(row);
        if (t >= nq) return;
        const int h = g * gq + row % half % gq;
        put4(static_cast<T *>(a.out) + (q0 + t) * a.o_ts + h * a.o_hs + col * 4, v);
        if (col == 0 && a.lse)
            a.lse[(q0 + t) * a.Hq + h] = row_lse(M, Z);
    };
    if (token(r) < nq) {
        float M = -INFINITY, Z = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        auto join = [&](auto batch) {
            constexpr int N = decltype(batch)::value;
            for (int b = 0; b < np; b += N) {
                float m[N], z[N], mx = M;
                float4 x[N];
#pragma unroll
                for (int p = 0; p < N; p++) {
                    // past the last part: the last one again, with no weight
                    const float *q = p0 + (size_t)min(b + p, np - 1) * PF;
                    m[p] = q[ROWS * D + r];
                    z[p] = q[ROWS * D + ROWS + r];
                    x[p] = reinterpret_cast<const float4 *>(q)[at];
                }
#pragma unroll
                for (int p = 0; p < N; p++) {
                    if (b + p >= np) m[p] = -INFINITY;
                    mx = fmaxf(mx, m[p]);
                }
                const float sh = mx == -INFINITY ? 0.f : mx, w = tc::ex2(M - sh);
                M = mx;
                Z *= w;
                v.x *= w; v.y *= w; v.z *= w; v.w *= w;
#pragma unroll
                for (int p = 0; p < N; p++) {
                    const float f = tc::ex2(m[p] - sh);
                    Z += f * z[p];
                    v.x += f * x[p].x; v.y += f * x[p].y; v.z += f * x[p].z; v.w += f * x[p].w;
                }
            }
        };
        if (!TC && np > 8) join(std::integral_constant<int, 16>()); else join(std::integral_constant<int, 8>());
        const float inv = row_scale(M, Z);
        v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        if constexpr (TC) {
            out_s[rr * LD + c] = v;
            if (c == 0) { m_s[rr] = M; z_s[rr] = Z; }
        } else {
            write(r, c, v, M, Z);
        }
    }
    if constexpr (TC) {
        __syncthreads();
        write(r0 + i / C4, i % C4, out_s[i / C4 * LD + i % C4], m_s[i / C4], z_s[i / C4]);
    }
}

// One block: do the query bounds ascend?  Before launches of more than kScanSeqs sequences, whose blocks search the
// bounds by halves instead of reading them all: a misplaced word would lead the search astray.
__global__ void __launch_bounds__(1024) prompt_order_kernel(const PromptArgs a) {
    next_may_start();
    after_previous();
    int bad = 0;
    for (int s = threadIdx.x; s < a.n_seqs; s += 1024) bad |= !ascend(a.cu_q[s], a.cu_q[s + 1], a.n_q);
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *a.disorder = bad;
}

template <typename T, bool TC>
cudaError_t join(const PromptArgs &a, int d, cudaStream_t s) {
    constexpr int ROWS = TC ? kRowsTc : kRowsF32;
    const int gq = a.Hq / a.G, tok = TC ? 2 * (kRowsTc / 2 / gq) : kRowsF32 / gq;
    constexpr int RB = join_rows(TC);
    const dim3 grid((unsigned)(prompt_slots(a.n_q, a.n_seqs, tok) * a.G), ROWS / RB);
    return d == 128 ? launch_overlapped(prompt_join_kernel<T, 128, TC>, grid, RB * 32, 0, s, a)
                    : launch_overlapped(prompt_join_kernel<T, 64, TC>, grid, RB * 16, 0, s, a);
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
    if (p->n_seqs < 0 || p->n_q < 0 || p->n_k < 0 || p->n_q > (1LL << 31) - 4096 || p->n_k > (1LL << 31) - 4096) return GKV_EINVAL;
    if (!p->cu_q || !p->cu_k || !al(p->cu_q, 4) || !al(p->cu_k, 4) || !al(p->lse, 4)) return GKV_EINVAL;
    if (p->n_q > 0 && (!rows_ok(p->q, p->q_ts, p->q_hs, p->dtype) ||
                       !out_ok(p->out, p->o_ts, p->o_hs, p->dtype, p->n_q, p->Hq, p->d)))
        return GKV_EINVAL;
    if (p->n_k > 0 && (!rows_ok(p->k, p->k_ts, p->k_hs, p->dtype) || !rows_ok(p->v, p->v_ts, p->v_hs, p->dtype)))
        return GKV_EINVAL;
    return GKV_OK;
}

}  // namespace

namespace serve {
cudaError_t launch_prompt_join(const PromptArgs &a, int d, int dtype, bool tc_parts, cudaStream_t s) {
    if (dtype == GKV_F32) return join<float, false>(a, d, s);
    return tc_parts ? join<__nv_bfloat16, true>(a, d, s) : join<__nv_bfloat16, false>(a, d, s);
}
}  // namespace serve
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_prompt_workspace_size(const gkv_prompt *p, size_t *bytes) {
    const gkv_status st = check_geometry(p);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    const size_t f32 = serve::kPartsF32 * serve::part_floats(serve::kRowsF32, p->d);
    const size_t tc = p->dtype == GKV_BF16 ? serve::kPartsTc * serve::part_floats(serve::kRowsTc, p->d) : 0;
    *bytes = serve::kWsHead + (f32 > tc ? f32 : tc) * sizeof(float);
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
                              reinterpret_cast<int *>(ws) + 1, reinterpret_cast<float *>(ws + serve::kWsHead), 1};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p->n_seqs > serve::kScanSeqs && launch_overlapped(prompt_order_kernel, 1, 1024, 0, s, a) != cudaSuccess)
        return GKV_ECUDA;
    cudaError_t e = cudaErrorNotSupported;
    if (p->dtype == GKV_BF16) e = serve::launch_prompt_tc(a, p->d, s);
    if (e == cudaErrorNotSupported) e = serve::launch_prompt_f32(a, p->d, p->dtype, s);
    return e == cudaSuccess ? GKV_OK : e == cudaErrorInvalidConfiguration ? GKV_EUNSUPPORTED : GKV_ECUDA;
}

extern "C" gkv_status gracekv_prompt_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
