// shared_attention.cu -- attention of one token per request where requests
// share long prefixes (gracekv_shared_*): its arguments, the join of its parts.
//
// For request b of slot p and a query head of KV head g, over the entries of the
// prefix (l, p, g) and then of the request's own (l, b, g):
//     x_e = q . k_e / sqrt(d) + log m_e,  out = sum_e softmax(x)_e v_e .
// Softmax parts join exactly: with a part's reference M (base 2), sum Z of
// 2^(x - M) and sums O = sum 2^(x - M) v, those of the whole are
//     M = max M_i,  Z = sum 2^(M_i - M) Z_i,  O the same,  out = O / Z,
// so the prefix is attended once for all its requests (their query heads are the
// rows of a matrix product) and only (M, Z, O) is kept of it per row.
// Reading the prefix once bounds it for few requests, the products for many.
//
// Three launches, which overlap at their ends: the own entries and, by one block more,
// the plan (paged_attention.cu, shared_plan.cuh); the prefix (shared_tc.cu, shared_f32.cu); the
// join.  (A last piece that joins, found with a counter, would save the third, but its reads
// are one block's: slower from a few pieces on.)  Of short calls they are all there is: 32
// requests with 200 entries of 8 heads on 4096 quantised ones 30 us: own entries and plan
// 12, the prefix 11 from 1 later on, the join what is left.
//
// The join: a thread holds four channels of a row, over the parts in order with
// eight loads of each in flight, or sixteen (32 requests on 4096 quantised entries, 33 parts
// a row: 31.5 -> 30.2 us).  The bf16 kernel's parts lie by channel, so a warp's
// lanes are rows; the fp32 kernel's by row.
#include "quant.cuh"
#include "shared_plan.cuh"
#include "tc.cuh"

#include <math.h>

namespace gkv {
namespace {

using namespace serve;

constexpr int kJoinThreads = 256, kJoinRows = 32, kJoinC4 = 8;         // rows and groups of 4 channels of a block

__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }

// N: parts in flight, 8 or, where a row has more, 16: a batch is the latency of a read.
template <typename T, int D, int N>
__global__ void __launch_bounds__(kJoinThreads) shared_join_kernel(const SharedArgs a, T *out) {
    constexpr bool BF = sizeof(T) == 2;
    constexpr int R = BF ? kShRowsTc : kShRowsF32;
    __shared__ float4 v_s[kJoinRows][kJoinC4 + 1];
    __shared__ float m_s[kJoinRows], z_s[kJoinRows];
    next_may_start();
    after_previous();
    const int gq = a.c.Hq / a.c.G, reqs = kJoinRows / gq, tid = threadIdx.x;
    const int g = blockIdx.x % a.c.G, b0 = blockIdx.x / a.c.G * reqs, c0 = blockIdx.y * kJoinC4;
    const int rr = BF ? tid % kJoinRows : tid / kJoinC4, cc = BF ? tid / kJoinRows : tid % kJoinC4;
    const int b = b0 + rr / gq, h = rr % gq;
    float M = -INFINITY, Z = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (rr / gq < reqs && b < a.B) {
        const PrefixParts pre = prefix_parts<BF, D>(a.plan, a.tok, b, g, a.c.G, gq);
        const int row = pre.row + h, c4 = c0 + cc;
        for (int p0 = 0; p0 < pre.count; p0 += N) {
            float m[N], z[N], mx = M;
            float4 x[N];
#pragma unroll
            for (int p = 0; p < N; p++) {
                const float *q = pre.at + (int64_t)min(p0 + p, pre.count - 1) * pre.step;
                m[p] = __ldcg(q + R * D + row);
                z[p] = __ldcg(q + R * (D + 1) + row);
                x[p] = __ldcg(reinterpret_cast<const float4 *>(q) + (BF ? c4 * R + row : row * (D / 4) + c4));
            }
#pragma unroll
            for (int p = 0; p < N; p++) {
                // past the last part, or one without an entry, whose sums may be anything
                if (p0 + p >= pre.count || (m[p] == -INFINITY && z[p] == 0.f)) {
                    m[p] = -INFINITY;
                    z[p] = 0.f;
                    x[p] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                mx = fmaxf(mx, m[p]);
            }
            const float sh = shift_of(mx), f = tc::ex2(M - sh);
            M = mx;
            Z *= f;
            v.x *= f; v.y *= f; v.z *= f; v.w *= f;
#pragma unroll
            for (int p = 0; p < N; p++) {
                // (a part of NaN weights alone has reference -inf and a NaN sum, which stays)
                const float w = tc::ex2(m[p] - sh);
                Z += w * z[p];
                v.x += w * x[p].x; v.y += w * x[p].y; v.z += w * x[p].z; v.w += w * x[p].w;
            }
        }
    }
    v_s[rr][cc] = v;
    if (cc == 0) { m_s[rr] = M; z_s[rr] = Z; }
    __syncthreads();
    // the own part, and out: by row
    const int r2 = tid / kJoinC4, k2 = tid % kJoinC4, b2 = b0 + r2 / gq;
    if (r2 / gq >= reqs || b2 >= a.B) return;
    const int64_t at = (int64_t)b2 * a.c.Hq + g * gq + r2 % gq;
    const float2 own = __ldcg(a.plan.own_mz + at);
    const bool none = own.x == -INFINITY && own.y == 0.f;
    const float m1 = m_s[r2], z1 = z_s[r2], mx = fmaxf(m1, none ? -INFINITY : own.x), sh = shift_of(mx);
    float4 x = v_s[r2][k2], y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!none) y = __ldcg(reinterpret_cast<const float4 *>(a.plan.own + at * D) + c0 + k2);
    const float w1 = tc::ex2(m1 - sh), w2 = none ? 0.f : tc::ex2(own.x - sh);
    const float Zs = w1 * z1 + (none ? 0.f : w2 * own.y), r = Zs == 0.f ? 0.f : 1.f / Zs;                // a NaN stays
    put4(out + at * D + (c0 + k2) * 4, make_float4((w1 * x.x + w2 * y.x) * r, (w1 * x.y + w2 * y.y) * r,
                                                   (w1 * x.z + w2 * y.z) * r, (w1 * x.w + w2 * y.w) * r));
}

template <typename T, int D>
cudaError_t launch_join(const SharedArgs &a, void *out, cudaStream_t s) {
    const int reqs = kJoinRows / (a.c.Hq / a.c.G);
    const dim3 grid((unsigned)(((a.B + reqs - 1) / reqs) * a.c.G), D / 4 / kJoinC4);
    // whether a row can have more than eight parts: by the room for them, as the plan's own number is on the device
    const bool many = (int64_t)a.pieces * shared_halves(sizeof(T) == 2) > 8 * (int64_t)a.blocks;
    return launch_overlapped(many ? shared_join_kernel<T, D, 16> : shared_join_kernel<T, D, 8>, grid, kJoinThreads, 0, s, a,
                             static_cast<T *>(out));
}

struct Layout {
    int tok;
    int64_t blocks, pieces;
    size_t scratch, counts, req, blk, first, piece, part, own, own_mz, bytes;
};

gkv_status layout_of(const gkv_paged_cache *c, const gkv_paged_cache *prefix, Layout &y) {
    gkv_status st = check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if ((st = check_paged_geometry(prefix)) != GKV_OK) return st;
    if (prefix->L != c->L || prefix->G != c->G || prefix->Hq != c->Hq || prefix->d != c->d || prefix->dtype != c->dtype) return GKV_EINVAL;
    const bool bf16 = c->dtype == GKV_BF16;
    y.tok = shared_tok(bf16, c->Hq / c->G);
    y.blocks = shared_row_blocks(c->B, prefix->B, y.tok) * c->G;
    y.pieces = shared_pieces(bf16, y.blocks);
    if (y.pieces * 2 >= (1LL << 31)) return GKV_EUNSUPPORTED;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    y.scratch = kWsHead;
    y.counts = up(y.scratch + paged_scratch_bytes(c->d));
    y.req = y.counts + 256;
    y.blk = up(y.req + (size_t)c->B * sizeof(int2));
    y.first = up(y.blk + (size_t)y.blocks * sizeof(int4));
    y.piece = up(y.first + (size_t)(y.blocks + 1) * sizeof(int));
    y.part = up(y.piece + (size_t)y.pieces * 2 * sizeof(int4));
    y.own = up(y.part + (size_t)y.pieces * shared_halves(bf16) * shared_part_floats(bf16, c->d) * sizeof(float));
    y.own_mz = up(y.own + (size_t)c->B * c->Hq * c->d * sizeof(float));
    y.bytes = y.own_mz + (size_t)c->B * c->Hq * sizeof(float2);
    return GKV_OK;
}

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_shared_workspace_size(const gkv_paged_cache *c, const gkv_paged_cache *prefix, size_t *bytes) {
    Layout y;
    const gkv_status st = layout_of(c, prefix, y);
    if (st != GKV_OK) return st;
    if (!bytes) return GKV_EINVAL;
    *bytes = y.bytes;
    return GKV_OK;
}

extern "C" gkv_status gracekv_shared_attention(const gkv_paged_cache *c, const gkv_paged_scales *scales,
                                               const gkv_paged_cache *prefix, const gkv_paged_scales *prefix_scales, int32_t l,
                                               const int32_t *cu_prefix, const void *q, void *out, void *workspace,
                                               void *stream) {
    gkv_status st = scales ? serve::check_quant(c, scales) : serve::check_paged(c);
    if (st != GKV_OK) return st;
    if ((st = prefix_scales ? serve::check_quant(prefix, prefix_scales) : serve::check_paged(prefix)) != GKV_OK) return st;
    Layout y;
    if ((st = layout_of(c, prefix, y)) != GKV_OK) return st;
    if (l < 0 || l >= c->L || !q || !out || !serve::al(q, 16) || !serve::al(out, 16) || !workspace || !serve::al(workspace, 256))
        return GKV_EINVAL;
    if (!serve::al(cu_prefix, 4) || (!cu_prefix && prefix->B != 1)) return GKV_EINVAL;
    if (c->page_size % 16 || prefix->page_size % 16) return GKV_EUNSUPPORTED;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = c->dtype == GKV_BF16;
    const int S = prefix->B * prefix->G;
    serve::SharedArgs a{};
    a.c = serve::paged_of(prefix);
    if (prefix_scales) a.scales = *prefix_scales;
    a.plan = {reinterpret_cast<int *>(ws + y.counts), reinterpret_cast<int4 *>(ws + y.piece), reinterpret_cast<int2 *>(ws + y.req),
              reinterpret_cast<int4 *>(ws + y.blk), reinterpret_cast<int *>(ws + y.first), reinterpret_cast<float *>(ws + y.part),
              reinterpret_cast<float *>(ws + y.own), reinterpret_cast<float2 *>(ws + y.own_mz)};
    a.B = c->B;
    a.P = prefix->B;
    a.tok = y.tok;
    a.blocks = (int)y.blocks;
    a.keys = bf16 ? serve::kShKeysTc : serve::kShKeysF32;
    a.pieces = (int)y.pieces;
    a.two = !bf16 ? serve::kPlanOne : c->d == 128 && !prefix_scales ? serve::kPlanTwoWide : serve::kPlanTwo;
    a.lens = prefix->lens + (int64_t)l * S;
    a.table = prefix->table + (int64_t)l * S * prefix->max_pages;
    a.cu = cu_prefix;
    a.q = q;
    a.status = reinterpret_cast<int *>(ws);
    a.box = prefix->page_size % 64 == 0 ? 64 : prefix->page_size % 32 == 0 ? 32 : 16;
    a.scale = (float)(1.4426950408889634 / sqrt((double)c->d));
    if ((st = serve::paged_attention_call(c, scales, l, q, out, a.status, ws + y.scratch, &a, s)) != GKV_OK) return st;
    cudaError_t e = bf16 ? serve::launch_shared_tc(a, c->d, prefix_scales, s) : serve::launch_shared_f32(a, c->d, prefix_scales, s);
    if (e == cudaSuccess)
        e = bf16 ? (c->d == 128 ? launch_join<__nv_bfloat16, 128>(a, out, s) : launch_join<__nv_bfloat16, 64>(a, out, s))
                 : (c->d == 128 ? launch_join<float, 128>(a, out, s) : launch_join<float, 64>(a, out, s));
    return e == cudaSuccess ? GKV_OK : e == cudaErrorInvalidConfiguration ? GKV_EUNSUPPORTED : GKV_ECUDA;
}

extern "C" gkv_status gracekv_shared_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
