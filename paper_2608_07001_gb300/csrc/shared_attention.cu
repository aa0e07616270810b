// shared_attention.cu -- attention of one token per request where requests
// share long prefixes (gracekv_shared_*): its plan, its arguments.
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
// The plan: the blocks of rows of all slots, and how many pieces each one's keys
// are cut into, so that the pieces fill the SMs at a time that is the least of 32
// candidates' (one a warp).
#include "shared.cuh"

#include <limits.h>
#include <math.h>

namespace gkv {
namespace {

using namespace serve;

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kPieceStart = 5;             // what a piece costs beside its tiles, in tiles

__device__ __forceinline__ int warp_scan_max(int v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v = max(v, u);
    }
    return v;
}
__device__ __forceinline__ int warp_scan_sum(int v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v += u;
    }
    return v;
}

// keys: of a tile.
__global__ void __launch_bounds__(kPlanThreads) shared_plan_kernel(const SharedArgs a, int keys, int most) {
    __shared__ int w_max[kPlanWarps], w_sum[kPlanWarps], lo_s[kPlanThreads], n_s[kPlanThreads], rb_s[kPlanThreads];
    __shared__ long long w_cost[kPlanWarps];
    __shared__ int w_run[kPlanWarps];
    __shared__ unsigned long long total_s;
    __shared__ int blocks_s, most_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.c.G;
    next_may_start();
    if (tid == 0) {
        total_s = 0;
        blocks_s = 0;
        most_s = 0;
    }
    after_previous();
    for (int b = tid; b < a.B; b += kPlanThreads) a.plan.req[b] = make_int2(-1, 0);
    __syncthreads();

    // ---- the slots' requests.  A slot is left out when its words do not ascend within the batch, or when it
    // begins below the end of an earlier one whose own do; the others have their requests to themselves.
    int end = 0, base = 0;                               // largest end, blocks of rows so far
    for (int p0 = 0; p0 < a.P; p0 += kPlanThreads) {
        const int p = p0 + tid;
        int lo = 0, hi = 0;
        if (p < a.P) {
            lo = a.cu ? a.cu[p] : 0;
            hi = a.cu ? a.cu[p + 1] : a.B;
        }
        const bool fits = lo >= 0 && lo <= hi && hi <= a.B;
        const int upto = warp_scan_max(fits ? hi : 0);
        if (lane == 31) w_max[warp] = upto;
        __syncthreads();
        int before = __shfl_up_sync(0xffffffffu, upto, 1);
        if (lane == 0) before = 0;
        before = max(before, end);
        for (int w = 0; w < kPlanWarps; w++) {
            if (w < warp) before = max(before, w_max[w]);
            end = max(end, w_max[w]);
        }
        const bool owned = p < a.P && fits && (lo >= before || lo == hi);
        if (p < a.P && !owned) atomicOr(a.status, kStRange);
        const int n = owned ? hi - lo : 0, rb = (n + a.tok - 1) / a.tok;
        const int incl = warp_scan_sum(rb);
        if (lane == 31) w_sum[warp] = incl;
        __syncthreads();
        int first = base + incl - rb;
        for (int w = 0; w < kPlanWarps; w++) {
            if (w < warp) first += w_sum[w];
            base += w_sum[w];
        }
        lo_s[tid] = lo;
        n_s[tid] = n;
        rb_s[tid] = first;
        __syncthreads();
        for (int s = warp; s < min(kPlanThreads, a.P - p0); s += kPlanWarps) {
            const int l0 = lo_s[s], ns = n_s[s], r0 = rb_s[s];
            for (int i = lane; i < ns; i += 32) a.plan.req[l0 + i] = make_int2(r0 + i / a.tok, i % a.tok);
            const int nb = (ns + a.tok - 1) / a.tok * G;
            for (int i = lane; i < nb; i += 32) {
                const int rb_i = i / G, g = i % G, len = a.lens[(int64_t)(p0 + s) * G + g];
                const int cap = a.c.page_size * a.c.max_pages, k = max(0, min(len, cap));
                if (len > cap) atomicOr(a.status, kStRange);
                a.plan.blk[(r0 + rb_i) * G + g] = make_int4(p0 + s, l0 + rb_i * a.tok, min(a.tok, ns - rb_i * a.tok), k);
                const int t = (k + keys - 1) / keys;
                atomicAdd(&total_s, (unsigned long long)t);
                if (t > 0) atomicAdd(&blocks_s, 1);
                atomicMax(&most_s, t);
            }
        }
        __syncthreads();
    }
    const int blocks = base * G, used = blocks_s, longest = most_s;
    const long long total = (long long)total_s;
    auto tiles = [&](int i) { return (a.plan.blk[i].w + keys - 1) / keys; };

    // ---- tiles of a piece: the candidates lie between an even share of all tiles and what is sure to give no more
    // pieces than there is room for (sum of ceil(t / run) <= total / run + used)
    const int room = most - used;                        // at least half of the SMs, or twice the SMs
    const int share = (int)min((total + most - 1) / most, (long long)INT_MAX), sure = (int)min((total + room - 1) / room, (long long)INT_MAX);
    {
        const long long widest = max((long long)sure, min((long long)longest, 4ll * sure));
        const int run = max(1, (int)(share + (widest - share) * warp / (kPlanWarps - 1)));
        long long n = 0;
        for (int i = lane; i < blocks; i += 32) n += (tiles(i) + run - 1) / run;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        if (lane == 0) {
            w_run[warp] = run;
            w_cost[warp] = n > most ? LLONG_MAX : (n + kShSms - 1) / kShSms * (run + kPieceStart);
        }
    }
    __syncthreads();
    long long best = LLONG_MAX;
    int run = max(1, sure);
    for (int w = 0; w < kPlanWarps; w++)
        if (w_cost[w] < best) {
            best = w_cost[w];
            run = w_run[w];
        }

    // ---- the pieces
    int pieces = 0;
    for (int i0 = 0; i0 < blocks; i0 += kPlanThreads) {
        const int i = i0 + tid;
        const int4 k = i < blocks ? a.plan.blk[i] : make_int4(0, 0, 0, 0);
        const int t = (k.w + keys - 1) / keys, np = (t + run - 1) / run;
        const int incl = warp_scan_sum(np);
        if (lane == 31) w_sum[warp] = incl;
        __syncthreads();
        int first = pieces + incl - np;
        for (int w = 0; w < kPlanWarps; w++) {
            if (w < warp) first += w_sum[w];
            pieces += w_sum[w];
        }
        if (i < blocks) a.plan.first[i] = first;
        // a warp writes the pieces of its 32 blocks, a block at a time
        for (int s = 0; s < 32; s++) {
            const int n = __shfl_sync(0xffffffffu, np, s), f = __shfl_sync(0xffffffffu, first, s), ts = __shfl_sync(0xffffffffu, t, s);
            const int4 ks = make_int4(__shfl_sync(0xffffffffu, k.x, s), __shfl_sync(0xffffffffu, k.y, s),
                                      __shfl_sync(0xffffffffu, k.z, s), __shfl_sync(0xffffffffu, k.w, s));
            const int g = (i0 + warp * 32 + s) % G;
            for (int j = lane; j < n; j += 32) {
                a.plan.piece[2 * (f + j)] = ks;
                a.plan.piece[2 * (f + j) + 1] = make_int4(g, (int)((long long)j * ts / n), (int)((j + 1ll) * ts / n), 0);
            }
        }
        __syncthreads();
    }
    if (tid == 0) {
        a.plan.first[blocks] = pieces;
        *a.plan.pieces = pieces;
    }
}

struct Layout {
    int tok;
    int64_t blocks, pieces;
    size_t scratch, counts, req, blk, first, piece, part, bytes;
};

gkv_status layout_of(const gkv_paged_cache *c, const gkv_paged_cache *prefix, Layout &y) {
    gkv_status st = check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if ((st = check_paged_geometry(prefix)) != GKV_OK) return st;
    if (prefix->L != c->L || prefix->G != c->G || prefix->Hq != c->Hq || prefix->d != c->d || prefix->dtype != c->dtype) return GKV_EINVAL;
    const bool bf16 = c->dtype == GKV_BF16;
    y.tok = shared_tok(bf16, c->Hq / c->G);
    y.blocks = shared_row_blocks(c->B, prefix->B, y.tok) * c->G;
    y.pieces = shared_pieces(y.blocks);
    if (y.pieces * 2 >= (1LL << 31)) return GKV_EUNSUPPORTED;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    y.scratch = kWsHead;
    y.counts = up(y.scratch + paged_scratch_bytes(c->d));
    y.req = y.counts + 256;
    y.blk = up(y.req + (size_t)c->B * sizeof(int2));
    y.first = up(y.blk + (size_t)y.blocks * sizeof(int4));
    y.piece = up(y.first + (size_t)(y.blocks + 1) * sizeof(int));
    y.part = up(y.piece + (size_t)y.pieces * 2 * sizeof(int4));
    y.bytes = y.part + (size_t)y.pieces * shared_halves(bf16) * shared_part_floats(bf16, c->d) * sizeof(float);
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
              reinterpret_cast<int4 *>(ws + y.blk), reinterpret_cast<int *>(ws + y.first), reinterpret_cast<float *>(ws + y.part)};
    a.B = c->B;
    a.P = prefix->B;
    a.tok = y.tok;
    a.blocks = (int)y.blocks;
    a.lens = prefix->lens + (int64_t)l * S;
    a.table = prefix->table + (int64_t)l * S * prefix->max_pages;
    a.cu = cu_prefix;
    a.q = q;
    a.status = reinterpret_cast<int *>(ws);
    a.box = prefix->page_size % 64 == 0 ? 64 : prefix->page_size % 32 == 0 ? 32 : 16;
    a.scale = (float)(1.4426950408889634 / sqrt((double)c->d));
    cudaError_t e = serve::launch_overlapped(shared_plan_kernel, 1, kPlanThreads, 0, s, a,
                                             bf16 ? serve::kShKeysTc : serve::kShKeysF32, (int)y.pieces);
    if (e == cudaSuccess) e = bf16 ? serve::launch_shared_tc(a, c->d, prefix_scales, s) : serve::launch_shared_f32(a, c->d, prefix_scales, s);
    if (e != cudaSuccess) return e == cudaErrorInvalidConfiguration ? GKV_EUNSUPPORTED : GKV_ECUDA;
    return serve::paged_attention_call(c, scales, l, q, out, a.status, ws + y.scratch, &a, s);
}

extern "C" gkv_status gracekv_shared_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
