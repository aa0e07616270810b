// paged_read.cu -- entries leave the paged cache (gracekv_paged_read /
// _unload): the inverses of its append and of its load, of plain pages and of
// quantised ones, whose rows become code 2^e, exact in fp32 and bf16.
//
// read: a row of tokens is the same entry of every head, so a chunk that
// continues a prompt finds the sequence as the prompt's attention takes it.
// unload: the entries of all layers as one packed cache, offsets first (a launch
// of one block), then the rows.
// One read and one write of every row, bound by HBM.  Quantised, of d = 128 into bf16: 16
// heads' rows of 32768 tokens 33 us (6.2 TB/s), 1M entries 134 us (6.1 TB/s) and 4 of the offsets.
#include "paged.cuh"
#include "quant.cuh"

#include <algorithm>
#include <type_traits>

namespace gkv {
namespace {

using namespace serve;

// A lane's two pieces of 16 bytes of a row in T (ch, and ch plus the row's lanes), from a pool of S.
template <typename T, typename S, int D>
struct Row {
    static constexpr int N = 16 / sizeof(T), CH = D / N / 2, PB = D * sizeof(S);
    struct Raw { uint4 u[2]; int byte; };
    // Plain loads: the launch before may still be writing when this kernel begins.
    static __device__ __forceinline__ Raw load(const char *pool, const uint8_t *scales, int64_t row, int ch) {
        Raw r;
        r.byte = 0;
        const char *p = pool + row * PB;
        if constexpr (sizeof(S) == sizeof(T)) {
#pragma unroll
            for (int i = 0; i < 2; i++) r.u[i] = *reinterpret_cast<const uint4 *>(p + (ch + i * CH) * 16);
        } else {
            r.byte = scales[row];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                if constexpr (N == 8) {
                    const uint2 c = *reinterpret_cast<const uint2 *>(p + (ch + i * CH) * 8);
                    r.u[i] = make_uint4(c.x, c.y, 0, 0);
                } else {
                    r.u[i] = make_uint4(*reinterpret_cast<const uint32_t *>(p + (ch + i * CH) * 4), 0, 0, 0);
                }
            }
        }
        return r;
    }
    static __device__ __forceinline__ uint4 value(const Raw &r, int i) {
        const uint4 u = r.u[i];
        if constexpr (sizeof(S) == sizeof(T)) {
            return u;
        } else {
            const float s = scale_of(r.byte);
            if constexpr (N == 8) {
                auto two = [&](uint32_t c) {
                    const float2 v = values2(c);
                    return bf16x2_of(v.x * s, v.y * s);
                };
                return make_uint4(two(u.x & 0xffffu), two(u.x >> 16), two(u.y & 0xffffu), two(u.y >> 16));
            } else {
                const float2 a = values2(u.x & 0xffffu), b = values2(u.x >> 16);
                return make_uint4(__float_as_uint(a.x * s), __float_as_uint(a.y * s), __float_as_uint(b.x * s),
                                  __float_as_uint(b.y * s));
            }
        }
    }
    // The row at p, or zeros.
    static __device__ __forceinline__ void put(char *p, int ch, const Raw &r, bool there) {
#pragma unroll
        for (int i = 0; i < 2; i++)
            *reinterpret_cast<uint4 *>(p + (ch + i * CH) * 16) = there ? value(r, i) : make_uint4(0, 0, 0, 0);
    }
};

struct ReadArgs {
    Paged c;
    gkv_paged_scales scales;
    int l, n_tokens;
    const int32_t *cu_new;
    char *k, *v;
    int64_t k_ts, k_hs, v_ts, v_hs;            // bytes
    int *status;
};

// A thread: two pieces of 16 bytes of the key's row and of the value's row of one entry.
template <typename T, typename S, int D>
__global__ void __launch_bounds__(256) paged_read_kernel(const ReadArgs a) {
    using X = Row<T, S, D>;
    next_may_start();
    after_previous();
    if (a.cu_new && blockIdx.x == gridDim.x - 1) {       // a block for the bounds alone
        for (int b = threadIdx.x; b < a.c.B; b += 256) {
            const int lo = a.cu_new[b], hi = a.cu_new[b + 1];
            if (lo < 0 || hi < lo || hi > a.n_tokens) atomicOr(a.status, kStRange);
        }
        return;
    }
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int ch = (int)(i % X::CH), h = (int)(i / X::CH % a.c.G);
    const int64_t t = i / X::CH / a.c.G;
    if (t >= a.n_tokens) return;
    int b = (int)t, tail = 1;
    if (a.cu_new) {
        b = seq_of(a.cu_new, a.c.B, t);
        if (t < a.cu_new[b] || t >= a.cu_new[b + 1]) return;           // of no request
        tail = a.cu_new[b + 1] - (int)t;
    }
    const int64_t s = ((int64_t)a.l * a.c.B + b) * a.c.G + h;
    const int idx = a.c.lens[s] - tail;
    const int64_t row = idx >= 0 ? entry_row(a.c, s, idx, a.status) : -1;
    typename X::Raw x, y;
    if (row >= 0) {
        x = X::load(a.c.K, a.scales.k, row, ch);
        y = X::load(a.c.V, a.scales.v, row, ch);
    }
    X::put(a.k + t * a.k_ts + h * a.k_hs, ch, x, row >= 0);
    X::put(a.v + t * a.v_ts + h * a.v_hs, ch, y, row >= 0);
}

struct UnloadArgs {
    Paged c;
    gkv_paged_scales scales;
    int b;
    char *K, *V;
    float *log_m;
    int64_t *off;
    int64_t n_entries;
    int *status;
};

// offsets[i] = the entries of the heads before i.
__global__ void __launch_bounds__(1024) paged_offsets_kernel(const UnloadArgs a) {
    __shared__ long long wsum[32];
    next_may_start();
    after_previous();
    const int heads = a.c.L * a.c.G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t cap = (int64_t)a.c.page_size * a.c.max_pages;
    long long base = 0;
    bool bad = false;
    for (int h0 = 0; h0 < heads; h0 += 1024) {
        const int h = h0 + threadIdx.x;
        long long n = 0;
        if (h < heads) {
            n = a.c.lens[((int64_t)(h / a.c.G) * a.c.B + a.b) * a.c.G + h % a.c.G];
            bad = bad || n < 0 || n > cap;
            n = n < 0 ? 0 : n > cap ? cap : n;
        }
        long long incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) wsum[warp] = incl;
        __syncthreads();
        long long before = base, all = base;
        for (int w = 0; w < 32; w++) {
            if (w < warp) before += wsum[w];
            all += wsum[w];
        }
        if (h < heads) a.off[h] = before + incl - n;
        base = all;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.off[heads] = base;
        bad = bad || base > a.n_entries;
    }
    if (bad) atomicOr(a.status, kStRange);
}

// A thread: two pieces of 16 bytes of the key's row and of the value's row of one entry.
template <typename T, typename S, int D>
__global__ void __launch_bounds__(256) paged_unload_kernel(const UnloadArgs a) {
    using X = Row<T, S, D>;
    constexpr int CH = X::CH, RB = D * sizeof(T);
    next_may_start();
    after_previous();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int heads = a.c.L * a.c.G, ch = (int)(i % CH);
    const int64_t e = i / CH;
    if (e >= a.n_entries) return;
    int h = 0, hi = heads;
    while (hi - h > 1) {
        const int mid = (h + hi) >> 1;
        if (a.off[mid] <= e) h = mid; else hi = mid;
    }
    if (e >= a.off[h + 1]) return;                       // past the request's last one
    const int64_t row = entry_row(a.c, ((int64_t)(h / a.c.G) * a.c.B + a.b) * a.c.G + h % a.c.G, (int)(e - a.off[h]), a.status);
    typename X::Raw x, y;
    if (row >= 0) {
        x = X::load(a.c.K, a.scales.k, row, ch);
        y = X::load(a.c.V, a.scales.v, row, ch);
    }
    X::put(a.K + e * RB, ch, x, row >= 0);
    X::put(a.V + e * RB, ch, y, row >= 0);
    if (ch == 0 && a.log_m) a.log_m[e] = row >= 0 && a.c.log_m ? a.c.log_m[row] : 0.f;
}

template <typename T, typename S, int D>
cudaError_t launch_read(const ReadArgs &a, cudaStream_t s) {
    const int64_t threads = (int64_t)a.n_tokens * a.c.G * Row<T, S, D>::CH;
    return launch_overlapped(paged_read_kernel<T, S, D>, (unsigned)((threads + 255) / 256) + (a.cu_new ? 1 : 0), 256, 0, s, a);
}

template <typename T, typename S, int D>
cudaError_t launch_unload(const UnloadArgs &a, cudaStream_t s) {
    cudaError_t e = launch_overlapped(paged_offsets_kernel, 1, 1024, 0, s, a);
    if (e != cudaSuccess || a.n_entries == 0) return e;
    return launch_overlapped(paged_unload_kernel<T, S, D>, (unsigned)((a.n_entries * Row<T, S, D>::CH + 255) / 256), 256, 0, s, a);
}

// f(rows' type, pools' type, channels) of a cache.
template <typename F>
cudaError_t by_type(const gkv_paged_cache *c, bool quant, F f) {
    auto dim = [&](auto t, auto p) {
        return c->d == 128 ? f(t, p, std::integral_constant<int, 128>()) : f(t, p, std::integral_constant<int, 64>());
    };
    if (c->dtype == GKV_BF16) return quant ? dim(__nv_bfloat16(), E4m3()) : dim(__nv_bfloat16(), __nv_bfloat16());
    return quant ? dim(0.f, E4m3()) : dim(0.f, 0.f);
}

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_paged_read(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l,
                                         const gkv_paged_rows *r, void *workspace, void *stream) {
    const gkv_status st = scales ? serve::check_quant(c, scales) : serve::check_paged(c);
    if (st != GKV_OK) return st;
    if (!r || l < 0 || l >= c->L || r->n_tokens < 0 || (!r->cu_new && r->n_tokens != c->B) || !serve::al(r->cu_new, 4))
        return GKV_EINVAL;
    if (!workspace || !serve::al(workspace, 256)) return GKV_EINVAL;
    if (r->n_tokens == 0) return GKV_OK;
    if (!serve::out_ok(r->k, r->k_ts, r->k_hs, c->dtype, r->n_tokens, c->G, c->d) ||
        !serve::out_ok(r->v, r->v_ts, r->v_hs, c->dtype, r->n_tokens, c->G, c->d))
        return GKV_EINVAL;
    const int es = serve::elem_bytes(c->dtype);
    if (((int64_t)r->n_tokens * c->G * (c->d * es / 16) + 255) / 256 + 1 >= (1LL << 31)) return GKV_EUNSUPPORTED;
    const ReadArgs a{serve::paged_of(c), scales ? *scales : gkv_paged_scales{}, l, r->n_tokens, r->cu_new,
                     static_cast<char *>(r->k), static_cast<char *>(r->v), r->k_ts * es, r->k_hs * es, r->v_ts * es,
                     r->v_hs * es, static_cast<int *>(workspace)};
    const cudaError_t e = by_type(c, scales, [&](auto t, auto p, auto d) {
        return launch_read<decltype(t), decltype(p), decltype(d)::value>(a, static_cast<cudaStream_t>(stream));
    });
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

extern "C" gkv_status gracekv_paged_unload(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t b, void *K,
                                           void *V, float *log_m, int64_t *offsets, int64_t n_entries, void *workspace,
                                           void *stream) {
    const gkv_status st = scales ? serve::check_quant(c, scales) : serve::check_paged(c);
    if (st != GKV_OK) return st;
    if (b < 0 || b >= c->B || !offsets || !serve::al(offsets, 8) || n_entries < 0 || n_entries >= (1LL << 31)) return GKV_EINVAL;
    if (n_entries > 0 && (!K || !V || !serve::al(K, 16) || !serve::al(V, 16))) return GKV_EINVAL;
    if (!serve::al(log_m, 4) || !workspace || !serve::al(workspace, 256)) return GKV_EINVAL;
    const UnloadArgs a{serve::paged_of(c), scales ? *scales : gkv_paged_scales{}, b, static_cast<char *>(K),
                       static_cast<char *>(V), log_m, offsets, n_entries, static_cast<int *>(workspace)};
    const cudaError_t e = by_type(c, scales, [&](auto t, auto p, auto d) {
        return launch_unload<decltype(t), decltype(p), decltype(d)::value>(a, static_cast<cudaStream_t>(stream));
    });
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}
