// paged.cu -- writing the paged cache (gracekv_paged_load / _advance /
// _append).
//
// load: the packed cache of a compressed request becomes its pages, entry for
// entry: one read and one write of 2 d elements and log m per entry.
//
// append: the pair (a, b) = (x[i], x[i + d/2]) of a key or query turns by the
// angle phi = p theta_i, theta_i = base^(-2i/d):  (a cos phi - b sin phi,
// a sin phi + b cos phi).  p can be large while only phi mod 2 pi counts, so
// the angle is kept in turns as a 64-bit fraction: F_i = 2^64 theta_i / (2 pi)
// (host, fp64), and p F_i mod 2^64 is the fraction of a turn -- one integer
// product whose error is |p| times that of F_i, which two powers, a product and a
// quotient in fp64 keep below 2^-53 turns (2^-55 found for bases from 1 to 1e7).
// Its upper 32 bits, rounded to the 24 of a float (2^-26 turns), go to sincospi; of
// quantised pages all 32 count (turn_of), as an angle that is off moves a key over the
// middle between two codes, which is 2^-4 of it.  A
// thread holds 16 bytes of each half of a row, so the rotation stays in its
// registers; its sines and cosines serve every row that it takes.
//
// Both move 2 es d bytes a row (in and out) and are bound by HBM, or by the
// latency of a launch for a few tokens.  GPU time: 128 us for 32768 tokens of
// 32 + 2 x 8 rows of 128 bf16 (805 MB, 6.3 TB/s; 16384 tokens of fp32 120 us,
// 6.7 TB/s), 2.5 us for one token (a call from Python takes 10 to 12); load
// 163 us for 1M entries of 2 x 128 bf16 (1082 MB, 6.6 TB/s).
//
// Quantised pages (quant.cuh): a row's threads find its largest size with shuffles and
// store 1 byte for 2 or 4, so HBM asks for half as much and what bounds both is the
// instructions of a row: the same tokens 138 us (738 MB, 5.3 TB/s), load 150 us (816 MB,
// 5.4 TB/s).
#include "paged.cuh"
#include "quant.cuh"

#include <math.h>

#include <algorithm>

namespace gkv {
namespace {

using namespace serve;

// F_i = a[i / 8] m[i % 8], m in 0.64 fixed point (m[0] is 1): 128 bytes of a
// launch's arguments instead of 512, one high product a pair.
struct Turns {
    unsigned long long a[8], m[8];
    __device__ __forceinline__ unsigned long long at(int i) const {
        const unsigned long long f = a[i >> 3];
        return (i & 7) ? __umul64hi(f, m[i & 7]) : f;
    }
};

// Sine and cosine of u 2^-32 turns, within 1.4 of a float's last bit, on average 0.27 (rounding alone: 0.25): the quadrant nearest, what is left of it as an angle
// y = yh + yl of at most pi / 4 in two floats, and the Taylor series of both there (next terms below 2^-29).
__device__ __forceinline__ void turn_of(unsigned u, float &sn, float &cs) {
    constexpr float kHi = 0x1.921fb60000000p-30f, kLo = -0x1.777a5c0000000p-55f;          // pi 2^-31
    const unsigned q = (u + (1u << 29)) >> 30;
    const int r = (int)(u - (q << 30));
    const float f = (float)(r & ~63), g = __uint_as_float(0x4b000000u | (unsigned)(r & 63)) - 0x1p23f;       // exact
    const float yh = f * kHi, yl = fmaf(g, kHi, fmaf(f, kLo, fmaf(f, kHi, -yh))), z = yh * yh;
    const float ps = z * fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
    const float pc = z * fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f);
    const float s = yh + fmaf(yh, ps, yl), c = 1.f + fmaf(-yh, yl, pc);
    sn = __uint_as_float(__float_as_uint(q & 1 ? c : s) ^ (q & 2) << 30);
    cs = __uint_as_float(__float_as_uint(q & 1 ? s : c) ^ ((q + 1) & 2) << 30);
}

// The table of a base, kept per host thread for the calls of a step (d / 2 fp64
// powers take longer than a launch).
const Turns &turns_of(double base, int d) {
    thread_local double have = 0.0;
    thread_local int have_d = 0;
    thread_local Turns t{};
    if (base > 0.0 && (base != have || d != have_d)) {
        // turns of the pair at position 1: theta / (2 pi), at most 1 / (2 pi) as bases are at least 1
        for (int i = 0; i < 8; i++) {
            const double f = pow(base, -16.0 * i / d) / 6.283185307179586476925287, m = pow(base, -2.0 * i / d);
            t.a[i] = (unsigned long long)ldexp(f, 64);
            t.m[i] = i == 0 ? 0 : m < 1.0 ? (unsigned long long)ldexp(m, 64) : ~0ull;
        }
        have = base;
        have_d = d;
    }
    return t;
}

constexpr int64_t kAppendMany = 1 << 19;      // row chunks from which a thread takes 4 rows

struct AppendArgs {
    Paged c;
    int l, n_tokens;
    const int32_t *cu_new, *pos;
    const char *k, *v, *q;
    char *q_out;
    int64_t k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, qo_ts, qo_hs;     // bytes
    int rotate;
    int *status;
    gkv_paged_scales scales;                   // of quantised pages
};

// Coherent: the kernel before may have written it while this one had begun, and q_out may be q.  As an instruction of
// its own, since the compiler turns the plain dereference of append's conditional rows into more live registers
// than it has (112 bytes of spills; 32768 tokens 181 us instead of 128).
__device__ __forceinline__ uint4 ld16(const char *p) {
    uint4 x;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p) : "memory");
    return x;
}
__device__ __forceinline__ void st16(char *p, uint4 x) { *reinterpret_cast<uint4 *>(p) = x; }

template <typename T>
__device__ __forceinline__ void turn16(uint4 &a, uint4 &b, const float *cs, const float *sn) {
    constexpr int N = 16 / sizeof(T);
    T xa[N], xb[N];
    *reinterpret_cast<uint4 *>(xa) = a;
    *reinterpret_cast<uint4 *>(xb) = b;
#pragma unroll
    for (int j = 0; j < N; j++) {
        const float u = to_f(xa[j]), w = to_f(xb[j]);
        put(&xa[j], u * cs[j] - w * sn[j]);
        put(&xb[j], u * sn[j] + w * cs[j]);
    }
    a = *reinterpret_cast<uint4 *>(xa);
    b = *reinterpret_cast<uint4 *>(xb);
}

// A token has 2 G + Hq rows (keys, values, queries).  One thread: the token,
// one 16-byte chunk of each half, and R of the rows, `stride` apart, so that
// its sines and cosines serve R rows.  Neighbouring threads take neighbouring
// chunks: a row's half is one 64- to 256-byte line.
// Five blocks a SM (48 registers): 128 us at 32768 tokens of 48 rows; four 132 to
// 146, six 139, eight (spills) 168.
// QUANT: a row's lanes find its largest size together and store codes; one row in flight, for the same five blocks (186 us
// of 4 rows with two in flight and four blocks, 178 this way; of 6 rows, read back, 171.8 though 21 registers are spilled,
// 173.5 with four blocks, which spill none).
template <typename T, int D, int R, bool QUANT>
__global__ void __launch_bounds__(256, 5) paged_append_kernel(const AppendArgs a, const __grid_constant__ Turns turns) {
    constexpr int N = 16 / sizeof(T), CH = D / 2 / N, RB = D * sizeof(T), PB = QUANT ? D : RB;      // bytes of a pool row
    next_may_start();
    after_previous();
    if (a.cu_new && blockIdx.x == gridDim.x - 1) {       // a block for the bounds alone, out of the others' way
        for (int b = threadIdx.x; b < a.c.B; b += 256) {
            const int lo = a.cu_new[b], hi = a.cu_new[b + 1];
            if (lo < 0 || hi < lo || hi > a.n_tokens) atomicOr(a.status, kStRange);
        }
        return;
    }
    const int rows = 2 * a.c.G + (a.q ? a.c.Hq : 0), stride = (rows + R - 1) / R;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int ch = (int)(i % CH);
    const int r0 = (int)(i / CH % stride);
    const int64_t t = i / CH / stride;
    if (t >= a.n_tokens) return;
    // the request and the entries from the token to its end: looked up by threads with a key or value row
    int b = (int)t, tail = r0 < 2 * a.c.G ? 1 : 0;
    if (tail && a.cu_new) {
        b = seq_of(a.cu_new, a.c.B, t);
        tail = t >= a.cu_new[b] && t < a.cu_new[b + 1] ? a.cu_new[b + 1] - (int)t : 0;       // 0: of no request
    }
    float cs[N], sn[N];
    if (a.rotate) {
        const long long p = a.pos[t];
#pragma unroll
        for (int j = 0; j < N; j++) {
            const int hi = (int)(((unsigned long long)p * turns.at(ch * N + j)) >> 32);
            if constexpr (QUANT) {
                turn_of((unsigned)hi, sn[j], cs[j]);
            } else {
                sincospif((float)hi * 0x1p-31f, &sn[j], &cs[j]);
            }
        }
    }
    constexpr int U = R < 2 || QUANT ? 1 : 2;       // rows in flight
#pragma unroll 1
    for (int k0 = 0; k0 < R; k0 += U) {
        uint4 x[U], y[U];
        char *dst[U];
        uint8_t *to_scale[U];
#pragma unroll
        for (int k = 0; k < U; k++) {
            const int r = r0 + (k0 + k) * stride;
            dst[k] = nullptr;
            if (r >= rows) continue;
            const char *src;
            if (r >= 2 * a.c.G) {
                const int h = r - 2 * a.c.G;
                src = a.q + t * a.q_ts + h * a.q_hs;
                dst[k] = a.q_out + t * a.qo_ts + h * a.qo_hs;
            } else {
                const bool is_v = r >= a.c.G;
                const int h = is_v ? r - a.c.G : r;
                src = is_v ? a.v + t * a.v_ts + h * a.v_hs : a.k + t * a.k_ts + h * a.k_hs;
                const int64_t s = ((int64_t)a.l * a.c.B + b) * a.c.G + h;
                const int idx = tail ? a.c.lens[s] - tail : -1;
                const int64_t row = idx >= 0 ? entry_row(a.c, s, idx, a.status) : -1;
                if (row >= 0) {
                    dst[k] = (is_v ? a.c.V : a.c.K) + row * PB;
                    if constexpr (QUANT) to_scale[k] = (is_v ? a.scales.v : a.scales.k) + row;
                    if (!is_v && ch == 0 && a.c.log_m) a.c.log_m[row] = 0.f;
                }
            }
            x[k] = ld16(src + ch * 16);
            y[k] = ld16(src + ch * 16 + RB / 2);
        }
#pragma unroll
        for (int k = 0; k < U; k++) {
            if (!dst[k]) continue;
            const int r = r0 + (k0 + k) * stride;
            if constexpr (QUANT) {
                if (r < 2 * a.c.G) {
                    float u[2 * N];
                    unpack16(x[k], reinterpret_cast<float(&)[N]>(u[0]));
                    unpack16(y[k], reinterpret_cast<float(&)[N]>(u[N]));
                    if (a.rotate && r < a.c.G) {
#pragma unroll
                        for (int j = 0; j < N; j++) {
                            const float p = u[j], w = u[N + j];
                            u[j] = p * cs[j] - w * sn[j];
                            u[N + j] = p * sn[j] + w * cs[j];
                        }
                    }
                    const int byte = row_scale<CH>(u);
                    put_codes(reinterpret_cast<uint8_t *>(dst[k]) + ch * N, u, inverse_of(byte), std::integral_constant<int, N>());
                    put_codes(reinterpret_cast<uint8_t *>(dst[k]) + D / 2 + ch * N, u + N, inverse_of(byte), std::integral_constant<int, N>());
                    if (ch == 0) *to_scale[k] = (uint8_t)byte;
                    continue;
                }
            }
            if (a.rotate && (r < a.c.G || r >= 2 * a.c.G)) turn16<T>(x[k], y[k], cs, sn);
            st16(dst[k] + ch * 16, x[k]);
            st16(dst[k] + ch * 16 + RB / 2, y[k]);
        }
    }
}

// R: rows of a thread.  Few tokens want every row on its own thread, the
// latency of one row; many want a thread's sines to serve several (32768 tokens
// of 48 rows of 128 bf16, the time with 1 / 2 / 4 / 8 rows a thread and two in
// flight: 201 / 158 / 137 / 144 us, before five blocks a SM; quantised, one in flight, with the rows read back, 2 / 3 / 4
// / 6 / 8 rows a thread: 204 / 183 / 177 / 170 / 175 us).
template <typename T, int D, bool QUANT>
cudaError_t launch_append(const AppendArgs &a, const Turns &turns, cudaStream_t s) {
    constexpr int CH = D * (int)sizeof(T) / 32;
    const int rows = 2 * a.c.G + (a.q ? a.c.Hq : 0);
    const int64_t one = (int64_t)a.n_tokens * rows * CH;
    constexpr int R = QUANT ? 6 : 4;
    const bool many = one >= kAppendMany;
    const int64_t threads = many ? (int64_t)a.n_tokens * ((rows + R - 1) / R) * CH : one;
    const unsigned n = (unsigned)((threads + 255) / 256) + (a.cu_new ? 1 : 0);
    return launch_overlapped(many ? paged_append_kernel<T, D, R, QUANT> : paged_append_kernel<T, D, 1, QUANT>, n, 256, 0, s, a, turns);
}

__global__ void paged_advance_kernel(int32_t *lens, const int32_t *cu_new, int n, int B, int G) {
    next_may_start();
    after_previous();
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= n) return;
    const int b = i / G % B, len = lens[i];
    lens[i] = len + (cu_new ? max(0, cu_new[b + 1] - cu_new[b]) : (len > 0));
}

struct LoadArgs {
    Paged c;
    int b;
    const char *K, *V;
    const float *log_m;
    const int64_t *off;
    int64_t n_entries;
    int *status;
    gkv_paged_scales scales;
};

// How a lane's P pieces of 16 bytes of a packed row (ch, and ch plus the row's lanes) become a pool row's: as they are, or
// as codes.  The row's lanes call it together.  Codes: two pieces a lane, as what a lane does for an entry bounds it.
template <int BYTES>
struct Plain {
    static constexpr int RB = BYTES, P = 1, CH = RB / 16;
    static __device__ __forceinline__ void put(char *pool, uint8_t *, int64_t row, int ch, const uint4 (&x)[P]) {
        st16(pool + row * RB + ch * 16, x[0]);
    }
};
template <typename T, int D>
struct Quantised {
    static constexpr int RB = D * sizeof(T), N = 16 / sizeof(T), P = 2, CH = RB / 32;
    static __device__ __forceinline__ void put(char *pool, uint8_t *scales, int64_t row, int ch, const uint4 (&x)[P]) {
        float u[2 * N];
        unpack16(x[0], reinterpret_cast<float(&)[N]>(u[0]));
        unpack16(x[1], reinterpret_cast<float(&)[N]>(u[N]));
        const int byte = row_scale<CH>(u);
        uint8_t *p = reinterpret_cast<uint8_t *>(pool) + row * D + ch * N;
        put_codes(p, u, inverse_of(byte), std::integral_constant<int, N>());
        put_codes(p + D / 2, u + N, inverse_of(byte), std::integral_constant<int, N>());
        if (ch == 0) scales[row] = (uint8_t)byte;
    }
};
template <class W>
__device__ __forceinline__ void take(uint4 (&x)[W::P], const char *row, int ch) {
#pragma unroll
    for (int p = 0; p < W::P; p++) x[p] = ld16(row + (ch + p * W::CH) * 16);
}

__device__ __forceinline__ bool head_fits(const LoadArgs &a, int64_t lo, int64_t hi) {
    return lo >= 0 && hi >= lo && hi <= a.n_entries;
}

// Offsets that run backwards or past the entries anywhere lead the search for an entry's head astray, so a block
// then copies the heads [first, first + 256) that fit itself, one after another.  What the search finds is copied
// too: the same entries to the same rows.  A call, so that it costs the caller no registers.
template <class W>
__device__ __noinline__ void load_heads_disordered(const LoadArgs &a, int first) {
    constexpr int RB = W::RB, CH = W::CH;
    const int heads = a.c.L * a.c.G;
    const int64_t cap = (int64_t)a.c.page_size * a.c.max_pages;
    for (int h = first; h < heads && h < first + 256; h++) {
        const int64_t lo = a.off[h], hi = a.off[h + 1];
        if (!head_fits(a, lo, hi)) continue;
        const int64_t n = hi - lo < cap ? hi - lo : cap, s = ((int64_t)(h / a.c.G) * a.c.B + a.b) * a.c.G + h % a.c.G;
        for (int64_t i = threadIdx.x; i < n * CH; i += 256) {
            const int64_t e = i / CH, row = entry_row(a.c, s, (int)e, a.status);
            const int ch = (int)(i % CH);
            if (row < 0) continue;
            uint4 x[W::P], y[W::P];
            take<W>(x, a.K + (lo + e) * RB, ch);
            take<W>(y, a.V + (lo + e) * RB, ch);
            W::put(a.c.K, a.scales.k, row, ch, x);
            W::put(a.c.V, a.scales.v, row, ch, y);
            if (ch == 0 && a.c.log_m) a.c.log_m[row] = a.log_m ? a.log_m[lo + e] : 0.f;
        }
    }
}

// The heads' lengths (offsets that do not fit give 0), one thread per (l, g);
// then a warp copies a run of entries, 16 bytes of the key and of the value a
// lane and IT times.  The head is searched for the run's first entry and
// followed from there.  Eight blocks a SM: the registers that the call would take
// otherwise leave room for six (1M entries of 2 x 256 bytes 163 us, 182 with 40; quantised,
// with 25 of them spilled, and unloaded again 282.7 us, 287 with six).
template <class W, int IT>
__global__ void __launch_bounds__(256, 8) paged_load_kernel(const __grid_constant__ LoadArgs a) {
    constexpr int RB = W::RB, CH = W::CH, RW = CH < 32 ? 32 / CH : 1;         // entries a warp copies at once
    constexpr int U = IT < 4 ? IT : 4;
    next_may_start();
    after_previous();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, cap = (int64_t)a.c.page_size * a.c.max_pages;
    const int heads = a.c.L * a.c.G, lane = threadIdx.x & 31;
    if ((int64_t)blockIdx.x * 256 < heads) {             // a block with a thread per head
        if (i < heads) {
            const int64_t lo = a.off[i], hi = a.off[i + 1];
            int64_t n = hi - lo;
            if (!head_fits(a, lo, hi)) { atomicOr(a.status, kStRange); n = 0; }
            if (n > cap) { atomicOr(a.status, kStRange); n = cap; }
            a.c.lens[((int64_t)(i / a.c.G) * a.c.B + a.b) * a.c.G + i % a.c.G] = (int)n;
        }
        int bad = 0;
        for (int h = threadIdx.x; h < heads; h += 256) bad |= !head_fits(a, a.off[h], a.off[h + 1]);
        if (__syncthreads_or(bad)) load_heads_disordered<W>(a, (int)blockIdx.x * 256);
    }
    const int64_t e0 = (i >> 5) * (RW * IT) + lane / CH;
    if (e0 >= a.n_entries) return;
    int h = 0, hi = heads;
    while (hi - h > 1) {
        const int mid = (h + hi) >> 1;
        if (a.off[mid] <= e0) h = mid; else hi = mid;
    }
    int64_t o0 = a.off[h], o1 = a.off[h + 1];
    const int ch = lane % CH;
#pragma unroll 1
    for (int k0 = 0; k0 < IT; k0 += U) {
        uint4 x[U][W::P], y[U][W::P];
        int64_t row[U];
#pragma unroll
        for (int k = 0; k < U; k++) {
            const int64_t e = e0 + (int64_t)(k0 + k) * RW;
            row[k] = -1;
            if (e >= a.n_entries) continue;
            while (e >= o1 && h + 1 < heads) {
                h++;
                o0 = a.off[h];
                o1 = a.off[h + 1];
            }
            // an entry of no head, of offsets that do not fit, past the table: not copied
            if (o0 < 0 || e < o0 || e >= o1 || o1 > a.n_entries || e - o0 >= cap) continue;
            const int64_t s = ((int64_t)(h / a.c.G) * a.c.B + a.b) * a.c.G + h % a.c.G;
            row[k] = entry_row(a.c, s, (int)(e - o0), a.status);
            take<W>(x[k], a.K + e * RB, ch);
            take<W>(y[k], a.V + e * RB, ch);
        }
#pragma unroll
        for (int k = 0; k < U; k++) {
            if (row[k] < 0) continue;
            W::put(a.c.K, a.scales.k, row[k], ch, x[k]);
            W::put(a.c.V, a.scales.v, row[k], ch, y[k]);
            if (ch == 0 && a.c.log_m) a.c.log_m[row[k]] = a.log_m ? a.log_m[e0 + (int64_t)(k0 + k) * RW] : 0.f;
        }
    }
}

template <class W>
cudaError_t launch_load(const LoadArgs &a, cudaStream_t s) {
    // two entries in flight a lane: 167 us for 1M entries of 2 x 256 bytes; one 187, four 200
    constexpr int IT = W::P == 1 ? 2 : 1;
    constexpr int64_t run = (W::CH < 32 ? 32 / W::CH : 1) * IT;     // entries of a warp
    const int64_t threads = std::max<int64_t>((int64_t)a.c.L * a.c.G, (a.n_entries + run - 1) / run * 32);
    return launch_overlapped(paged_load_kernel<W, IT>, (unsigned)((threads + 255) / 256), 256, 0, s, a);
}

// scales: of a quantised cache, else null.
gkv_status load_call(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t b, const void *K, const void *V,
                     const float *log_m, const int64_t *offsets, int64_t n_entries, void *workspace, void *stream) {
    if (b < 0 || b >= c->B || !offsets || !al(offsets, 8) || n_entries < 0 || n_entries >= (1LL << 31)) return GKV_EINVAL;
    if (n_entries > 0 && (!K || !V || !al(K, 16) || !al(V, 16))) return GKV_EINVAL;
    if (!al(log_m, 4) || (log_m && !c->log_m) || !workspace || !al(workspace, 256)) return GKV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const LoadArgs a{paged_of(c), b, static_cast<const char *>(K), static_cast<const char *>(V), log_m, offsets,
                     n_entries, static_cast<int *>(workspace), scales ? *scales : gkv_paged_scales{}};
    const int rb = c->d * elem_bytes(c->dtype);
    cudaError_t e;
    if (!scales)
        e = rb == 128 ? launch_load<Plain<128>>(a, s) : rb == 256 ? launch_load<Plain<256>>(a, s) : launch_load<Plain<512>>(a, s);
    else if (c->dtype == GKV_BF16)
        e = c->d == 128 ? launch_load<Quantised<__nv_bfloat16, 128>>(a, s) : launch_load<Quantised<__nv_bfloat16, 64>>(a, s);
    else
        e = c->d == 128 ? launch_load<Quantised<float, 128>>(a, s) : launch_load<Quantised<float, 64>>(a, s);
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

template <bool QUANT>
gkv_status append_call(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l, const gkv_paged_tokens *t,
                       void *workspace, void *stream) {
    if (!t || l < 0 || l >= c->L || t->n_tokens < 0 || (!t->cu_new && t->n_tokens != c->B) || !al(t->cu_new, 4))
        return GKV_EINVAL;
    if (!workspace || !al(workspace, 256)) return GKV_EINVAL;
    if (c->rope_base != 0.0 && !(c->rope_base >= 1.0 && c->rope_base < HUGE_VAL)) return GKV_EINVAL;
    const int n_tokens = t->n_tokens;
    if (n_tokens == 0) return GKV_OK;
    if (!t->pos || !al(t->pos, 4) || !rows_ok(t->k, t->k_ts, t->k_hs, c->dtype) || !rows_ok(t->v, t->v_ts, t->v_hs, c->dtype))
        return GKV_EINVAL;
    const void *q = t->q;
    if ((q != nullptr) != (t->q_out != nullptr)) return GKV_EINVAL;
    if (q && (!rows_ok(q, t->q_ts, t->q_hs, c->dtype) ||
              !out_ok(t->q_out, t->qo_ts, t->qo_hs, c->dtype, n_tokens, c->Hq, c->d)))
        return GKV_EINVAL;
    const int es = elem_bytes(c->dtype);
    const AppendArgs a{paged_of(c), l, n_tokens, t->cu_new, t->pos, static_cast<const char *>(t->k),
                       static_cast<const char *>(t->v), static_cast<const char *>(q), static_cast<char *>(t->q_out),
                       t->k_ts * es, t->k_hs * es, t->v_ts * es, t->v_hs * es, t->q_ts * es, t->q_hs * es,
                       t->qo_ts * es, t->qo_hs * es, c->rope_base > 0.0, static_cast<int *>(workspace),
                       scales ? *scales : gkv_paged_scales{}};
    const int64_t items = (int64_t)n_tokens * (2 * c->G + (q ? c->Hq : 0)) * (c->d * es / 32);
    if ((items + 255) / 256 + 1 >= (1LL << 31)) return GKV_EUNSUPPORTED;
    const Turns &turns = turns_of(c->rope_base, c->d);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = c->dtype == GKV_BF16 ? (c->d == 128 ? launch_append<__nv_bfloat16, 128, QUANT>(a, turns, s)
                                                              : launch_append<__nv_bfloat16, 64, QUANT>(a, turns, s))
                                               : (c->d == 128 ? launch_append<float, 128, QUANT>(a, turns, s)
                                                              : launch_append<float, 64, QUANT>(a, turns, s));
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

}  // namespace
}  // namespace gkv

using namespace gkv;

extern "C" gkv_status gracekv_paged_load(const gkv_paged_cache *c, int32_t b, const void *K, const void *V,
                                         const float *log_m, const int64_t *offsets, int64_t n_entries,
                                         void *workspace, void *stream) {
    const gkv_status st = check_paged(c);
    return st != GKV_OK ? st : load_call(c, nullptr, b, K, V, log_m, offsets, n_entries, workspace, stream);
}

extern "C" gkv_status gracekv_quant_load(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t b, const void *K,
                                         const void *V, const float *log_m, const int64_t *offsets, int64_t n_entries,
                                         void *workspace, void *stream) {
    const gkv_status st = check_quant(c, scales);
    return st != GKV_OK ? st : load_call(c, scales, b, K, V, log_m, offsets, n_entries, workspace, stream);
}

extern "C" gkv_status gracekv_paged_advance(const gkv_paged_cache *c, const int32_t *cu_new, void *stream) {
    const gkv_status st = check_paged(c);
    if (st != GKV_OK) return st;
    if (!al(cu_new, 4)) return GKV_EINVAL;
    const int n = c->L * c->B * c->G;
    const cudaError_t e = launch_overlapped(paged_advance_kernel, (n + 255) / 256, 256, 0, static_cast<cudaStream_t>(stream),
                                            c->lens, cu_new, n, c->B, c->G);
    return e == cudaSuccess ? GKV_OK : GKV_ECUDA;
}

extern "C" gkv_status gracekv_paged_append(const gkv_paged_cache *c, int32_t l, const gkv_paged_tokens *t,
                                           void *workspace, void *stream) {
    const gkv_status st = check_paged(c);
    return st != GKV_OK ? st : append_call<false>(c, nullptr, l, t, workspace, stream);
}

extern "C" gkv_status gracekv_quant_append(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l,
                                           const gkv_paged_tokens *t, void *workspace, void *stream) {
    const gkv_status st = check_quant(c, scales);
    return st != GKV_OK ? st : append_call<true>(c, scales, l, t, workspace, stream);
}

extern "C" gkv_status gracekv_paged_status(void *workspace, void *stream) {
    return serve::read_status(workspace, stream);
}
