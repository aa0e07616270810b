// shared.cuh -- the attention over a shared prefix as its kernels see it.
//
// Requests [cu[p], cu[p + 1]) of a batch share slot p of a prefix cache.  Three
// launches: the requests' own entries (paged_attention.cu), whose first block makes
// the plan meanwhile (shared_plan.cuh); the slots' entries, for all their requests at
// once (shared_tc.cu, shared_f32.cu); and the join of the parts that both leave
// (shared_attention.cu).
//
// The rows of (slot, KV head) are its requests' gq query heads, `tok` requests
// to a block of rows; a block's key tiles are cut into pieces, one CTA each.
#pragma once

#include "paged.cuh"

namespace gkv {
namespace serve {

constexpr int kShSms = 152;
// log m (base 2) counts up to this size, in the prefix and in the own entries, so that it stays a number beside every
// scale and masks of the type's lowest value meet there.
constexpr float kShMost = 0x1p40f;
constexpr int kShRowsTc = 128, kShRowsF32 = 64;        // rows of a part
constexpr int kShKeysTc = 128, kShKeysF32 = 64;        // keys of a tile

// Requests of a block of rows: two row tiles (bf16) or one (fp32).
__host__ __device__ constexpr int shared_tok(bool bf16, int gq) { return bf16 ? 2 * (kShRowsTc / gq) : kShRowsF32 / gq; }
// Blocks of rows of one KV head at most: sum over slots of ceil(n_p / tok).
__host__ __device__ inline int64_t shared_row_blocks(int B, int P, int tok) { return (int64_t)B / tok + P; }
// Pieces that run at once: one a SM (bf16), two (fp32: 64 rows of 4 warps; one a SM 24 TFLOP/s at d = 128, two 48).
__host__ __device__ constexpr int shared_at_once(bool bf16) { return bf16 ? kShSms : 2 * kShSms; }
// Pieces at most: as many where the blocks are few enough to share the SMs among them, else (a block's last
// piece is a partial one) twice as many and one more a block.
__host__ __device__ inline int64_t shared_pieces(bool bf16, int64_t blocks) {
    return blocks <= shared_at_once(bf16) / 2 ? shared_at_once(bf16) : blocks + 2 * shared_at_once(bf16);
}
// Floats of a part: sums by 4 channels, the rows' references (base 2), their weights' sums.
__host__ __device__ constexpr size_t shared_part_floats(bool bf16, int d) {
    return (size_t)(bf16 ? kShRowsTc : kShRowsF32) * (d + 2);
}
// Parts of a piece: two (a row tile each, or where the block has one row tile every other key tile each), or one.
__host__ __device__ constexpr int shared_halves(bool bf16) { return bf16 ? 2 : 1; }

// The plan, in the workspace.
struct SharedPlan {
    int *pieces;            // their number
    int4 *piece;            // [pieces][2] (slot, first request, requests, entries), (head, first key tile, end, 0)
    int2 *req;              // [B] (block of rows, place in it) of a request, (-1, 0) for none
    int4 *blk;              // [blocks] (slot, first request, requests, entries); block = block of rows * G + head
    int *first;             // [blocks + 1] first piece
    float *part;            // [pieces][halves][part floats]
    float *own;             // [B][Hq][D] sums over the requests' own entries
    float2 *own_mz;         // [B][Hq] their references and sums of weights
};

struct SharedArgs {
    Paged c;                // the prefix cache
    gkv_paged_scales scales;
    SharedPlan plan;
    int B, P, tok, blocks;  // requests, slots, requests of a block of rows, blocks at most
    int keys, pieces;       // keys of a tile, pieces at most
    int two;                // what a key tile costs with more than half of a block's requests (shared_plan.cuh)
    const int32_t *lens, *table;                       // of the layer
    const int32_t *cu;      // [P + 1]; null: one slot for all
    const void *q;          // [B][Hq][d]
    int *status;
    int box;                // rows of a TMA box
    float scale;            // log2(e) / sqrt(d)
};

// Where a request's rows of the prefix's parts are: count parts from `at`, `step` floats apart, its first head at row.
struct PrefixParts {
    const float *at;
    int count, row;
    int64_t step;
};
template <bool BF16, int D>
__device__ __forceinline__ PrefixParts prefix_parts(const SharedPlan &p, int tok, int b, int g, int G, int gq) {
    constexpr int64_t PF = (int64_t)shared_part_floats(BF16, D);
    PrefixParts r{nullptr, 0, 0, 0};
    const int2 rq = p.req[b];
    if (rq.x < 0) return r;
    const int block = rq.x * G + g, p0 = p.first[block], n = p.first[block + 1] - p0;
    if constexpr (BF16) {
        const int tpt = tok / 2;
        const bool two = p.blk[block].z > tpt;
        const int half = two && rq.y >= tpt;
        r.row = (rq.y - half * tpt) * gq;
        r.count = two ? n : 2 * n;
        r.step = two ? 2 * PF : PF;
        r.at = p.part + (2 * (int64_t)p0 + half) * PF;
    } else {
        r.row = rq.y * gq;
        r.count = n;
        r.step = PF;
        r.at = p.part + p0 * PF;
    }
    return r;
}

cudaError_t launch_shared_tc(const SharedArgs &a, int d, bool quant, cudaStream_t s);
cudaError_t launch_shared_f32(const SharedArgs &a, int d, bool quant, cudaStream_t s);

// Attention of a request's own entries (paged_attention.cu): out; or, with shared, the plan of the prefix and the own
// parts.  Its scratch: paged_scratch_bytes(d), zeroed once.
size_t paged_scratch_bytes(int d);
gkv_status paged_attention_call(const gkv_paged_cache *c, const gkv_paged_scales *scales, int32_t l, const void *q, void *out,
                                int *status, void *scratch, const SharedArgs *shared, cudaStream_t s);

}  // namespace serve
}  // namespace gkv
