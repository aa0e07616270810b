// paged.cuh -- the paged cache as the kernels see it, and its host checks.
#pragma once

#include "serve.cuh"

namespace gkv {
namespace serve {

struct Paged {
    char *K, *V;
    float *log_m;
    const int32_t *table;
    int32_t *lens;
    int L, B, G, Hq, page_size, max_pages;
    int64_t n_pages;
};

inline Paged paged_of(const gkv_paged_cache *c) {
    return Paged{static_cast<char *>(c->K), static_cast<char *>(c->V), c->log_m, c->table, c->lens,
                 c->L, c->B, c->G, c->Hq, c->page_size, c->max_pages, c->n_pages};
}

inline gkv_status check_paged_geometry(const gkv_paged_cache *c) {
    if (!c || c->L <= 0 || c->B <= 0 || c->G <= 0 || c->Hq <= 0 || c->Hq % c->G) return GKV_EINVAL;
    if (c->dtype != GKV_F32 && c->dtype != GKV_BF16) return GKV_EINVAL;
    if ((int64_t)c->L * c->B * c->G >= (1LL << 31)) return GKV_EINVAL;
    if ((c->d != 64 && c->d != 128) || c->Hq / c->G > 8) return GKV_EUNSUPPORTED;
    return GKV_OK;
}

inline gkv_status check_paged(const gkv_paged_cache *c) {
    const gkv_status st = check_paged_geometry(c);
    if (st != GKV_OK) return st;
    if (c->page_size < 1 || c->max_pages < 1 || c->n_pages < 1 || c->n_pages >= (1LL << 31) / c->page_size) return GKV_EINVAL;
    if ((int64_t)c->page_size * c->max_pages > (1LL << 31) - 4096) return GKV_EINVAL;
    if (!c->K || !c->V || !c->table || !c->lens) return GKV_EINVAL;
    if (!al(c->K, 16) || !al(c->V, 16) || !al(c->log_m, 16) || !al(c->table, 4) || !al(c->lens, 4)) return GKV_EINVAL;
    return GKV_OK;
}

// Pool row of entry idx of sequence s = (l B + b) G + g; -1 (and the status
// bit) when the table does not lead into the pool.
__device__ __forceinline__ int64_t entry_row(const Paged &c, int64_t s, int idx, int *status) {
    const int slot = idx / c.page_size;
    const int page = slot < c.max_pages ? c.table[s * c.max_pages + slot] : -1;
    if ((unsigned)page >= (unsigned)c.n_pages) {
        atomicOr(status, kStRange);
        return -1;
    }
    return (int64_t)page * c.page_size + (idx - slot * c.page_size);
}

}  // namespace serve
}  // namespace gkv
