// dm_cache.cuh -- what the kernels of an instance's prefix cache share: the
// host's checks of dm_cache, the layout of its work buffer, small helpers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dm_internal.cuh"

namespace dm {

constexpr uint64_t align_up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }

inline bool aligned(const void *p, uint64_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Shape checks alone: what dm_cache_work_bytes and dm_plan_bytes need.
inline bool cache_shape_ok(const dm_cache *c) {
    if (!c || c->reserved0 || c->dtype > DM_F16 || c->layout > DM_PAGES_TOKENS) return false;
    const uint32_t B = c->page_tokens;
    if (!(B == 4 || B == 8 || B == 16 || B == 32 || B == 64)) return false;
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->kv_heads < 1 || c->kv_heads > 65535 || c->layers < 1) return false;
    if (c->pages < 1 || c->pages > (1u << 30) || c->max_seqs < 1 || c->max_seqs > (1u << 30)) return false;
    if (c->max_blocks < 1 || uint64_t(c->max_blocks) * B >= (1ull << 31)) return false;
    if (c->page_stride % 8 || c->page_stride < uint64_t(c->kv_heads) * B * c->head_dim) return false;
    return c->layer_stride % 8 == 0;
}

// The work buffer of the calls that change pages.  All int32:
//   head[16]           0: 1 if the call may go on, 1: pages it needs or moves, 2: pages in use
//   off[max_seqs + 1]  pages needed before request i
//   aux[max_seqs]      extend: blocks that sequence i holds; fork: the page given to child i
//   mark[max_seqs]     which request named a sequence last
//   list[2 * pages]    compact: free ids below `live`, then pages in use above it
//   to[pages]          compact: where a page moves
struct CacheWork {
    int32_t *head, *off, *aux, *mark, *list, *to;
};
inline uint64_t cache_work_ints(const dm_cache *c) {
    return 16 + align_up(c->max_seqs + 1ull, 4) + 2 * align_up(c->max_seqs, 4) + 3 * align_up(c->pages, 4);
}
inline CacheWork cache_work(const dm_cache *c) {
    CacheWork w;
    w.head = static_cast<int32_t *>(c->work);
    w.off = w.head + 16;
    w.aux = w.off + align_up(c->max_seqs + 1ull, 4);
    w.mark = w.aux + align_up(c->max_seqs, 4);
    w.list = w.mark + align_up(c->max_seqs, 4);
    w.to = w.list + 2 * align_up(c->pages, 4);
    return w;
}

inline bool cache_ok(const dm_cache *c) {
    if (!cache_shape_ok(c) || !c->k || !c->v || !c->tables || !c->lengths || !c->refs || !c->status || !c->work)
        return false;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->refs, 16) || !aligned(c->work, 16)) return false;
    return c->work_bytes >= cache_work_ints(c) * 4;
}

inline dm_status status_of(cudaError_t e) { return e == cudaSuccess ? DM_OK : DM_ERR_CUDA; }

// Elements of a page, and where (head, token) of it begins.
struct PageShape {
    uint32_t heads, tokens, dim, head_step, token_step;
};
inline PageShape page_shape(const dm_cache *c) {
    const bool hf = c->layout == DM_PAGES_HEADS;
    return {c->kv_heads, c->page_tokens, c->head_dim, hf ? c->page_tokens * c->head_dim : c->head_dim,
            hf ? c->head_dim : c->kv_heads * c->head_dim};
}

// The largest i with off[i] <= x, for off[0] <= x < off[n].
__device__ __forceinline__ uint32_t owner_of(const int32_t *off, uint32_t n, int32_t x) {
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (off[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace dm
