// dm_pages.cu -- the pages of an instance's prefix cache: growing, forking,
// freeing and compacting (dm_cache_extend, _fork, _free, _compact).
//
// Which pages a call hands out has to be the same every time (the free ids
// from the lowest on), so it is a scan over refs, not a race for a list.  A
// cluster of eight CTAs does it in one launch: every warp owns a run of
// pages, counts, the counts are scanned over the warps and, through
// distributed shared memory, over the CTAs, and a second walk gives each free
// page its rank.  A call that cannot be met is found between the two walks,
// before anything is written.
//
// Bound: latency of one launch where few pages change hands (k_grow 7 to 11 us,
// k_compact_plan 8, k_free 3 to 5); the copies' bandwidth where pages move
// (k_compact_copy below; k_fork_copy 45 us for 512 sequences' last pages in
// eight layers, runs of 0.25 to 4 KB a head).
#include <algorithm>
#include <cooperative_groups.h>

#include "dm_cache.cuh"

namespace cg = cooperative_groups;

namespace dm {
namespace {

constexpr uint32_t kCl = 8;             // CTAs of the cluster
constexpr uint32_t kPt = 1024;          // threads of each
constexpr uint32_t kPw = kPt / 32;
constexpr uint32_t kFewRequests = 2048; // whose places are searched in shared memory
constexpr int kCopyT = 256;             // threads of a copying CTA

struct PagesArgs {
    int32_t *tables, *lengths, *refs;
    uint32_t *status;
    CacheWork w;
    uint32_t pages, B, max_seqs, max_blocks;
};

// Which of pages i .. i+3 (below end) are free, one bit each; i is a
// multiple of 4.
__device__ __forceinline__ uint32_t free4(const int32_t *refs, uint32_t i, uint32_t end) {
    if (i + 4 <= end) {
        const int4 r = __ldcg(reinterpret_cast<const int4 *>(refs + i));
        return (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
    }
    uint32_t m = 0;
    for (uint32_t j = 0; j < 4; ++j)
        if (i + j < end && __ldcg(refs + i + j) == 0) m |= 1u << j;
    return m;
}

// Pages of a warp of the cluster: [begin, end).
__device__ __forceinline__ void warp_run(uint32_t pages, uint32_t gw, uint32_t &begin, uint32_t &end) {
    const uint32_t per = (pages + kCl * kPw * 128 - 1) / (kCl * kPw * 128) * 128;
    begin = min(pages, gw * per);
    end = min(pages, begin + per);
}

// Sums stop at kTooMany, more than the pages of any cache: 1,024 sequences may
// each ask for 2^22 blocks and more, which 32 bits do not hold.
constexpr uint32_t kTooMany = (1u << 30) + 1;

__device__ __forceinline__ uint32_t scan_incl(uint32_t x) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x = min(x + y, kTooMany);
    }
    return x;
}

// Exclusive scan over the CTA's threads; total receives the sum.  Where that is
// kTooMany the scan is not one: the caller refuses the call.
__device__ uint32_t block_scan(uint32_t x, uint32_t *s_warp, uint32_t &total) {
    const uint32_t wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t in = scan_incl(x);
    __syncthreads();
    if (lane == 31) s_warp[wid] = in;
    __syncthreads();
    if (wid == 0) s_warp[lane] = scan_incl(s_warp[lane]);
    __syncthreads();
    total = s_warp[kPw - 1];
    return in - x + (wid ? s_warp[wid - 1] : 0);
}

// Extend (kFork false): request i is (a[i] = sequence, b[i] = tokens to add).
// Fork: (a[i] = parent, c[i] = child, b[i] = tokens to keep); the rows and
// the copies follow in k_fork_copy.
template <bool kFork>
__global__ void __cluster_dims__(kCl, 1, 1) __launch_bounds__(kPt) k_grow(PagesArgs p, const int32_t *a, const int32_t *b,
                                                                        const int32_t *c, uint32_t n) {
    __shared__ uint32_t s_warp[32], s_free, s_need, s_err;
    __shared__ int32_t s_off[kFewRequests + 1];
    pdl_enter();
    cg::cluster_group cl = cg::this_cluster();
    const uint32_t rank = cl.block_rank(), tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    if (tid == 0) s_err = 0;
    __syncthreads();
    if (rank == 0) {
        if (tid == 0 && has_err(p.status)) s_err = ~0u;   // an earlier call's error stands
        const int32_t *own = kFork ? c : a;               // the sequences that change
        for (uint32_t i = tid; i < n; i += kPt)
            if ((uint32_t)own[i] < p.max_seqs) p.w.mark[own[i]] = (int32_t)i;
        __syncthreads();
        uint64_t carry = 0;
        for (uint32_t i0 = 0; i0 < n; i0 += kPt) {
            const uint32_t i = i0 + tid;
            uint32_t need = 0, bad = 0;
            if (i < n) {
                const int32_t s = own[i], x = b[i], from = a[i];
                if ((uint32_t)s >= p.max_seqs || (uint32_t)from >= p.max_seqs || x < 0 || p.w.mark[s] != (int32_t)i) {
                    bad = DM_ERR_INVALID_ARG;
                } else if (kFork) {
                    if (p.lengths[s] != 0 || x > p.lengths[from] || (uint32_t)x > p.max_blocks * p.B) bad = DM_ERR_INVALID_ARG;
                    else need = x % p.B != 0;
                } else {
                    const uint64_t len = (uint32_t)p.lengths[s], nb0 = (len + p.B - 1) / p.B;
                    const uint64_t nb1 = (len + (uint32_t)x + p.B - 1) / p.B;
                    if (nb1 > p.max_blocks) bad = DM_ERR_CAPACITY;
                    else need = (uint32_t)(nb1 - nb0);
                    p.w.aux[i] = (int32_t)nb0;
                }
            }
            if (bad) atomicMax(&s_err, bad == DM_ERR_INVALID_ARG ? 2u : 1u);
            uint32_t total;
            const uint32_t before = block_scan(need, s_warp, total);
            // sums past 2^30 pages are refused below; keep the table in range
            if (i < n) p.w.off[i] = (int32_t)min(carry + before, (uint64_t)1 << 30);
            carry += total;
        }
        if (tid == 0) {
            p.w.off[n] = (int32_t)min(carry, (uint64_t)1 << 30);
            s_need = (uint32_t)min(carry, (uint64_t)0xFFFFFFFFu);
        }
    }
    // the free pages of this warp's run
    uint32_t begin, end, mine = 0;
    warp_run(p.pages, rank * kPw + wid, begin, end);
    for (uint32_t i = begin + lane * 4; i < end; i += 128) mine += __popc(free4(p.refs, i, end));
    mine = __reduce_add_sync(~0u, mine);
    __syncthreads();
    if (lane == 0) s_warp[wid] = mine;
    __syncthreads();
    if (wid == 0) {
        const uint32_t in = scan_incl(s_warp[lane]);
        s_warp[lane] = in - s_warp[lane];   // before this warp
        if (lane == 31) s_free = in;
    }
    cl.sync();
    const uint32_t need = *cl.map_shared_rank(&s_need, 0), err = *cl.map_shared_rank(&s_err, 0);
    uint32_t before = 0, all = 0;
    for (uint32_t r = 0; r < kCl; ++r) {
        const uint32_t f = *cl.map_shared_rank(&s_free, r);
        if (r < rank) before += f;
        all += f;
    }
    const bool ok = err == 0 && need <= all;
    if (rank == 0 && tid == 0) {
        if (!ok && err != ~0u) set_err(p.status, err == 2u ? DM_ERR_INVALID_ARG : DM_ERR_CAPACITY);
        p.w.head[0] = ok;
    }
    const bool few = n <= kFewRequests;
    if (ok && need && few) {
        for (uint32_t i = tid; i <= n; i += kPt) s_off[i] = __ldcg(p.w.off + i);
        __syncthreads();
    }
    const int32_t *off = few ? s_off : p.w.off;
    if (ok) {
        uint32_t next = before + s_warp[wid];
        for (uint32_t i0 = begin; i0 < end && next < need; i0 += 128) {
            const uint32_t i = i0 + lane * 4;
            uint32_t m = i < end ? free4(p.refs, i, end) : 0;
            const uint32_t cnt = __popc(m), in = scan_incl(cnt);
            uint32_t at = next + in - cnt;
            for (; m && at < need; m &= m - 1, ++at) {
                const uint32_t page = i + __ffs(m) - 1, r = owner_of(off, n, (int32_t)at);
                if (kFork) {
                    p.w.aux[r] = (int32_t)page;
                } else {
                    const uint64_t row = (uint64_t)(uint32_t)a[r] * p.max_blocks;
                    p.tables[row + __ldcg(p.w.aux + r) + (at - off[r])] = (int32_t)page;
                }
                p.refs[page] = 1;
            }
            next += __shfl_sync(~0u, in, 31);
        }
        if (!kFork && rank == 0)
            for (uint32_t i = tid; i < n; i += kPt) p.lengths[a[i]] += b[i];
    }
    cl.sync();   // no CTA leaves while another reads its counts
}

// bytes (a multiple of 16) from src to dst by N threads, eight loads of each in
// flight.
template <uint32_t N>
__device__ __forceinline__ void copy_run(char *dst, const char *src, uint32_t bytes, uint32_t thread) {
    constexpr uint32_t U = 8, step = N * 16;
    for (uint32_t i = thread * 16; i < bytes; i += U * step) {
        uint4 x[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
            if (i + u * step < bytes) x[u] = __ldcs(reinterpret_cast<const uint4 *>(src + i + u * step));
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
            if (i + u * step < bytes) __stcs(reinterpret_cast<uint4 *>(dst + i + u * step), x[u]);
    }
}

struct CopyArgs {
    char *k, *v;
    uint64_t layer_bytes, page_bytes;   // strides
    uint32_t layers, heads, row_bytes;  // row_bytes: one token of one head
    uint32_t tokens_first;
};

// One request's share of k_fork_copy is 1 + 2 * layers jobs: its table row,
// then each pool's copied tokens.
__global__ void __launch_bounds__(kCopyT, 4) k_fork_copy(PagesArgs p, CopyArgs c, const int32_t *parents,
                                                      const int32_t *children, const int32_t *keep, uint32_t n) {
    pdl_enter();
    if (p.w.head[0] == 0) return;
    const uint32_t per = 1 + 2 * c.layers;
    for (uint64_t job = blockIdx.x; job < (uint64_t)n * per; job += gridDim.x) {
        const uint32_t i = (uint32_t)(job / per), part = (uint32_t)(job % per), len = (uint32_t)keep[i];
        const uint32_t full = len / p.B, tail = len % p.B;
        const int32_t *from = p.tables + (uint64_t)(uint32_t)parents[i] * p.max_blocks;
        if (part == 0) {
            int32_t *to = p.tables + (uint64_t)(uint32_t)children[i] * p.max_blocks;
            for (uint32_t j = threadIdx.x; j < full; j += kCopyT) {
                const int32_t page = from[j];
                to[j] = page;
                if ((uint32_t)page < p.pages) atomicAdd(p.refs + page, 1);
                else set_err(p.status, DM_ERR_INVALID_ARG);
            }
            if (threadIdx.x == 0) {
                if (tail) to[full] = p.w.aux[i];
                p.lengths[children[i]] = (int32_t)len;
            }
        } else if (tail) {
            const uint32_t old = (uint32_t)from[full], layer = (part - 1) / 2;
            if (old >= p.pages) {
                if (threadIdx.x == 0) set_err(p.status, DM_ERR_INVALID_ARG);
                continue;
            }
            char *pool = (part & 1 ? c.k : c.v) + layer * c.layer_bytes;
            const char *src = pool + old * c.page_bytes;
            char *dst = pool + (uint64_t)(uint32_t)p.w.aux[i] * c.page_bytes;
            if (c.tokens_first) {
                copy_run<kCopyT>(dst, src, tail * c.heads * c.row_bytes, threadIdx.x);
            } else {
                // a warp per head, a run of up to 16 KB each
                const uint32_t run = tail * c.row_bytes, head = p.B * c.row_bytes;
                for (uint32_t h = threadIdx.x / 32; h < c.heads; h += kCopyT / 32)
                    copy_run<32>(dst + (uint64_t)h * head, src + (uint64_t)h * head, run, threadIdx.x & 31);
            }
        }
    }
}

__global__ void __launch_bounds__(256) k_free(PagesArgs p, const int32_t *seqs, uint32_t n) {
    __shared__ int32_t s_len;
    pdl_enter();
    if (__syncthreads_or(has_err(p.status))) return;   // another CTA may be setting it
    uint32_t bad = 0;   // every CTA looks at every id: one out of range stops them all
    for (uint32_t i = threadIdx.x; i < n; i += 256) bad |= (uint32_t)seqs[i] >= p.max_seqs;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) set_err(p.status, DM_ERR_INVALID_ARG);
        return;
    }
    for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t s = (uint32_t)seqs[i];
        // a sequence named twice is empty the second time
        if (threadIdx.x == 0) s_len = atomicExch(p.lengths + s, 0);
        __syncthreads();
        const uint32_t nb = min(((uint32_t)s_len + p.B - 1) / p.B, p.max_blocks);
        for (uint32_t j = threadIdx.x; j < nb; j += 256) {
            const uint32_t page = (uint32_t)p.tables[(uint64_t)s * p.max_blocks + j];
            if (page < p.pages) atomicAdd(p.refs + page, -1);
            else set_err(p.status, DM_ERR_INVALID_ARG);
        }
        __syncthreads();
    }
}

// Which page moves where: list[0..) the free ids below `live`, list[pages..)
// the pages in use from `live` on, to[] the new id of each of the latter.
__global__ void __cluster_dims__(kCl, 1, 1) __launch_bounds__(kPt) k_compact_plan(PagesArgs p, uint32_t *moved) {
    __shared__ uint32_t s_warp[32], s_free, s_cnt;
    pdl_enter();
    cg::cluster_group cl = cg::this_cluster();
    const uint32_t rank = cl.block_rank(), tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    uint32_t begin, end;
    warp_run(p.pages, rank * kPw + wid, begin, end);
    // free pages below `limit` in this warp's run, scanned: before the warp
    // in the cluster, and over all
    auto count = [&](uint32_t limit, uint32_t &all) {
        uint32_t mine = 0;
        const uint32_t e = min(end, max(limit, begin));
        for (uint32_t i = begin + lane * 4; i < e; i += 128) mine += __popc(free4(p.refs, i, e));
        mine = __reduce_add_sync(~0u, mine);
        if (lane == 0) s_warp[wid] = mine;
        __syncthreads();
        if (wid == 0) {
            const uint32_t in = scan_incl(s_warp[lane]);
            s_warp[lane] = in - s_warp[lane];
            if (lane == 31) s_cnt = in;
        }
        cl.sync();
        uint32_t before = s_warp[wid];
        all = 0;
        for (uint32_t r = 0; r < kCl; ++r) {
            const uint32_t f = *cl.map_shared_rank(&s_cnt, r);
            if (r < rank) before += f;
            all += f;
        }
        cl.sync();
        return before;
    };
    if (tid == 0) s_free = has_err(p.status);
    cl.sync();
    const bool ok = *cl.map_shared_rank(&s_free, 0) == 0;
    uint32_t frees, holes;
    const uint32_t free_before = count(p.pages, frees);
    const uint32_t live = p.pages - frees;
    const uint32_t hole_before = count(live, holes);
    if (rank == 0 && tid == 0) {
        p.w.head[0] = ok;
        p.w.head[1] = ok ? (int32_t)holes : 0;
        p.w.head[2] = (int32_t)live;
        if (moved && ok) *moved = holes;
    }
    uint32_t h = hole_before;
    uint32_t u = begin > live ? (begin - live) - (free_before - holes) : 0;   // pages in use in [live, begin)
    for (uint32_t i0 = begin; ok && i0 < end; i0 += 128) {
        const uint32_t i = i0 + lane * 4;
        const uint32_t in_run = i >= end ? 0u : i + 4 <= end ? 15u : (1u << (end - i)) - 1;
        const uint32_t low = i >= live ? 0u : i + 4 <= live ? 15u : (1u << (live - i)) - 1;
        const uint32_t f = in_run ? free4(p.refs, i, end) : 0;
        uint32_t hole = f & low, use = in_run & ~f & ~low;
        const uint32_t hi = scan_incl(__popc(hole)), ui = scan_incl(__popc(use));
        uint32_t at = h + hi - __popc(hole);
        for (; hole; hole &= hole - 1) p.w.list[at++] = (int32_t)(i + __ffs(hole) - 1);
        at = u + ui - __popc(use);
        for (; use; use &= use - 1) p.w.list[p.pages + at++] = (int32_t)(i + __ffs(use) - 1);
        h += __shfl_sync(~0u, hi, 31);
        u += __shfl_sync(~0u, ui, 31);
    }
    cl.sync();
    if (ok)
        for (uint32_t k = rank * kPt + tid; k < holes; k += kCl * kPt)
            p.w.to[__ldcg(p.w.list + p.pages + k)] = __ldcg(p.w.list + k);
}

// Jobs: each moved page in each pool, then the table rows, then chunks of refs.
constexpr uint32_t kRefChunk = 4096;
__global__ void __launch_bounds__(kCopyT) k_compact_copy(PagesArgs p, CopyArgs c, int32_t *tables_out,
                                                         int32_t *refs_out) {
    pdl_enter();
    if (p.w.head[0] == 0) return;
    const uint32_t moves = (uint32_t)p.w.head[1], live = (uint32_t)p.w.head[2];
    const uint64_t copies = (uint64_t)moves * 2 * c.layers, rows = p.max_seqs;
    const uint64_t refs = (p.pages + kRefChunk - 1) / kRefChunk;
    for (uint64_t job = blockIdx.x; job < copies + rows + refs; job += gridDim.x) {
        if (job < copies) {
            const uint32_t pool = (uint32_t)(job / moves), k = (uint32_t)(job % moves);
            char *base = (pool & 1 ? c.v : c.k) + (pool >> 1) * c.layer_bytes;
            copy_run<kCopyT>(base + (uint64_t)(uint32_t)p.w.list[k] * c.page_bytes,
                             base + (uint64_t)(uint32_t)p.w.list[p.pages + k] * c.page_bytes, c.heads * p.B * c.row_bytes,
                             threadIdx.x);
        } else if (job < copies + rows) {
            const uint64_t s = job - copies;
            const uint32_t nb = min(((uint32_t)p.lengths[s] + p.B - 1) / p.B, p.max_blocks);
            for (uint32_t j = threadIdx.x; j < nb; j += kCopyT) {
                const uint64_t at = s * p.max_blocks + j;
                const int32_t page = p.tables[at];
                tables_out[at] = (uint32_t)page >= live && (uint32_t)page < p.pages ? p.w.to[page] : page;
            }
        } else {
            const uint32_t i0 = (uint32_t)(job - copies - rows) * kRefChunk;
            if (refs_out != p.refs)
                for (uint32_t i = i0 + threadIdx.x; i < min(p.pages, i0 + kRefChunk); i += kCopyT) {
                    if (i >= live) refs_out[i] = 0;
                    else if (p.refs[i] != 0) refs_out[i] = p.refs[i];
                }
            // the moved pages' counts, a chunk of the moves to each of these jobs
            for (uint32_t k = i0 + threadIdx.x; k < min(moves, i0 + kRefChunk); k += kCopyT) {
                const uint32_t from = (uint32_t)p.w.list[p.pages + k];
                refs_out[p.w.list[k]] = p.refs[from];
                refs_out[from] = 0;
            }
        }
    }
}

PagesArgs pages_args(const dm_cache *c) {
    return {c->tables, c->lengths, c->refs, c->status, cache_work(c), c->pages, c->page_tokens, c->max_seqs,
            c->max_blocks};
}

CopyArgs copy_args(const dm_cache *c) {
    return {static_cast<char *>(c->k), static_cast<char *>(c->v), c->layer_stride * 2, c->page_stride * 2, c->layers,
            c->kv_heads, c->head_dim * 2, c->layout == DM_PAGES_TOKENS};
}

// Many more CTAs than fit at once: late ones even the ends out (4,915 of
// 8,192 pages in use, eight layers of 64 KB a page compacted: 333 us with 8 an
// SM, 313 with 32, 6.6 TB/s).
uint32_t copy_grid(uint64_t jobs) { return (uint32_t)std::min<uint64_t>(jobs, (uint64_t)sm_count() * 32); }

}  // namespace
}  // namespace dm

extern "C" uint64_t dm_cache_work_bytes(const dm_cache *c) {
    return dm::cache_shape_ok(c) ? dm::cache_work_ints(c) * 4 : 0;
}

extern "C" dm_status dm_cache_last_error(const dm_cache *c, void *stream) {
    if (!c || !c->status) return DM_ERR_INVALID_ARG;
    const auto st = static_cast<cudaStream_t>(stream);
    uint32_t e = 0;
    if (cudaMemcpyAsync(&e, c->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return DM_ERR_CUDA;
    if (e && cudaMemsetAsync(c->status, 0, 4, st) != cudaSuccess) return DM_ERR_CUDA;
    return static_cast<dm_status>(e);
}

extern "C" dm_status dm_cache_extend(const dm_cache *c, const int32_t *seqs, const int32_t *add, uint32_t n,
                                     void *stream) {
    if (!dm::cache_ok(c) || n > c->max_seqs || (n && (!seqs || !add))) return DM_ERR_INVALID_ARG;
    if (n == 0) return DM_OK;
    return dm::status_of(dm::launch_pdl(dm::k_grow<false>, dm::kCl, dm::kPt, 0, static_cast<cudaStream_t>(stream),
                                        dm::pages_args(c), seqs, add, nullptr, n));
}

extern "C" dm_status dm_cache_fork(const dm_cache *c, const int32_t *parents, const int32_t *children,
                                   const int32_t *len, uint32_t n, void *stream) {
    if (!dm::cache_ok(c) || n > c->max_seqs || (n && (!parents || !children || !len))) return DM_ERR_INVALID_ARG;
    if (n == 0) return DM_OK;
    const auto st = static_cast<cudaStream_t>(stream);
    const dm::PagesArgs p = dm::pages_args(c);
    cudaError_t e = dm::launch_pdl(dm::k_grow<true>, dm::kCl, dm::kPt, 0, st, p, parents, len, children, n);
    if (e == cudaSuccess)
        e = dm::launch_pdl(dm::k_fork_copy, dm::copy_grid((uint64_t)n * (1 + 2 * c->layers)), dm::kCopyT, 0, st, p,
                           dm::copy_args(c), parents, children, len, n);
    return dm::status_of(e);
}

extern "C" dm_status dm_cache_free(const dm_cache *c, const int32_t *seqs, uint32_t n, void *stream) {
    if (!dm::cache_ok(c) || n > c->max_seqs || (n && !seqs)) return DM_ERR_INVALID_ARG;
    if (n == 0) return DM_OK;
    return dm::status_of(
        dm::launch_pdl(dm::k_free, dm::copy_grid(n), 256, 0, static_cast<cudaStream_t>(stream), dm::pages_args(c), seqs, n));
}

extern "C" dm_status dm_cache_compact(const dm_cache *c, int32_t *tables_out, int32_t *refs_out, uint32_t *moved,
                                      void *stream) {
    if (!dm::cache_ok(c) || !dm::aligned(refs_out, 16)) return DM_ERR_INVALID_ARG;
    const auto st = static_cast<cudaStream_t>(stream);
    const dm::PagesArgs p = dm::pages_args(c);
    cudaError_t e = dm::launch_pdl(dm::k_compact_plan, dm::kCl, dm::kPt, 0, st, p, moved);
    const uint64_t jobs = (uint64_t)c->pages * c->layers + c->max_seqs + (c->pages + dm::kRefChunk - 1) / dm::kRefChunk;
    if (e == cudaSuccess)
        e = dm::launch_pdl(dm::k_compact_copy, dm::copy_grid(jobs), dm::kCopyT, 0, st, p, dm::copy_args(c),
                           tables_out ? tables_out : c->tables, refs_out ? refs_out : c->refs);
    return dm::status_of(e);
}
