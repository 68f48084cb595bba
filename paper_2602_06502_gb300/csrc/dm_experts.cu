// dm_experts.cu -- what surrounds the products of an expert layer: rows in 8
// bits (dm_quantize), the choice of experts (dm_choose_experts), the sum of
// their parts, and the layer made of all (dm_experts).
#include <algorithm>
#include <cooperative_groups.h>

#include "dm_product.cuh"
#include "dm_quantize.cuh"

namespace cg = cooperative_groups;

namespace dm {
namespace {

// -- rows in 8 bits -------------------------------------------------------------------
//
// Bound: memory, 2 bytes read and 1 written per value (8,191 x 4,096, tensors in
// turn: f16 22 us, 4.6 TB/s, bf16 with a norm 29); the instructions, about ten a
// value, are close behind.  A row stays in
// the registers of a warp (up to 2,048 values) or of a CTA (up to 16,384); a
// longer one is read twice.

struct QuantizeArgs {
    const char *x;
    void *q;   // int8, or halves that hold the same whole numbers
    float *scale;
    const int32_t *count;
    uint64_t x_row, q_row;   // elements
    uint32_t rows, k;
    float eps;
    const int32_t *slots;    // halves: row r of x is written to rows slots[copies * r] .. of q (-1: none); NULL: to row r
    uint32_t copies;
};

template <class T, bool kHalves, bool kNorm, uint32_t kLanes, uint32_t kHeld>
__global__ void __launch_bounds__(kLanes == 32 ? 256 : kLanes, (kHeld <= 2 ? 6 : kHeld <= 4 ? 4 : 3) * (kLanes == 128 ? 2 : 1))
    k_quantize(QuantizeArgs p) {
    constexpr uint32_t kPer = kLanes == 32 ? 8 : 1;   // rows of a CTA; kHeld: vectors of 8 values a lane keeps
    __shared__ uint32_t s_top[8];
    __shared__ float s_sum[8];
    pdl_enter();
    const uint32_t lane = threadIdx.x % kLanes, rows = p.count ? (uint32_t)min(max(__ldcg(p.count), 0), (int32_t)p.rows) : p.rows;
    for (uint32_t r = blockIdx.x * kPer + threadIdx.x / kLanes; r < rows; r += gridDim.x * kPer) {
        const T *x = reinterpret_cast<const T *>(p.x) + r * p.x_row;
        uint32_t tops = 0;
        float sum = 0.f;
        // values from the row's end on are zeros
        auto load = [&](uint32_t at) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (at < p.k) v = *reinterpret_cast<const uint4 *>(x + at);
            return v;
        };
        auto cut = [&](uint4 &v, uint32_t at) {
            if (at < p.k && p.k - at < 8) {
                uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) w[i] &= (at + 2 * i < p.k ? 0xFFFFu : 0u) | (at + 2 * i + 1 < p.k ? 0xFFFF0000u : 0u);
            }
        };
        auto look = [&](const uint4 &v) {
            tops = larger2(larger2(larger2(larger2(tops, v.x), v.y), v.z), v.w);
            if constexpr (kNorm) {
                float f[8];
                unpack<T>(v, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += f[i] * f[i];
            }
        };
        uint4 held[kHeld];
#pragma unroll
        for (uint32_t i = 0; i < kHeld; ++i) held[i] = load((i * kLanes + lane) * 8);
#pragma unroll
        for (uint32_t i = 0; i < kHeld; ++i) {
            cut(held[i], (i * kLanes + lane) * 8);
            look(held[i]);
        }
        for (uint32_t at = (kHeld * kLanes + lane) * 8; at < p.k; at += kLanes * 8) {
            uint4 v = load(at);
            cut(v, at);
            look(v);
        }
        uint32_t bits = __reduce_max_sync(~0u, max(tops & 0xFFFFu, tops >> 16));
        if constexpr (kNorm)
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
        if constexpr (kLanes > 32) {
            __syncthreads();   // the row before has been read
            if (lane % 32 == 0) s_top[lane / 32] = bits, s_sum[lane / 32] = sum;
            __syncthreads();
            bits = 0;
            sum = 0.f;
#pragma unroll
            for (uint32_t i = 0; i < kLanes / 32; ++i) bits = max(bits, s_top[i]), sum += s_sum[i];
        }
        float scale;
        const RowStep step = row_step<T>(bits, scale);
        if constexpr (kNorm) {
            if (plain_squares<T>(bits)) {
                scale *= rsqrtf(sum / (float)p.k + p.eps);
            } else if (far_squares<T>(bits)) {   // the whole row goes here, and is read again: registers are for what is common
                const float shift = far_shift(bits);
                sum = 0.f;
#pragma unroll 1
                for (uint32_t at = lane * 8; at < p.k; at += kLanes * 8) {
                    uint4 v = load(at);
                    cut(v, at);
                    float f[8];
                    unpack<T>(v, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += f[i] * shift * (f[i] * shift);
                }
#pragma unroll
                for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
                if constexpr (kLanes > 32) {
                    __syncthreads();   // the sums before have been read
                    if (lane % 32 == 0) s_sum[lane / 32] = sum;
                    __syncthreads();
                    sum = 0.f;
#pragma unroll
                    for (uint32_t i = 0; i < kLanes / 32; ++i) sum += s_sum[i];
                }
                scale = far_scale(bits, sum / (float)p.k, p.eps);
            }
        }
        if (lane == 0) p.scale[r] = scale;
        auto put = [&](const uint4 &v, uint32_t at) {
            uint32_t n[8];
            steps8<T>(v, step, n);
            if constexpr (kHalves) {
                const uint4 y = halves8(n);
                __half *q = static_cast<__half *>(p.q) + at;   // rows of whole vectors
                if (p.slots == nullptr) *reinterpret_cast<uint4 *>(q + r * p.q_row) = y;
                else
                    for (uint32_t j = 0; j < p.copies; ++j) {
                        const int32_t slot = __ldcg(p.slots + r * p.copies + j);
                        if (slot >= 0) *reinterpret_cast<uint4 *>(q + (uint64_t)slot * p.q_row) = y;
                    }
            } else {
                int8_t *q = static_cast<int8_t *>(p.q) + r * p.q_row + at;
                const uint2 y = make_uint2(__byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410),
                                           __byte_perm(__byte_perm(n[4], n[5], 0x0040), __byte_perm(n[6], n[7], 0x0040), 0x5410));
                if (at + 8 <= p.k) {
                    *reinterpret_cast<uint2 *>(q) = y;
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i)
                        if (at + i < p.k) q[i] = (int8_t)n[i];
                }
            }
        };
#pragma unroll
        for (uint32_t i = 0; i < kHeld; ++i) {
            const uint32_t at = (i * kLanes + lane) * 8;
            if (at < p.k) put(held[i], at);
        }
        for (uint32_t at = (kHeld * kLanes + lane) * 8; at < p.k; at += kLanes * 8) {
            uint4 v = load(at);
            cut(v, at);
            put(v, at);
        }
    }
}

template <class T, bool kHalves, bool kNorm>
cudaError_t launch_quantize(const QuantizeArgs &p, cudaStream_t st) {
    // Few rows go a CTA each, many a warp each (61 x 1,024: 2.0 and 3.6 us).
    if (p.k <= 2048 && (p.k <= 512 || p.rows > 4 * (uint32_t)sm_count())) {
        const auto k = p.k <= 512 ? k_quantize<T, kHalves, kNorm, 32, 2> : p.k <= 1024 ? k_quantize<T, kHalves, kNorm, 32, 4> : k_quantize<T, kHalves, kNorm, 32, 8>;
        return launch_pdl(k, (p.rows + 7) / 8, 256, 0, st, p);
    }
    // What a row costs besides its values, each thread pays, so with many rows half
    // as many threads have one (8,191 x 4,096, one tensor over and over: 19.9 us, 22.8 with 256, 33 with a warp).
    if (p.k <= 4096 && p.rows > 4 * (uint32_t)sm_count()) return launch_pdl(k_quantize<T, kHalves, kNorm, 128, 4>, p.rows, 128, 0, st, p);
    const auto k = p.k <= 4096 ? k_quantize<T, kHalves, kNorm, 256, 2> : p.k <= 8192 ? k_quantize<T, kHalves, kNorm, 256, 4> : k_quantize<T, kHalves, kNorm, 256, 8>;
    return launch_pdl(k, p.rows, 256, 0, st, p);
}

template <class T>
cudaError_t launch_quantize(const QuantizeArgs &p, bool halves, cudaStream_t st) {
    if (p.eps >= 0.f) return halves ? launch_quantize<T, true, true>(p, st) : launch_quantize<T, false, true>(p, st);
    return halves ? launch_quantize<T, true, false>(p, st) : launch_quantize<T, false, false>(p, st);
}

// -- the choice of experts ---------------------------------------------------------------
//
// A warp per token: scores in the lanes' registers as whole numbers of the same
// order; the best that is left is a maximum over the warp, top_k times.  A CTA
// has a tile of up to 32 tokens and 256 pairs and counts each expert's; an
// expert's first slot in a tile is the sum of the counts of the experts before it
// and of its own in the tiles before, and within a tile a pair's place is the
// number of equal ones before it.  Up to kCluster tiles see each other's counts
// as a cluster, in one launch; more leave them in memory for a second kernel, each
// of whose CTAs adds up those before its own; beyond kFewTiles a kernel between
// the two does that once for all (128 experts, 8 each, with and without it: 2,048
// tokens 10.4 and 10.0 us, 4,096 11.4 and 12.0, 65,536 63 and 252).
//
// Bound: latency, then instructions.  Four tokens of 8 experts: 3.1 us; 8,192 of
// 128, 8 each: 12 us.

constexpr uint32_t kChooseT = 1024, kTilePairs = 256, kTileTokens = 32, kCluster = 8, kFewTiles = 96;

struct ChooseArgs {
    const char *logits;
    uint64_t row;   // elements
    uint32_t tokens, experts, top_k, renormalize, tile, tiles;   // tokens of a tile; how many tiles
    int32_t *ids, *offsets, *slots, *sources;
    float *weights;
    int32_t *counts;   // [tile][expert]; many tiles: those before, and behind the last tile all
};

uint32_t tile_tokens(uint32_t top_k) { return std::min(kTileTokens, kTilePairs / top_k); }

// Whole numbers in the order of the scores; 0: nothing to choose.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x == -INFINITY) return 0;
    if (x != x) x = -3.4028235e38f;
    if (x == 0.f) x = 0.f;   // -0 is 0
    const uint32_t b = __float_as_uint(x);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t o) { return o == 0 ? -INFINITY : __uint_as_float(o >> 31 ? o & 0x7FFFFFFFu : ~o); }

// The slots of a tile's pairs, an expert (or -1) a thread.  s_off: where each
// expert's pairs of this tile begin; s_seen: counts of each for kTilePairs / 32 warps.
__device__ __forceinline__ void place_pairs(const ChooseArgs &p, uint32_t first, uint32_t pairs, int32_t e, const int32_t *s_off, uint32_t *s_seen) {
    const uint32_t tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, E = p.experts;
    for (uint32_t i = tid; i < kTilePairs / 32 * E; i += kChooseT) s_seen[i] = 0;
    __syncthreads();
    uint32_t same = 0;
    if (tid < kTilePairs) {
        same = __match_any_sync(~0u, e);
        if (e >= 0 && lane == (uint32_t)__ffs(same) - 1) s_seen[wid * E + e] = __popc(same);
    }
    __syncthreads();
    if (tid < E) {
        uint32_t sum = (uint32_t)s_off[tid];
#pragma unroll
        for (uint32_t q = 0; q < kTilePairs / 32; ++q) {
            const uint32_t n = s_seen[q * E + tid];
            s_seen[q * E + tid] = sum;
            sum += n;
        }
    }
    __syncthreads();
    if (tid < pairs) {
        int32_t slot = -1;
        if (e >= 0) {
            slot = (int32_t)(s_seen[wid * E + e] + __popc(same & ((1u << lane) - 1)));
            p.sources[slot] = (int32_t)(first + tid);
        }
        p.slots[first + tid] = slot;
    }
}

// What the experts before this thread's have together; total: all of them.
__device__ int32_t scan_experts(int32_t x, int32_t *s_warp, int32_t &total) {
    const uint32_t wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int32_t in = x;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t y = __shfl_up_sync(~0u, in, d);
        if ((int)lane >= d) in += y;
    }
    if (lane == 31) s_warp[wid] = in;
    __syncthreads();
    if (wid == 0) {
        int32_t z = s_warp[lane];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int32_t y = __shfl_up_sync(~0u, z, d);
            if ((int)lane >= d) z += y;
        }
        s_warp[lane] = z;
    }
    __syncthreads();
    total = s_warp[31];
    return in - x + (wid ? s_warp[wid - 1] : 0);
}

// The offsets, and the sources behind the last slot: `mine` of thread e is
// expert e's count, `earlier` that in the tiles before.  Fills s_off.
__device__ __forceinline__ void place_experts(const ChooseArgs &p, int32_t mine, int32_t earlier, uint32_t tile, int32_t *s_off, int32_t *s_warp) {
    const uint32_t tid = threadIdx.x;
    int32_t total;
    const int32_t before = scan_experts(mine, s_warp, total);
    s_off[tid] = before + earlier;
    if (tile == 0) {
        if (tid < p.experts) p.offsets[tid] = before;
        if (tid == 0) p.offsets[p.experts] = total;
    }
    for (uint64_t i = (uint64_t)total + (uint64_t)tile * kChooseT + tid; i < p.tokens * p.top_k; i += (uint64_t)p.tiles * kChooseT) p.sources[i] = -1;
}

template <class T, uint32_t kV>
__global__ void __launch_bounds__(kChooseT) k_choose(ChooseArgs p) {
    extern __shared__ uint32_t s_seen[];
    __shared__ int32_t s_count[kChooseT], s_off[kChooseT], s_warp[32], s_ids[kTilePairs];
    pdl_enter();
    const uint32_t tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, tile = blockIdx.x;
    const uint32_t first = tile * p.tile, token = first + wid;
    s_count[tid] = 0;
    if (tid < kTilePairs) s_ids[tid] = -1;
    __syncthreads();
    if (wid < p.tile && token < p.tokens) {
        const T *row = reinterpret_cast<const T *>(p.logits) + token * p.row;
        uint32_t o[kV];
        bool nan = false;
#pragma unroll
        for (uint32_t v = 0; v < kV; ++v) {
            const uint32_t e = v * 32 + lane;
            const float x = e < p.experts ? score_at(row + e) : -INFINITY;
            nan |= x != x;
            o[v] = order_of(x);
        }
        nan = __any_sync(~0u, nan);
        uint32_t best = 0, at = ~0u;   // of this lane
        float all = 0.f, top = 0.f, score = -INFINITY;
        int32_t mine = -1;   // lane j keeps the j-th choice
        for (uint32_t j = 0; j < p.top_k; ++j) {
            best = 0;
#pragma unroll
            for (uint32_t v = 0; v < kV; ++v)
                if (o[v] > best) best = o[v], at = v * 32 + lane;
            const uint32_t got = __reduce_max_sync(~0u, best);
            if (j == 0) {
                top = score_of(got);
                if (!p.renormalize)
#pragma unroll
                    for (uint32_t v = 0; v < kV; ++v) all += o[v] ? expf(score_of(o[v]) - top) : 0.f;
            }
            if (got == 0) break;
            const uint32_t e = __reduce_min_sync(~0u, best == got ? at : ~0u);
#pragma unroll
            for (uint32_t v = 0; v < kV; ++v)
                if (v * 32 + lane == e) o[v] = 0;
            if (lane == j) {
                mine = (int32_t)e;
                score = score_of(got);
            }
        }
        float w = mine >= 0 ? expf(score - top) : 0.f, sum = p.renormalize ? w : all;
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
        if (mine >= 0) w = nan ? __int_as_float(0x7FC00000) : w / sum;
        if (lane < p.top_k) {
            p.ids[token * p.top_k + lane] = mine;
            p.weights[token * p.top_k + lane] = w;
            s_ids[wid * p.top_k + lane] = mine;
            if (mine >= 0) atomicAdd(s_count + mine, 1);   // whole numbers: in any order
        }
    }
    __syncthreads();
    if (p.tiles > kCluster) {
        if (tid < p.experts) p.counts[(uint64_t)tile * p.experts + tid] = s_count[tid];
        return;
    }
    cg::cluster_group cl = cg::this_cluster();
    int32_t count = s_count[tid], earlier = 0;
    if (p.tiles > 1) {
        cl.sync();
        count = 0;
        if (tid < p.experts)
            for (uint32_t r = 0; r < p.tiles; ++r) {
                const int32_t x = *cl.map_shared_rank(s_count + tid, r);
                count += x;
                if (r < tile) earlier += x;
            }
    }
    place_experts(p, count, earlier, tile, s_off, s_warp);
    const uint32_t tokens = first < p.tokens ? min(p.tile, p.tokens - first) : 0;
    place_pairs(p, first * p.top_k, tokens * p.top_k, tid < kTilePairs ? s_ids[tid] : -1, s_off, s_seen);
    if (p.tiles > 1) cl.sync();   // the counts have been read
}

// Counts become the sums of those in the tiles before, an expert a CTA.
__global__ void __launch_bounds__(kChooseT) k_choose_sums(ChooseArgs p) {
    __shared__ int32_t s_warp[32];
    pdl_enter();
    int32_t before = 0;
    for (uint64_t i0 = 0; i0 < p.tiles; i0 += kChooseT) {
        const uint64_t i = i0 + threadIdx.x;
        int32_t *c = p.counts + i * p.experts + blockIdx.x;
        int32_t total;
        const int32_t mine = scan_experts(i < p.tiles ? __ldcg(c) : 0, s_warp, total);
        if (i < p.tiles) *c = before + mine;
        before += total;
        __syncthreads();   // s_warp has been read
    }
    if (threadIdx.x == 0) p.counts[(uint64_t)p.tiles * p.experts + blockIdx.x] = before;
}

__global__ void __launch_bounds__(kChooseT) k_choose_place(ChooseArgs p) {
    extern __shared__ uint32_t s_seen[];
    __shared__ int32_t s_off[kChooseT], s_warp[32], s_mine[kChooseT], s_earlier[kChooseT];
    pdl_enter();
    const uint32_t tid = threadIdx.x, tile = blockIdx.x, first = tile * p.tile;
    const uint32_t pairs = min(p.tile, p.tokens - first) * p.top_k;
    const int32_t e = tid < pairs ? __ldcg(p.ids + first * p.top_k + tid) : -1;
    int32_t mine = 0, earlier = 0;
    if (p.tiles > kFewTiles) {
        if (tid < p.experts) {
            earlier = __ldcg(p.counts + (uint64_t)tile * p.experts + tid);
            mine = __ldcg(p.counts + (uint64_t)p.tiles * p.experts + tid);
        }
    } else {
        // tiles are shared out to groups of threads, one of them an expert's
        s_mine[tid] = s_earlier[tid] = 0;
        __syncthreads();
        const uint32_t groups = kChooseT / p.experts, x = tid % p.experts;
        if (tid / p.experts < groups) {
#pragma unroll 8
            for (uint32_t i = tid / p.experts; i < p.tiles; i += groups) {
                const int32_t n = __ldcg(p.counts + i * p.experts + x);
                mine += n;
                if (i < tile) earlier += n;
            }
            atomicAdd(s_mine + x, mine);   // whole numbers: in any order
            atomicAdd(s_earlier + x, earlier);
        }
        __syncthreads();
        mine = s_mine[tid], earlier = s_earlier[tid];
    }
    place_experts(p, mine, earlier, tile, s_off, s_warp);
    place_pairs(p, first * p.top_k, pairs, e, s_off, s_seen);
}

template <class T>
cudaError_t launch_choose(const ChooseArgs &p, cudaStream_t st) {
    const uint32_t per = (p.experts + 31) / 32, seen = kTilePairs / 32 * 4 * p.experts;
    const auto k = per <= 1 ? k_choose<T, 1> : per <= 2 ? k_choose<T, 2> : per <= 4 ? k_choose<T, 4> : per <= 8 ? k_choose<T, 8>
                 : per <= 16 ? k_choose<T, 16> : k_choose<T, 32>;
    DM_TRY(launch_pdl_cluster(k, p.tiles, p.tiles > kCluster ? 1 : p.tiles, kChooseT, seen, st, p));
    if (p.tiles > kFewTiles) DM_TRY(launch_pdl(k_choose_sums, p.experts, kChooseT, 0, st, p));
    return p.tiles > kCluster ? launch_pdl(k_choose_place, p.tiles, kChooseT, seen, st, p) : cudaSuccess;
}

uint64_t choose_bytes(uint32_t tokens, uint32_t experts, uint32_t top_k) {
    if (experts < 1 || experts > 1024 || top_k < 1 || top_k > std::min(experts, 32u) || (uint64_t)tokens * top_k > 0x7FFFFFFFull) return 0;
    const uint64_t tiles = ((uint64_t)tokens + tile_tokens(top_k) - 1) / tile_tokens(top_k);
    return tiles <= kCluster ? 1 : (tiles + 1) * experts * 4;
}

cudaError_t choose(const ChooseArgs &from, uint32_t dtype, cudaStream_t st) {
    ChooseArgs p = from;
    p.tile = tile_tokens(p.top_k);
    p.tiles = (uint32_t)(((uint64_t)p.tokens + p.tile - 1) / p.tile);
    if (p.tokens == 0) p.tiles = 1;   // the offsets
    return dtype == DM_BF16 ? launch_choose<__nv_bfloat16>(p, st) : dtype == DM_F16 ? launch_choose<__half>(p, st) : launch_choose<float>(p, st);
}

// -- the sum of the experts' parts ---------------------------------------------------------

struct JoinArgs {
    const float *parts;   // slot x pitch
    const int32_t *slots;
    const float *weights;
    const char *residual;
    char *y;
    uint32_t *status;
    uint64_t pitch, residual_row, y_row;   // elements
    uint32_t tokens, top_k, k;
    uint32_t words;   // rows of residual and y begin on 8 bytes
};

// 4 channels a thread, the parts in the order of the choice.  Bound: memory, 4
// bytes read for each value of a token's parts (4,096 tokens of 4 parts, 4,096
// wide: 56 us, 5.9 TB/s; with four parts on their way at a time 70).  Parts of 16
// bits take 25 of that layer's 538 us, and its error from 0.0020 to 0.0023.
template <class T>
__global__ void __launch_bounds__(256) k_join_experts(JoinArgs p) {
    pdl_enter();
    if (has_err(p.status)) return;
    const uint32_t each = (p.k + 3) / 4;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < (uint64_t)p.tokens * each; i += gridDim.x * 256ull) {
        const uint32_t token = (uint32_t)(i / each), at = (uint32_t)(i % each) * 4, n = min(p.k - at, 4u);
        float y[4] = {};
        const T *from = reinterpret_cast<const T *>(p.residual) + token * p.residual_row + at;
        if (p.residual && n == 4 && p.words) {
            const uint2 x = *reinterpret_cast<const uint2 *>(from);
            const float2 lo = Two<T>::up(*reinterpret_cast<const typename Two<T>::type *>(&x.x)), hi = Two<T>::up(*reinterpret_cast<const typename Two<T>::type *>(&x.y));
            y[0] = lo.x, y[1] = lo.y, y[2] = hi.x, y[3] = hi.y;
        } else if (p.residual) {
            for (uint32_t j = 0; j < n; ++j) y[j] = score_at(from + j);
        }
        for (uint32_t j = 0; j < p.top_k; ++j) {
            const int32_t slot = __ldcg(p.slots + token * p.top_k + j);
            if (slot < 0) continue;
            const float w = __ldcg(p.weights + token * p.top_k + j);
            const float4 x = __ldcg(reinterpret_cast<const float4 *>(p.parts + (uint64_t)slot * p.pitch + at));
            y[0] += w * x.x;
            y[1] += w * x.y;
            y[2] += w * x.z;
            y[3] += w * x.w;
        }
        T *to = reinterpret_cast<T *>(p.y) + token * p.y_row + at;
        if (n == 4 && p.words) {
            const auto a = Two<T>::down(y[0], y[1]), b = Two<T>::down(y[2], y[3]);
            *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
        } else {
            for (uint32_t j = 0; j < n; ++j) to[j] = Two<T>::down(y[j], 0.f).x;
        }
    }
}

// -- the layer ---------------------------------------------------------------------------------

// The layer's work buffer.
struct LayerWork {
    int32_t *ids, *offsets, *slots, *sources, *counts;
    float *weights, *x_scale, *h_scale, *parts;
    char *xq, *h, *hq, *product;
    uint64_t h_row, parts_row, xq_row, hq_row;   // elements
    uint64_t product_bytes;
    RowsAre x_are, h_are;
};

uint64_t layer_work(const dm_weights *up, const dm_weights *down, uint32_t tokens, uint32_t top_k, void *base, LayerWork &w) {
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        char *p = static_cast<char *>(base) + at;
        at += align_up(bytes, 256);
        return p;
    };
    const uint64_t slots = (uint64_t)tokens * top_k;
    const bool eight = up->dtype == DM_I8;
    w.x_are = rows_are(up, (uint32_t)slots, true), w.h_are = rows_are(down, (uint32_t)slots, false);
    w.h_row = align_up(down->k, 16), w.parts_row = align_up(down->n, 4), w.xq_row = align_up(up->k, 16), w.hq_row = w.h_row;
    w.offsets = (int32_t *)take(4ull * (up->experts + 1));
    w.ids = (int32_t *)take(4 * slots);
    w.weights = (float *)take(4 * slots);
    w.slots = (int32_t *)take(4 * slots);
    w.sources = (int32_t *)take(4 * slots);
    w.counts = (int32_t *)take(choose_bytes(tokens, up->experts, top_k));
    w.h = take(2 * slots * w.h_row);
    w.parts = (float *)take(4 * slots * w.parts_row);
    w.xq = take(!eight ? 0 : w.x_are == kHalves ? slots * w.xq_row * 2 : tokens * w.xq_row);
    w.x_scale = (float *)take(eight ? 4ull * tokens : 0);
    w.hq = take(eight ? slots * w.hq_row * (w.h_are == kHalves ? 2 : 1) : 0);
    w.h_scale = (float *)take(eight ? 4 * slots : 0);
    w.product_bytes = std::max(product_bytes(up, (uint32_t)slots, 1, w.x_are), product_bytes(down, (uint32_t)slots, 0, w.h_are));
    w.product = take(w.product_bytes);
    return at;
}

bool layer_ok(const dm_weights *up, const dm_weights *down, uint32_t tokens, uint32_t top_k) {
    if (!weights_ok(up) || !weights_ok(down) || up->dtype != down->dtype || up->experts != down->experts) return false;
    return up->n % 2 == 0 && down->k == up->n / 2 && down->n == up->k && choose_bytes(tokens, up->experts, top_k) != 0;
}

cudaError_t quantize(uint32_t dtype, const QuantizeArgs &p, bool halves, cudaStream_t st) {
    return dtype == DM_BF16 ? launch_quantize<__nv_bfloat16>(p, halves, st) : launch_quantize<__half>(p, halves, st);
}

// A projection's work buffer.
struct LinearWork {
    char *q, *product;
    float *scale;
    uint64_t q_row;   // elements
    uint64_t product_bytes;
    RowsAre are;
};

uint64_t linear_work(const dm_weights *w, uint32_t rows, void *base, LinearWork &x) {
    if (takes_raw(w, rows)) return 1;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        char *p = static_cast<char *>(base) + at;
        at += align_up(bytes, 256);
        return p;
    };
    x.q_row = align_up(w->k, 16);
    x.are = rows_are(w, rows, false);
    x.q = take(rows * x.q_row * (x.are == kHalves ? 2 : 1));
    x.scale = (float *)take(4ull * rows);
    x.product_bytes = product_bytes(w, rows, 0, x.are);
    x.product = take(x.product_bytes);
    return at;
}

bool linear_ok(const dm_weights *w, uint32_t rows) { return weights_ok(w) && w->dtype == DM_I8 && w->experts == 1 && rows <= 0x7FFFFFFFu; }

}  // namespace
}  // namespace dm

extern "C" dm_status dm_products_last_error(uint32_t *status, void *stream) {
    if (!dm::status_ok(status)) return DM_ERR_INVALID_ARG;
    const auto st = static_cast<cudaStream_t>(stream);
    uint32_t e = 0;
    if (cudaMemcpyAsync(&e, status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return DM_ERR_CUDA;
    if (e && cudaMemsetAsync(status, 0, 4, st) != cudaSuccess) return DM_ERR_CUDA;
    return static_cast<dm_status>(e);
}

extern "C" dm_status dm_quantize(const dm_quantize_args *a, void *stream) {
    using namespace dm;
    if (!a || a->dtype > DM_F16 || a->k < 1 || a->k > (1u << 24) || a->rows > 0x7FFFFFFFu || !(a->eps <= 3.4e38f)) return DM_ERR_INVALID_ARG;
    if (a->rows == 0) return DM_OK;
    if (!a->x || !a->q || !a->scale || !aligned(a->x, 16) || !aligned(a->q, 16) || !aligned(a->scale, 4) || !aligned(a->count, 4))
        return DM_ERR_INVALID_ARG;
    if (a->x_row % 8 || a->q_row % 16 || a->x_row > (1ull << 32) || a->q_row > (1ull << 32)) return DM_ERR_INVALID_ARG;
    if (a->rows > 1 && (a->x_row < a->k || a->q_row < a->k)) return DM_ERR_INVALID_ARG;
    return status_of(quantize(a->dtype, {static_cast<const char *>(a->x), a->q, a->scale, a->count, a->x_row, a->q_row, a->rows, a->k, a->eps},
                              false, static_cast<cudaStream_t>(stream)));
}

extern "C" uint64_t dm_linear_bytes(const dm_weights *w, uint32_t rows) {
    using namespace dm;
    LinearWork x;
    return linear_ok(w, rows) ? linear_work(w, rows, nullptr, x) : 0;
}

extern "C" dm_status dm_linear(const dm_weights *w, const dm_linear_args *a, void *stream) {
    using namespace dm;
    if (!a || !linear_ok(w, a->rows) || !status_ok(a->status) || a->dtype > DM_F16 || a->y_dtype > DM_F32 || a->y_dtype == DM_I8 || !(a->eps <= 3.4e38f))
        return DM_ERR_INVALID_ARG;
    LinearWork x;
    const uint64_t need = linear_work(w, a->rows, a->work, x);
    if (need > 1 && (!a->work || !aligned(a->work, 256) || a->work_bytes < need)) return DM_ERR_INVALID_ARG;
    if (a->rows == 0) return DM_OK;
    if (!a->x || !a->y || !aligned(a->x, 16) || !aligned(a->y, dtype_size(a->y_dtype))) return DM_ERR_INVALID_ARG;
    if (a->x_row % 8 || a->x_row > (1ull << 32) || a->y_row > (1ull << 32)) return DM_ERR_INVALID_ARG;
    if (a->rows > 1 && (a->x_row < w->k || a->y_row < w->n)) return DM_ERR_INVALID_ARG;
    const auto st = static_cast<cudaStream_t>(stream);
    const auto linear = [&]() -> cudaError_t {
        dm_product_args d{};
        d.x_rows = d.rows = a->rows;
        d.y = a->y, d.y_row = a->y_row, d.y_dtype = a->y_dtype, d.status = a->status;
        ProductArgs p = product_args(w, &d);
        if (need == 1) {
            p.x = static_cast<const char *>(a->x), p.x_row = a->x_row * 2, p.eps = a->eps;
            return launch_product_raw(p, a->dtype, st);
        }
        p.x = x.q, p.x_scale = x.scale;
        p.x_halves = x.are == kHalves;
        p.x_row = x.q_row * (p.x_halves ? 2 : 1);
        DM_TRY(quantize(a->dtype, {static_cast<const char *>(a->x), x.q, x.scale, nullptr, a->x_row, x.q_row, a->rows, w->k, a->eps}, p.x_halves, st));
        return launch_product(w, p, x.product, x.product_bytes, st);
    };
    return status_of(linear());
}

extern "C" uint64_t dm_choose_bytes(uint32_t tokens, uint32_t experts, uint32_t top_k) { return dm::choose_bytes(tokens, experts, top_k); }

extern "C" dm_status dm_choose_experts(const dm_choose_args *a, void *stream) {
    using namespace dm;
    if (!a || a->reserved0 || a->dtype > DM_F32 || a->dtype == DM_I8 || a->renormalize > 1) return DM_ERR_INVALID_ARG;
    const uint64_t need = choose_bytes(a->tokens, a->experts, a->top_k);
    if (!need || (need > 1 && (a->work_bytes < need || !a->work || !aligned(a->work, 16))) || !a->offsets || !aligned(a->offsets, 4)) return DM_ERR_INVALID_ARG;
    if (a->logits_row > (1ull << 32) || (a->tokens > 1 && a->logits_row < a->experts)) return DM_ERR_INVALID_ARG;
    if (a->tokens && (!a->logits || !a->ids || !a->weights || !a->slots || !a->sources || !aligned(a->logits, dtype_size(a->dtype)) ||
                      !aligned(a->ids, 4) || !aligned(a->weights, 4) || !aligned(a->slots, 4) || !aligned(a->sources, 4)))
        return DM_ERR_INVALID_ARG;
    ChooseArgs p{};
    p.logits = static_cast<const char *>(a->logits), p.row = a->logits_row;
    p.tokens = a->tokens, p.experts = a->experts, p.top_k = a->top_k, p.renormalize = a->renormalize;
    p.ids = a->ids, p.weights = a->weights, p.offsets = a->offsets, p.slots = a->slots, p.sources = a->sources;
    p.counts = static_cast<int32_t *>(a->work);
    return status_of(choose(p, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" uint64_t dm_experts_bytes(const dm_weights *up, const dm_weights *down, uint32_t tokens, uint32_t top_k) {
    using namespace dm;
    LayerWork w;
    return layer_ok(up, down, tokens, top_k) ? layer_work(up, down, tokens, top_k, nullptr, w) : 0;
}

extern "C" dm_status dm_experts(const dm_weights *up, const dm_weights *down, const dm_experts_args *a, void *stream) {
    using namespace dm;
    if (!a || a->reserved0 || a->renormalize > 1 || a->dtype > DM_F16 || a->logits_dtype > DM_F32 || a->logits_dtype == DM_I8)
        return DM_ERR_INVALID_ARG;
    if (!layer_ok(up, down, a->tokens, a->top_k) || !status_ok(a->status)) return DM_ERR_INVALID_ARG;
    const bool eight = up->dtype == DM_I8;
    if (!eight && up->dtype != a->dtype) return DM_ERR_INVALID_ARG;
    LayerWork w;
    if (!a->work || !aligned(a->work, 256) || a->work_bytes < layer_work(up, down, a->tokens, a->top_k, a->work, w)) return DM_ERR_INVALID_ARG;
    if (a->tokens == 0) return DM_OK;
    if (!a->x || !a->logits || !a->y || !aligned(a->x, 16) || !aligned(a->y, 2) || !aligned(a->residual, 2) ||
        !aligned(a->logits, dtype_size(a->logits_dtype)))
        return DM_ERR_INVALID_ARG;
    if (a->x_row % 8 || a->logits_row > (1ull << 32) || a->x_row > (1ull << 32) ||
        a->y_row > (1ull << 32) || a->residual_row > (1ull << 32))
        return DM_ERR_INVALID_ARG;
    if (a->tokens > 1 && (a->x_row < up->k || a->y_row < up->k || a->logits_row < up->experts || (a->residual && a->residual_row < up->k)))
        return DM_ERR_INVALID_ARG;
    const auto st = static_cast<cudaStream_t>(stream);
    const uint32_t slots = a->tokens * a->top_k;
    ChooseArgs c{};
    c.logits = static_cast<const char *>(a->logits), c.row = a->logits_row;
    c.tokens = a->tokens, c.experts = up->experts, c.top_k = a->top_k, c.renormalize = a->renormalize;
    c.ids = w.ids, c.weights = w.weights, c.offsets = w.offsets, c.slots = w.slots, c.sources = w.sources, c.counts = w.counts;
    const auto layer = [&]() -> cudaError_t {
        DM_TRY(choose(c, a->logits_dtype, st));
        dm_product_args u{};
        // h is rounded to x's type: the tensor cores take 16-bit rows with 16-bit
        // weights, and its rest as a second row would double the next product.  Against
        // 64 bits a bf16 layer's error is 0.0020 so (4,096 tokens, 4 of 32 experts, 4,096 x
        // 1,536), 0.0017 with h in 32 bits, which is y's own rounding.  With 8-bit weights
        // the steps that follow are at least as coarse as this rounding.
        u.x = a->x, u.x_row = a->x_row, u.x_rows = a->tokens, u.sources = w.sources, u.per_source = a->top_k, u.offsets = w.offsets;
        u.y = w.h, u.y_row = w.h_row, u.y_dtype = a->dtype, u.rows = slots, u.gated = 1, u.status = a->status;
        ProductArgs up_args = product_args(up, &u);
        if (eight) {
            // halves go straight to the slots of their experts
            const bool halves = w.x_are == kHalves;
            up_args.x = w.xq, up_args.x_scale = w.x_scale, up_args.x_halves = halves, up_args.x_row = w.xq_row * (halves ? 2 : 1);
            DM_TRY(quantize(a->dtype, {static_cast<const char *>(a->x), w.xq, w.x_scale, nullptr, a->x_row, w.xq_row, a->tokens, up->k, -1.f,
                                       halves ? w.slots : nullptr, a->top_k}, halves, st));
        }
        DM_TRY(launch_product(up, up_args, w.product, w.product_bytes, st));
        dm_product_args d{};
        d.x = w.h, d.x_row = w.h_row, d.x_rows = slots, d.offsets = w.offsets;
        d.y = w.parts, d.y_row = w.parts_row, d.y_dtype = DM_F32, d.rows = slots, d.status = a->status;
        ProductArgs dp = product_args(down, &d);
        if (eight) {
            // straight to the halves that the tensor cores take, where they do
            dp.x = w.hq, dp.x_scale = w.h_scale, dp.x_halves = w.h_are == kHalves;
            dp.x_row = w.hq_row * (dp.x_halves ? 2 : 1);
            DM_TRY(quantize(a->dtype, {w.h, w.hq, w.h_scale, w.offsets + up->experts, w.h_row, w.hq_row, slots, down->k, -1.f}, dp.x_halves, st));
        }
        DM_TRY(launch_product(down, dp, w.product, w.product_bytes, st));
        JoinArgs j{w.parts, w.slots, w.weights, static_cast<const char *>(a->residual), static_cast<char *>(a->y), a->status,
                   w.parts_row, a->residual_row, a->y_row, a->tokens, a->top_k, up->k,
                   aligned(a->residual, 8) && aligned(a->y, 8) && (a->residual_row | a->y_row) % 4 == 0};
        const uint64_t each = (uint64_t)a->tokens * ((up->k + 3) / 4);
        const uint32_t grid = (uint32_t)std::min<uint64_t>((each + 255) / 256, (uint64_t)sm_count() * 8);
        return a->dtype == DM_BF16 ? launch_pdl(k_join_experts<__nv_bfloat16>, grid, 256, 0, st, j) : launch_pdl(k_join_experts<__half>, grid, 256, 0, st, j);
    };
    return status_of(layer());
}
