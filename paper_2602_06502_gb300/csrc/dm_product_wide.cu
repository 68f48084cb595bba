// dm_product_wide.cu -- products of many rows on the tensor cores.
//
// The weights are the tensor cores' first operand, 256 channels at a time (or
// 128 and their 128 partners), and rows the second, up to kRows of one expert,
// so that an expert with few rows costs few: a tile's width is any multiple of
// 16.  Two CTAs share a tile (tcgen05 over a pair): each holds 128 channels,
// half of the rows, and the sums of its channels in tensor memory, twice, so
// that one tile is stored while the next is summed.  Pairs walk the tiles of
// all experts in one line; offsets are read on the device.
//
//   warps 0-3   sums to y, a channel per lane
//   warps 4, 6  copies of weights and of rows by tensor map, into a ring of stages
//   warp 5      tcgen05.mma, in the first CTA of the pair
//   warps 8-23  8-bit weights alone: to halves, in tensor memory, from where
//               the tensor cores take them: no second pass through shared memory
//
// A pair because each CTA then reads half of the rows from shared memory for
// the same products; 256 x 256 because what a stage brings (64 KB for 512 cycles
// of products) is what L2 gives.
//
// Bound: the tensor cores and the power they may draw where there are many rows
// (one expert, 8,191 x 6,144 x 4,096, bf16: 240 us, 1.72 PFLOP/s, with sets of rows and
// weights in turn, in 8 bits 265; with one set over and over 224, 0.97 of the
// library's rate, and 241; 16,384 rows of 32 experts, 2 x 1,536 x 4,096, gated, bf16: 250
// us, 1.65 PFLOP/s); memory where there are few
// (64 experts of 2,048 x 2,048 with 16 rows each: 91 us, 5.9 TB/s). In 8 bits a
// product whose first operand is in tensor memory takes about 125 cycles, however
// few its rows, so there memory gives 3.5 TB/s (77 us).
#include <algorithm>
#include <atomic>

#include "dm_product.cuh"
#include "dm_tensor.cuh"

namespace dm {
namespace {

template <bool kEight>
struct Wide {
    static constexpr uint32_t kThreads = kEight ? 768 : 224;
    static constexpr uint32_t kRows = kEight ? 192 : 256;             // of a tile
    static constexpr uint32_t kStep = kEight ? 128 : 64;              // elements of k in a stage
    static constexpr uint32_t kStages = kEight ? 5 : 6;
    static constexpr uint32_t kW = 128 * 128;                         // bytes of a stage's weights
    static constexpr uint32_t kHalf = kRows / 2 * 128;                // bytes of 64 elements of this CTA's rows
    static constexpr uint32_t kX = kW, kStage = kW + kHalf * (kStep / 64);
    static constexpr uint32_t kA = 2 * kRows, kAs = (512 - kA) / 32;  // 8-bit: columns of the weights in tensor memory, in places of 64 elements of k
    static constexpr uint32_t kSwap = kStages * kStage;               // gated: 32 rows of 64 channels, floats
    static constexpr uint32_t kFirst = kSwap + 32 * 64 * 4;           // tiles before each expert
    static constexpr uint32_t kBars = kFirst + 1032 * 4;
    // per stage: full (the pair's), empty, weights full, weights empty; per
    // buffer of sums: full, empty (the pair's); per place of weights: full (the
    // pair's), empty
    static constexpr uint32_t kWord = kBars + 32 * kStages + 32 + 16 * kAs + 16;   // after the last, `done`
    static constexpr uint32_t kBytes = kWord + 16 + 1024;
};

constexpr uint32_t kSmallBox = 16;   // rows

struct WideArgs {
    ProductArgs p;
    float *part;          // splits > 1: [split][row][channel], sums of a part of k
    uint64_t part_split;  // elements
    uint32_t channels;    // of the weights
    uint32_t blocks;      // tiles across the channels
    uint32_t splits, steps;
    uint32_t even_rows;   // that are as many bytes as an expert's weights
#ifdef DM_DEBUG
    uint64_t test_wait_ns;   // dm_test_product_wait: 0, or how long waits last
#endif
};

// Whether a test has stage c of this CTA's weights never arrive.
__device__ __forceinline__ bool withheld(const WideArgs &a, uint32_t c) {
#ifdef DM_DEBUG
    return a.test_wait_ns && blockIdx.x == 0 && c == 0;
#else
    return false;
#endif
}

// -- pairs of CTAs -----------------------------------------------------------------

__device__ __forceinline__ uint32_t of_first(uint32_t addr) {   // the same place in the pair's first CTA
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
// What is handed over is tensor memory, which tcgen05's own fences order, so
// neither this nor the waits order other memory between the CTAs (at cluster
// scope each costs some hundred cycles).
__device__ __forceinline__ void arrive_pair(uint32_t bar) {   // bar: of_first()
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t peer_word(uint32_t addr, uint32_t rank) {
    uint32_t x;
    asm volatile(
        "{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.u32 %0, [a];\n\t}"
        : "=r"(x)
        : "r"(addr), "r"(rank)
        : "memory");
    return x;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Into this CTA's shared memory; the bytes are counted at `bar`, the pair's.
__device__ __forceinline__ void load3(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void load2(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void mma2_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void mma2_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(desc), "r"(add)
        : "memory");
}
// Arrives at `bar` of both CTAs once all that was issued before is done.
__device__ __forceinline__ void commit2(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}

// Whether the phase is over; does not wait.
__device__ __forceinline__ bool over(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Waits for the phase, by a whole warp; false: it is not over, and a wait of this
// CTA has given up, which ends the others at once.  Who copies, converts or
// multiplies then stops where it is: a barrier whose copies have not come takes
// no further arrival.  Who stores goes on to the end of its tiles, as its four
// warps meet on the way.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up, const WideArgs &a) {
    bool over = mbar_try(bar, parity);
    if (!over) {
        uint64_t ns = kWaitNs;
#ifdef DM_DEBUG
        if (a.test_wait_ns) ns = a.test_wait_ns;
#endif
        const uint64_t t0 = now_ns();
        for (uint32_t i = 0;; ++i) {
            if ((over = mbar_try(bar, parity)) || *gave_up) break;
            if ((i & 63) == 63 && (now_ns() - t0 > ns || i > kWaits)) {
                *gave_up = 1;
                set_err(a.p.status, DM_ERR_TIMEOUT);
                break;
            }
        }
    }
    return __all_sync(~0u, over);
}

// -- tiles --------------------------------------------------------------------------

struct Tile {
    uint32_t e, row, rows, width;   // the first row; rows of it; width: rows rounded up to 16
    uint32_t c0, split;
};

template <uint32_t kRows>
__device__ __forceinline__ uint32_t row_blocks(uint32_t rows) { return (rows + kRows - 1) / kRows; }

// An expert's rows in blocks of about the same size, multiples of 16.
template <uint32_t kRows>
__device__ __forceinline__ uint32_t block_rows(uint32_t rows) {
    const uint32_t n = row_blocks<kRows>(rows);
    return ((rows + n - 1) / n + 15) / 16 * 16;
}

struct Line {   // of tiles
    const uint32_t *first;
    uint32_t tiles, pair, pairs;
};

// Tile i.  An expert's tiles go through its rows first, which share weights, or
// where its rows are more bytes than its weights through the channels first: what
// is shared is read from memory once, and the other finds room in L2 (16,384 rows,
// 4,096 x 4,096, bf16: 279 us, 338 through the rows; 271 and 300 us for the library's
// product in the same runs).
template <uint32_t kRows>
__device__ __forceinline__ Tile tile_at(const WideArgs &a, const Line &l, uint32_t i) {
    uint32_t lo = 0, hi = a.p.experts;   // the last expert that begins by then
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (l.first[mid] <= i) lo = mid;
        else hi = mid;
    }
    Tile t;
    t.e = lo;
    const int32_t from = a.p.offsets ? __ldcg(a.p.offsets + t.e) : 0, to = a.p.offsets ? __ldcg(a.p.offsets + t.e + 1) : (int32_t)a.p.rows;
    const uint32_t rows = (uint32_t)(to - from), n = row_blocks<kRows>(rows), each = block_rows<kRows>(rows);
    uint32_t x = i - l.first[lo];
    t.split = x % a.splits;
    x /= a.splits;
    const bool rows_first = rows <= a.even_rows;
    const uint32_t block = rows_first ? x % n : x / a.blocks, across = rows_first ? x / n : x % a.blocks;
    t.row = (uint32_t)from + block * each;
    t.rows = min(each, rows - block * each);
    t.width = (t.rows + 15) / 16 * 16;
    t.c0 = across * (a.p.gated ? 128 : 256);
    return t;
}

// A pair's tiles, in turn with the other pairs, and their steps of k.
template <uint32_t kRows>
struct Walk {
    uint32_t turn, k0, steps;   // turns so far; of the present tile
    Tile t;

    __device__ __forceinline__ Walk() : turn(0) {}
    __device__ __forceinline__ bool next(const WideArgs &a, const Line &l) {
        const uint32_t i = turn++ * l.pairs + l.pair;
        if (i >= l.tiles) return false;
        t = tile_at<kRows>(a, l, i);
        k0 = (uint32_t)((uint64_t)t.split * a.steps / a.splits);
        steps = (uint32_t)((uint64_t)(t.split + 1) * a.steps / a.splits) - k0;
        return true;
    }
};

template <class Y>
__device__ __forceinline__ Y to_y(float x) {
    if constexpr (sizeof(Y) == 4) return x;
    else if constexpr (std::is_same_v<Y, __half>) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}

// A warp's channel per lane of `n` rows from row r on: 64 consecutive bytes a store, or 128.
template <class Y>
__device__ __forceinline__ void store_rows(const ProductArgs &p, const uint32_t *raw, uint32_t r, uint32_t n, uint32_t c, bool on) {
    Y *to = static_cast<Y *>(p.y) + (uint64_t)r * p.y_row + c;
    if (!on) return;
#pragma unroll
    for (uint32_t i = 0; i < 32; ++i)
        if (i < n) to[(uint64_t)i * p.y_row] = to_y<Y>(__uint_as_float(raw[i]));
}
__device__ __forceinline__ void store_rows(const ProductArgs &p, const uint32_t *raw, uint32_t r, uint32_t n, uint32_t c, bool on) {
    if (p.y_dtype == DM_BF16) store_rows<__nv_bfloat16>(p, raw, r, n, c, on);
    else if (p.y_dtype == DM_F16) store_rows<__half>(p, raw, r, n, c, on);
    else store_rows<float>(p, raw, r, n, c, on);
}

template <class T, bool kEight>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Wide<kEight>::kThreads, 1)
    k_product_wide(const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap ms, WideArgs a) {
    using W = Wide<kEight>;
    extern __shared__ char s_raw[];
    char *s = reinterpret_cast<char *>(align_up(reinterpret_cast<uint64_t>(s_raw), 1024));
    const ProductArgs &p = a.p;
    const uint32_t s_at = smem_addr(s), bars = s_at + W::kBars, more = bars + 32 * W::kStages;
    uint32_t *first = reinterpret_cast<uint32_t *>(s + W::kFirst);
    volatile uint32_t *gave_up = reinterpret_cast<uint32_t *>(s + W::kWord);
    const uint32_t tid = threadIdx.x, wid = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31, rank = blockIdx.x & 1;
    auto full = [&](uint32_t i) { return bars + 32 * i; };
    auto empty = [&](uint32_t i) { return bars + 32 * i + 8; };
    auto w_full = [&](uint32_t i) { return bars + 32 * i + 16; };
    auto w_empty = [&](uint32_t i) { return bars + 32 * i + 24; };
    auto sum_full = [&](uint32_t i) { return more + 16 * i; };
    auto sum_empty = [&](uint32_t i) { return more + 16 * i + 8; };
    auto a_full = [&](uint32_t i) { return more + 32 + 16 * i; };
    auto a_empty = [&](uint32_t i) { return more + 32 + 16 * i + 8; };
    const uint32_t done = more + 32 + 16 * W::kAs;
    if (tid == 0) {
        for (uint32_t i = 0; i < W::kStages; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
            mbar_init(w_full(i), 1);
            mbar_init(w_empty(i), 8);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(sum_full(i), 1);
            mbar_init(sum_empty(i), 8);   // four warps of two CTAs
        }
        for (uint32_t i = 0; i < W::kAs; ++i) {
            mbar_init(a_full(i), 8);
            mbar_init(a_empty(i), 1);
        }
        mbar_init(done, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (tid == 32) {
        for (const CUtensorMap *m : {&mw, &mx, &ms}) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }
    pdl_enter();
    if (wid == 5) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s_at + W::kWord + 4) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    // the tiles before each expert; with an earlier error there are none
    const bool stop = __syncthreads_or(has_err(p.status));
    for (uint32_t e = tid; e < p.experts; e += W::kThreads) {
        const Rows r = stop ? Rows{0, 0} : expert_rows(p, e);
        const uint32_t rows = (uint32_t)(r.b - r.a);
        first[e + 1] = p.most && rows <= p.most ? 0 : row_blocks<W::kRows>(rows) * a.blocks * a.splits;
    }
    if (tid == 0) first[0] = 0;
    if (p.experts > 1) {
        __syncthreads();
        if (wid == 0) {
            uint32_t carry = 0;
            for (uint32_t e0 = 0; e0 < p.experts; e0 += 32) {
                uint32_t x = e0 + lane < p.experts ? first[e0 + lane + 1] : 0;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const uint32_t y = __shfl_up_sync(~0u, x, d);
                    if ((int)lane >= d) x += y;
                }
                if (e0 + lane < p.experts) first[e0 + lane + 1] = carry + x;
                carry += __shfl_sync(~0u, x, 31);
            }
        }
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    // Should an error have come between what the two CTAs of a pair have seen,
    // neither has a tile.
    uint32_t tiles = first[p.experts];
    if (peer_word(smem_addr(first + p.experts), rank ^ 1) != tiles) tiles = 0;
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(s + W::kWord + 4);
    const Line line{first, tiles, blockIdx.x / 2, gridDim.x / 2};
    Walk<W::kRows> walk;
    const Tile &t = walk.t;
    if (wid == 4 || wid == 6) {
        // One warp copies weights, one rows: a copy takes its warp about 100
        // cycles to issue.  An elected thread issues what is the same in every
        // lane, as it goes through uniform registers.
        const bool weights = wid == 4, one = elect();
        uint32_t c = 0;   // stages so far
        bool on = true;
        while (on && walk.next(a, line)) {
            const uint32_t half = t.width / 2, boxes = half > W::kRows / 4 ? 0 : (half + kSmallBox - 1) / kSmallBox;
            const int row = (int)(t.row + rank * half), e = (int)t.e;
            const int w0 = (int)(p.gated ? t.c0 + rank * 64 : t.c0 + rank * 128), w1 = (int)(p.gated ? p.n + t.c0 + rank * 64 : t.c0 + rank * 128 + 64);
            const uint32_t x_bytes = (boxes ? boxes * kSmallBox * 128 : W::kHalf) * (W::kStep / 64);
            const uint32_t steps = walk.steps;
            for (uint32_t j = 0; j < steps; ++j, ++c) {
                const uint32_t st = c % W::kStages, round = c / W::kStages, at = s_at + st * W::kStage, bar = of_first(full(st));
                const int k0 = (int)((walk.k0 + j) * W::kStep);
                if (round && !(on = wait(!kEight || !weights ? empty(st) : w_empty(st), (round - 1) & 1, gave_up, a))) break;
                if (weights && withheld(a, c)) continue;
                if (weights) {
                    const uint32_t w_bar = kEight ? w_full(st) : bar;
                    if (one) {
                        if (kEight || rank == 0) mbar_expect(kEight ? w_full(st) : full(st), kEight ? W::kW : 2 * (x_bytes + W::kW));
                        load3(at, &mw, w_bar, k0, w0, e);
                        load3(at + W::kW / 2, &mw, w_bar, k0, w1, e);
                    }
                } else if (boxes == 0) {
                    if (one) {
                        if (kEight && rank == 0) mbar_expect(full(st), 2 * x_bytes);
#pragma unroll
                        for (uint32_t sub = 0; sub < W::kStep / 64; ++sub) load2(at + W::kX + sub * W::kHalf, &mx, bar, k0 + 64 * sub, row);
                    }
                } else if (one) {
                    if (kEight && rank == 0) mbar_expect(full(st), 2 * x_bytes);
#pragma unroll
                    for (uint32_t sub = 0; sub < W::kStep / 64; ++sub)
                        for (uint32_t b = 0; b < boxes; ++b)
                            load2(at + W::kX + sub * W::kHalf + b * kSmallBox * 128, &ms, bar, k0 + 64 * sub, row + b * kSmallBox);
                }
                __syncwarp();
            }
        }
        // no copy may be in flight when the CTA ends: its stages have been taken
        for (uint32_t i = c > W::kStages ? c - W::kStages : 0; on && i < c; ++i) {
            wait(empty(i % W::kStages), (i / W::kStages) & 1, gave_up, a);
            if (kEight && weights) wait(w_empty(i % W::kStages), (i / W::kStages) & 1, gave_up, a);
        }
    } else if (wid == 5) {
        if (rank == 0) {
            constexpr uint32_t kType = std::is_same_v<T, __nv_bfloat16> ? 1 : 0;
            const bool one = elect();
            const uint32_t tm = __shfl_sync(~0u, tmem, 0);
            const uint64_t w_op = operand(s_at, 16), x_op = operand(s_at + W::kX, 16);
            // The next stage is asked for while the present one's products are
            // issued: asking takes about as long as they do.
            uint32_t n = 0, st = 0, parity = 0, as = 0, a_parity = 0;
            bool ready = false, a_ready = false, on = true;
            for (; on && walk.next(a, line); ++n) {
                const uint32_t steps = walk.steps, buf = n & 1, d = tm + buf * W::kRows;
                // f32 sums, the operands' type, N, M = 256
                const uint32_t desc = 1u << 4 | kType << 7 | kType << 10 | (t.width / 8) << 17 | 16u << 24;
                if (n >= 2 && !(on = wait(sum_empty(buf), (n / 2 - 1) & 1, gave_up, a))) break;
                for (uint32_t j = 0; j < steps; ++j) {
                    if (!ready && !(on = wait(full(st), parity, gave_up, a))) break;
                    const uint64_t wa = w_op + st * (W::kStage >> 4), xa = x_op + st * (W::kStage >> 4);
                    const uint32_t now = st;
                    if (++st == W::kStages) st = 0, parity ^= 1;
#pragma unroll
                    for (uint32_t sub = 0; sub < W::kStep / 64; ++sub) {
                        if (kEight && !a_ready && !(on = wait(a_full(as), a_parity, gave_up, a))) break;
                        fence_after();
                        if (one) {
#pragma unroll
                            for (uint32_t kk = 0; kk < 4; ++kk) {
                                const uint64_t x = xa + ((sub * W::kHalf + kk * 32) >> 4);
                                if constexpr (kEight) mma2_ts(d, tm + W::kA + as * 32 + kk * 8, x, desc, j > 0 || sub > 0 || kk > 0);
                                else mma2_ss(d, wa + (kk * 32 >> 4), x, desc, j > 0 || kk > 0);
                            }
                            if constexpr (kEight) commit2(a_empty(as));
                        }
                        if constexpr (kEight) {
                            if (++as == W::kAs) as = 0, a_parity ^= 1;
                            a_ready = __all_sync(~0u, over(a_full(as), a_parity));
                        }
                    }
                    if (!on) break;
                    if (one) {
                        commit2(empty(now));
                        if (j + 1 == steps) commit2(sum_full(buf));
                    }
                    ready = __all_sync(~0u, over(full(st), parity));
                }
            }
            // nothing may be in flight when tensor memory is given back
            if (one) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(done) : "memory");
            __syncwarp();
            mbar_drain(done, 0);
        }
    } else if (wid < 4) {
        float *swap = reinterpret_cast<float *>(s + W::kSwap);
        uint32_t n = 0;
        for (; walk.next(a, line); ++n) {   // the four warps meet, so none leaves early
            const uint32_t buf = n & 1, at = tmem + buf * W::kRows + ((wid & 3) << 21);
            // this lane's channel of the weights, and of y
            const uint32_t c = p.gated ? t.c0 + rank * 64 + (tid & 63) : t.c0 + rank * 128 + tid;
            const bool partner = p.gated && wid >= 2;
            const uint32_t wc = partner ? p.n + c : c;
            const bool on = c < p.n;
            float scale = 1.f;
            if constexpr (kEight) scale = on ? __ldcg(p.w_scale + (uint64_t)t.e * a.channels + wc) : 0.f;
            wait(sum_full(buf), (n / 2) & 1, gave_up, a);
            fence_after();
            for (uint32_t q = 0; q < t.width; q += 32) {
                uint32_t raw[32];
                tm_ld(raw, at + q);
                wait_ld(raw);
                __syncwarp();
                if (q + 32 >= t.width) {   // the sums have been read
                    fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_pair(of_first(sum_empty(buf)));
                }
                const uint32_t rows = t.rows > q ? min(t.rows - q, 32u) : 0;
                if (a.splits > 1) {
                    if (on)
#pragma unroll
                        for (uint32_t r = 0; r < 32; ++r)
                            if (r < rows) a.part[t.split * a.part_split + (uint64_t)(t.row + q + r) * a.channels + wc] = __uint_as_float(raw[r]);
                    continue;
                }
                if constexpr (kEight) {
                    float sx = 0.f;
                    if (lane < rows) sx = __ldcg(p.x_scale + source_row(p, t.row + q + lane));
#pragma unroll
                    for (uint32_t r = 0; r < 32; ++r) raw[r] = __float_as_uint(__uint_as_float(raw[r]) * (__shfl_sync(~0u, sx, r) * scale));
                }
                if (!p.gated) {
                    store_rows(p, raw, t.row + q, rows, c, on);
                    continue;
                }
                // Gates and partners are in different warps: each hands half of
                // the rows over and works on the other half.
                asm volatile("bar.sync 1, 128;" ::: "memory");   // what was there has been read
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) swap[((partner ? 0 : 16) + r) * 64 + (tid & 63)] = __uint_as_float(partner ? raw[r] : raw[16 + r]);
                asm volatile("bar.sync 1, 128;" ::: "memory");
                const uint32_t r0 = partner ? 16 : 0;
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) {
                    const float other = swap[(r0 + r) * 64 + (tid & 63)];
                    const float x = __uint_as_float(partner ? raw[16 + r] : raw[r]);
                    raw[r] = __float_as_uint(partner ? gate(other, x) : gate(x, other));
                }
                store_rows(p, raw, t.row + q + r0, rows > r0 ? min(rows - r0, 16u) : 0, c, on);
            }
        }
    } else if (kEight && wid >= 8) {
        // 128 channels of 128 bytes to columns of halves: four groups of four warps
        // have 64 bytes of every other stage each
        const uint32_t group = (wid - 8) / 4, half = group & 1, r = (wid & 3) * 32 + lane;
        const uint32_t places = tmem + W::kA + ((wid & 3) << 21), bars_first = of_first(a_full(0));
        uint32_t c = 0, as = group, round = 0;
        bool on = true;
        while (on && walk.next(a, line)) {
            const uint32_t end = c + walk.steps;
            for (; c < end; ++c) {
                if ((c & 1) != group >> 1) continue;
                const uint32_t st = c % W::kStages;
                if (!(on = wait(w_full(st), (c / W::kStages) & 1, gave_up, a))) break;
                uint4 v[4];
#pragma unroll
                for (uint32_t x = 0; x < 4; ++x) v[x] = *reinterpret_cast<const uint4 *>(s + st * W::kStage + r * 128 + (((4 * half + x) ^ (r & 7)) << 4));
                __syncwarp();
                if (lane == 0) mbar_arrive(w_empty(st));
                uint32_t y[32];
#pragma unroll
                for (uint32_t x = 0; x < 4; ++x) {
                    bytes_to_halves(v[x].x, y[8 * x], y[8 * x + 1]);
                    bytes_to_halves(v[x].y, y[8 * x + 2], y[8 * x + 3]);
                    bytes_to_halves(v[x].z, y[8 * x + 4], y[8 * x + 5]);
                    bytes_to_halves(v[x].w, y[8 * x + 6], y[8 * x + 7]);
                }
                if (round && !(on = wait(a_empty(as), (round - 1) & 1, gave_up, a))) break;
                fence_after();
                tm_st(places + as * 32, y);
                wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) arrive_pair(bars_first + 16 * as);
                as += 4;   // the group's next use is the fourth from here
                if (as >= W::kAs) as -= W::kAs, ++round;
            }
        }
        // the last uses of all places have ended before the CTA does
        if constexpr (kEight) {
            const uint32_t uses = 2 * c;
            for (uint32_t u = uses > W::kAs ? uses - W::kAs : 0; on && u < uses; ++u) wait(a_empty(u % W::kAs), (u / W::kAs) & 1, gave_up, a);
        }
    }
    fence_before();
    __syncthreads();
    if (*gave_up && wid == 4) {   // copies whose stages nobody waited for
        const uint64_t t0 = now_ns();
        for (uint32_t i = 0; i < kWaits && now_ns() - t0 < 2'000'000; ++i) __nanosleep(1000);
    }
    __syncwarp();
    cluster_sync();   // nobody's shared memory or barriers are used any more
    fence_after();
    if (wid == 5) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// -- rows laid out for the tensor maps ----------------------------------------------------

// Row r of `to` is the row of x that row r reads, 8-bit values as halves: a warp
// a row.  Bound: memory, 2 bytes written for each value that is read.
template <bool kEight>
__global__ void __launch_bounds__(256) k_product_rows(ProductArgs p, char *to, uint64_t to_row) {
    pdl_enter();
    if (has_err(p.status)) return;
    const int32_t lo = p.offsets ? max(__ldcg(p.offsets), 0) : 0;
    const int32_t hi = p.offsets ? min(__ldcg(p.offsets + p.experts), (int32_t)p.rows) : (int32_t)p.rows;
    const uint32_t each = (p.k + 7) / 8, lane = threadIdx.x & 31;
    for (int64_t r = lo + blockIdx.x * 8ll + threadIdx.x / 32; r < hi; r += gridDim.x * 8ll) {
        const char *x = p.x + source_row(p, (uint32_t)r) * p.x_row;
        uint4 *y = reinterpret_cast<uint4 *>(to + (uint64_t)r * to_row);
#pragma unroll 8
        for (uint32_t at = lane; at < each; at += 32) {
            uint4 v;
            if constexpr (kEight) {
                const uint2 b = __ldcg(reinterpret_cast<const uint2 *>(x) + at);
                bytes_to_halves(b.x, v.x, v.y);
                bytes_to_halves(b.y, v.z, v.w);
            } else {
                v = __ldcg(reinterpret_cast<const uint4 *>(x) + at);
            }
            y[at] = v;
        }
    }
}

// -- joining parts of k ---------------------------------------------------------------------

// One expert's sums over parts of k, in their order, kV channels a thread.  Bound:
// memory (L2).
template <uint32_t kV>
__global__ void __launch_bounds__(256) k_product_join(WideArgs a) {
    pdl_enter();
    const ProductArgs &p = a.p;
    if (has_err(p.status)) return;
    const Rows rows = expert_rows(p, 0);
    const uint32_t each = p.n / kV, r = (uint32_t)rows.a + blockIdx.y;
    if (r >= (uint32_t)rows.b) return;
    const float sx = p.w_scale ? __ldcg(p.x_scale + source_row(p, r)) : 0.f;
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < each; i += gridDim.x * 256) {
        const uint32_t c = i * kV;
        float z[2][kV] = {};
        for (uint32_t h = 0; h < 1 + p.gated; ++h) {
            const float *from = a.part + (uint64_t)r * a.channels + h * p.n + c;
#pragma unroll 8
            for (uint32_t s = 0; s < a.splits; ++s, from += a.part_split) {
                float x[kV];
                if constexpr (kV == 4) *reinterpret_cast<float4 *>(x) = __ldcg(reinterpret_cast<const float4 *>(from));
                else x[0] = __ldcg(from);
#pragma unroll
                for (uint32_t v = 0; v < kV; ++v) z[h][v] += x[v];
            }
            if (p.w_scale)
#pragma unroll
                for (uint32_t v = 0; v < kV; ++v) z[h][v] *= sx * __ldcg(p.w_scale + h * p.n + c + v);
        }
#pragma unroll
        for (uint32_t v = 0; v < kV; ++v) store_y(p, (uint64_t)r * p.y_row + c + v, p.gated ? gate(z[0][v], z[1][v]) : z[0][v]);
    }
}

// -- launches ---------------------------------------------------------------------------------

CUtensorMapDataType map_type(uint32_t dtype) {
    return dtype == DM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : dtype == DM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
}

// Boxes of 128 bytes by `box` rows; rows and elements outside are zeros.
bool matrix_map(CUtensorMap *m, uint32_t dtype, const void *base, uint64_t k, uint64_t rows, uint64_t experts, uint64_t row_bytes,
                uint64_t expert_bytes, uint32_t box) {
    const uint32_t rank = experts ? 3 : 2;
    const cuuint64_t dims[3] = {k, rows, experts}, strides[2] = {row_bytes, expert_bytes};
    const cuuint32_t boxes[3] = {128 / dtype_size(dtype), box, 1}, steps[3] = {1, 1, 1};
    const EncodeTiled f = encode_tiled();
    return f && f(m, map_type(dtype), rank, const_cast<void *>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

#ifdef DM_DEBUG
std::atomic<uint64_t> g_test_wait_ns{0};
#endif

template <class T, bool kEight>
cudaError_t launch(const dm_weights *w, const WideArgs &a, const CUtensorMap &mw, const CUtensorMap &mx, const CUtensorMap &ms, uint32_t grid,
                   cudaStream_t st) {
    static SmemOptIn opt;
    DM_TRY(opt_in_smem(opt, Wide<kEight>::kBytes, k_product_wide<T, kEight>));
    return launch_pdl(k_product_wide<T, kEight>, grid, Wide<kEight>::kThreads, Wide<kEight>::kBytes, st, mw, mx, ms, a);
}

}  // namespace

WideShape wide_shape(const dm_weights *w, uint32_t rows, uint32_t gated, RowsAre are) {
    WideShape s{};
    const bool eight = w->dtype == DM_I8;
    const uint32_t most = eight ? Wide<true>::kRows : Wide<false>::kRows, step = eight ? Wide<true>::kStep : Wide<false>::kStep;
    s.blocks = gated ? (w->n / 2 + 127) / 128 : (w->n + 255) / 256;
    s.steps = (w->k + step - 1) / step;
    s.splits = 1;
    const uint32_t pairs = std::max(1, sm_count() / 2);
    if (w->experts == 1) {
        const uint64_t tiles = (uint64_t)s.blocks * ((rows + most - 1) / most);
        if (tiles * 2 <= pairs) s.splits = (uint32_t)std::min<uint64_t>({pairs / tiles, s.steps, 8});
    }
    s.x_row = align_up(w->k, 8) * 2;
    s.x_bytes = are == dm::kGathered || (eight && are == kPlain) ? align_up(rows * s.x_row, 256) : 0;
    s.part_bytes = s.splits > 1 ? align_up((uint64_t)s.splits * rows * w->n * 4, 256) : 0;
    return s;
}

cudaError_t launch_product_wide(const dm_weights *w, const ProductArgs &p, const WideShape &s, void *work, cudaStream_t st) {
    const bool eight = w->dtype == DM_I8;
    WideArgs a{p, nullptr, (uint64_t)p.rows * w->n, w->n, s.blocks, s.splits, s.steps, eight ? w->n / 2 : w->n};
#ifdef DM_DEBUG
    a.test_wait_ns = g_test_wait_ns;
#endif
    if (s.splits > 1) a.part = reinterpret_cast<float *>(static_cast<char *>(work) + s.x_bytes);
    const char *x = p.x;
    const uint64_t given = p.x_halves ? p.rows : p.x_rows;   // halves lie as the rows do
    uint64_t x_row = given > 1 ? p.x_row : s.x_row, x_rows = given;
    if (s.x_bytes) {
        const uint32_t grid = std::min((p.rows + 7) / 8, (uint32_t)sm_count() * 64);
        char *to = static_cast<char *>(work);
        const auto lay = eight ? k_product_rows<true> : k_product_rows<false>;
        DM_TRY(launch_pdl(lay, grid, 256, 0, st, p, to, s.x_row));
        x = to, x_row = s.x_row, x_rows = p.rows;
    }
    CUtensorMap mw, mx, ms;
    const uint32_t x_type = eight ? (uint32_t)DM_F16 : w->dtype, big = (eight ? Wide<true>::kRows : Wide<false>::kRows) / 2;
    if (!matrix_map(&mw, w->dtype, w->w, w->k, w->n, w->experts, p.w_row, w->experts > 1 ? p.w_expert : align_up(w->n * p.w_row, 16), 64) ||
        !matrix_map(&mx, x_type, x, p.k, x_rows, 0, x_row, 0, big) || !matrix_map(&ms, x_type, x, p.k, x_rows, 0, x_row, 0, kSmallBox))
        return cudaErrorInvalidValue;
    const uint32_t grid = std::max(2u, (uint32_t)sm_count() / 2 * 2);
    const auto run = eight ? launch<__half, true> : w->dtype == DM_F16 ? launch<__half, false> : launch<__nv_bfloat16, false>;
    DM_TRY(run(w, a, mw, mx, ms, grid, st));
    if (s.splits == 1) return cudaSuccess;
    const bool four = p.n % 4 == 0;
    const uint32_t each = four ? p.n / 4 : p.n;
    return launch_pdl(four ? k_product_join<4> : k_product_join<1>, dim3((each + 255) / 256, p.rows), 256, 0, st, a);
}

}  // namespace dm

extern "C" dm_status dm_test_product_wait(uint64_t ns) {
#ifdef DM_DEBUG
    dm::g_test_wait_ns = ns;
    return DM_OK;
#else
    return ns ? DM_ERR_INVALID_ARG : DM_OK;
#endif
}
