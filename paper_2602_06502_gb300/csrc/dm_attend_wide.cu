// dm_attend_wide.cu -- attention over the paged cache for many rows per key
// head: a group's rows against its shared prefix, prompts, drafts.
//
// One CTA per SM walks its units (dm_attend.cuh).  Rows come in two tiles of
// 128 (A and B) that read the same keys:
//   warps 0-3, 4-7  softmax of A and of B, a row per thread
//   warp 8          TMA: keys and values page by page into a ring of stages
//   warp 9          tcgen05.mma: S = Q K^T (128 x 128, both operands in shared
//                   memory), O += P V (P in tensor memory over S, V in shared
//                   memory, dims contiguous)
// While A's softmax runs the tensor cores have B's products, and the other way
// round.  Everything that one thread issues to the tensor cores completes in
// order, so a score tile's commit also says that the product before it is done,
// and S can be written over P without a wait.
//
// O stays in tensor memory.  Its scale follows a row's maximum only when that
// has grown by more than 2^8: until then the weights are at most 2^8, exact in
// the sums, and the rescaling of 128 x D values is skipped.
//
// Bound: the exponentials and the tensor cores in about equal parts where
// there are 256 rows; memory where there are few.
#include <algorithm>

#include "dm_attend.cuh"

namespace dm {
namespace {

constexpr uint32_t kWideT = 320;

template <int D>
struct Wide {
    static constexpr uint32_t kTile = 128 * D * 2;                  // bytes of 128 rows
    static constexpr uint32_t kStages = D == 128 ? 5 : 10;
    static constexpr uint32_t kRing = 2 * kTile;                    // after Q of A and B
    static constexpr uint32_t kBars = kRing + kStages * kTile;
    // full, empty per stage; then per tile: q, s, p, o; then done
    static constexpr uint32_t kWord = kBars + 16 * kStages + 8 * 9; // give-up word, tensor memory address
    static constexpr uint32_t kBytes = kWord + 16 + 1024;
    static constexpr uint32_t kS = 0, kO = 256;                     // tensor memory columns: S of A, B; O of A, B
};

// Shared-memory operand of 128-byte rows in groups of 8 (128-byte swizzle).
// K contiguous: groups of 8 rows are 1024 bytes apart.  Rows contiguous (V):
// groups of 8 keys are 1024 bytes apart, halves of 64 dims 128 rows.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading) {
    return (uint64_t)((at & 0x3FFFF) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(desc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 32 columns of this warp's 32 lanes.
__device__ __forceinline__ void tm_ld(uint32_t *r, uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tm_st(uint32_t at, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// The loads are asynchronous: their registers are only theirs after the wait.
// Naming them here keeps the compiler from using them before it.
__device__ __forceinline__ void tm_use(uint32_t *r) {
    asm volatile(""
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void wait_ld(uint32_t *r, uint32_t n = 32) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (uint32_t i = 0; i < n; i += 32) tm_use(r + i);
}

template <class T, int D>
__global__ void __launch_bounds__(kWideT, 1)
    k_attend_wide(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, AttendArgs p) {
    using W = Wide<D>;
    extern __shared__ char s_raw[];
    char *s = reinterpret_cast<char *>(align_up(reinterpret_cast<uint64_t>(s_raw), 1024));
    const uint32_t s_at = smem_addr(s), bars = s_at + W::kBars, more = bars + 16 * W::kStages;
    volatile uint32_t *gave_up = reinterpret_cast<uint32_t *>(s + W::kWord);
    const uint32_t tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    auto full = [&](uint32_t i) { return bars + 16 * i; };
    auto empty = [&](uint32_t i) { return bars + 16 * i + 8; };
    auto q_full = [&](uint32_t x) { return more + 8 * x; };
    auto s_full = [&](uint32_t x) { return more + 16 + 8 * x; };
    auto p_full = [&](uint32_t x) { return more + 32 + 8 * x; };
    auto o_full = [&](uint32_t x) { return more + 48 + 8 * x; };
    const uint32_t done = more + 64;
    if (__syncthreads_or(has_err(p.status) || !p.w.head->ok || p.w.head->units[0] == 0)) return;
    if (tid == 0) {
        for (uint32_t i = 0; i < W::kStages; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
        }
        for (uint32_t x = 0; x < 2; ++x) {
            mbar_init(q_full(x), 128);
            mbar_init(s_full(x), 1);
            mbar_init(p_full(x), 128);
            mbar_init(o_full(x), 1);
        }
        mbar_init(done, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s_at + W::kWord + 4) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(s + W::kWord + 4);
    Walk<0> w(p);

    if (wid == 8) {
        uint32_t c = 0;   // stages so far: K of unit 0, V of unit 0, K of unit 1, ...
        bool stop = false;
        while (!stop && w.next(p)) {
            const int32_t *table = p.tables + (uint64_t)w.k.row * p.max_blocks;
            const uint32_t blocks = ((uint32_t)w.k.kv1 + p.B - 1) / p.B;
            for (uint32_t j = 0; j < 2 * w.units; ++j, ++c) {
                const uint32_t i = c % W::kStages, round = c / W::kStages;
                if (round) mbar_wait(empty(i), (round - 1) & 1, gave_up, p.status);
                if (__any_sync(~0u, *gave_up)) {
                    stop = true;
                    break;
                }
                if (lane == 0) mbar_expect(full(i), W::kTile);
                __syncwarp();
                load_keys<D, kWideKeys>(p, j & 1 ? &mv : &mk, s_at + W::kRing + i * W::kTile, full(i), table,
                                        (uint32_t)w.k.kv0 + (w.j0 + j / 2) * kWideKeys, blocks, w.head);
            }
        }
        // no copy may be in flight when the CTA ends
        for (uint32_t i = c > W::kStages ? c - W::kStages : 0; i < c; ++i)
            mbar_drain(full(i % W::kStages), (i / W::kStages) & 1);
    } else if (wid == 9) {
        constexpr uint32_t kType = Pack2<T>::kMmaType;
        // f32 accumulators, the operands' type, N, M = 128; V's rows (dims) are contiguous
        constexpr uint32_t desc_s = 1u << 4 | kType << 7 | kType << 10 | (kWideKeys / 8) << 17 | 8u << 24;
        constexpr uint32_t desc_o = 1u << 4 | kType << 7 | kType << 10 | 1u << 16 | (D / 8) << 17 | 8u << 24;
        auto scores = [&](uint32_t x, uint32_t stage) {   // S_x = Q_x K^T
            const uint32_t qa = s_at + x * W::kTile, ka = s_at + W::kRing + stage * W::kTile;
            if (lane == 0 && !*gave_up) {
#pragma unroll
                for (uint32_t kk = 0; kk < D / 16; ++kk) {
                    const uint32_t at = kk / 4 * 16384 + kk % 4 * 32;
                    mma_ss(tmem + W::kS + x * 128, operand(qa + at, 16), operand(ka + at, 16), desc_s, kk > 0);
                }
                mma_commit(s_full(x));
            }
            __syncwarp();
        };
        auto product = [&](uint32_t x, uint32_t stage, bool first) {   // O_x += P_x V
            const uint32_t va = s_at + W::kRing + stage * W::kTile;
            if (lane == 0 && !*gave_up) {
#pragma unroll
                for (uint32_t kk = 0; kk < kWideKeys / 16; ++kk)
                    mma_ts(tmem + W::kO + x * D, tmem + W::kS + x * 128 + kk * 8, operand(va + kk * 2048, 16384), desc_o, !first || kk > 0);
            }
            __syncwarp();
        };
        auto release = [&](uint32_t bar) {
            if (lane == 0 && !*gave_up) mma_commit(bar);
            __syncwarp();
        };
        uint32_t c = 0, pieces[2] = {0, 0}, ps[2] = {0, 0};   // stages; pieces and weight tiles of A and B
        while (w.next(p)) {
            const uint32_t X = w.k.rows > 128 ? 2 : 1;
            for (uint32_t x = 0; x < X; ++x) mbar_wait(q_full(x), pieces[x] & 1, gave_up, p.status);
            mbar_wait(full(c % W::kStages), (c / W::kStages) & 1, gave_up, p.status);
            fence_after();
            for (uint32_t x = 0; x < X; ++x) scores(x, c % W::kStages);
            release(empty(c % W::kStages));
            for (uint32_t j = 0; j < w.units; ++j) {
                const uint32_t v = c + 1, vs = v % W::kStages, nk = c + 2, ns = nk % W::kStages;
                const bool last = j + 1 == w.units;
                mbar_wait(full(vs), (v / W::kStages) & 1, gave_up, p.status);
                const int32_t left = w.k.kv1 - (w.k.kv0 + (int32_t)((w.j0 + j) * kWideKeys));
                if (left > 0 && left < (int32_t)kWideKeys && left % (int32_t)p.B) {
                    // slots of the last page behind the end hold whatever was
                    // there; a weight of zero does not silence an infinity
                    const uint32_t to = align_up((uint32_t)left, p.B), chunks = (to - left) * (D / 8);
                    for (uint32_t e = lane; e < chunks; e += 32) {
                        const uint32_t row = left + e / (D / 8), ch = e % (D / 8);
                        *reinterpret_cast<uint4 *>(s + W::kRing + vs * W::kTile + ch / 8 * 16384 + row * 128 + ((ch % 8) ^ (row % 8)) * 16) =
                            make_uint4(0, 0, 0, 0);
                    }
                    fence_async();
                    __syncwarp();
                }
                for (uint32_t x = 0; x < X; ++x) {
                    mbar_wait(p_full(x), ps[x] & 1, gave_up, p.status);
                    ++ps[x];
                    fence_after();
                    product(x, vs, j == 0);
                    if (last) {
                        release(o_full(x));
                    } else {
                        if (x == 0) mbar_wait(full(ns), (nk / W::kStages) & 1, gave_up, p.status);
                        fence_after();
                        scores(x, ns);
                    }
                }
                release(empty(vs));
                if (!last) release(empty(ns));
                c += 2;
            }
            for (uint32_t x = 0; x < X; ++x) ++pieces[x];
        }
        // nothing may be in flight when tensor memory is given back
        if (lane == 0) mma_commit(done);
        __syncwarp();
        mbar_drain(done, 0);
    } else {
        const uint32_t x = wid >> 2, r = tid & 127;   // tile, row (= tensor memory lane)
        const uint32_t lanes = (wid & 3) << 21;       // this warp's lanes of tensor memory
        const uint32_t t_s = tmem + W::kS + x * 128 + lanes, t_o = tmem + W::kO + x * D + lanes;
        uint32_t ss = 0, pieces = 0;
        while (w.next(p)) {
            if (w.k.rows <= 128 * x) continue;
            const uint32_t rows = min(128u, w.k.rows - 128 * x);
            // Q of this tile: 16 bytes a thread and step, zeros for the rows that are not there
#pragma unroll
            for (uint32_t it = 0; it < D / 8; ++it) {
                const uint32_t e = it * 128 + r, row = e / (D / 8), ch = e % (D / 8);
                uint4 v = make_uint4(0, 0, 0, 0);
                if (row < rows) {
                    const uint32_t rr = w.k.row0 + 128 * x + row;
                    v = __ldg(reinterpret_cast<const uint4 *>(p.q + (uint64_t)(w.k.token0 + rr / p.G) * p.q_token +
                                                              (uint64_t)(w.head * p.G + rr % p.G) * p.q_head + ch * 16));
                }
                *reinterpret_cast<uint4 *>(s + x * W::kTile + ch / 8 * 16384 + row * 128 + ((ch % 8) ^ (row % 8)) * 16) = v;
            }
            fence_async();
            fence_before();   // the last piece's O has been read
            mbar_arrive(q_full(x));
            const int32_t limit = r < rows ? row_limit(w.k, 128 * x + r, p.G) : 0;
            float m = -INFINITY, l = 0.f;   // the maximum in the scores' own unit
            for (uint32_t j = 0; j < w.units; ++j, ++ss) {
                mbar_wait(s_full(x), ss & 1, gave_up, p.status);
                fence_after();
                uint32_t raw[128];
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) tm_ld(raw + 32 * q, t_s + 32 * q);
                wait_ld(raw, 128);
                float *sc = reinterpret_cast<float *>(raw);
                const int32_t seen = limit - (w.k.kv0 + (int32_t)((w.j0 + j) * kWideKeys));
                if (seen < (int32_t)kWideKeys)
#pragma unroll
                    for (int32_t i = 0; i < (int32_t)kWideKeys; ++i)
                        if (i >= seen) sc[i] = -INFINITY;
                float m0 = sc[0], m1 = sc[1], m2 = sc[2], m3 = sc[3];
#pragma unroll
                for (uint32_t i = 4; i < kWideKeys; i += 4) {
                    m0 = fmaxf(m0, sc[i]);
                    m1 = fmaxf(m1, sc[i + 1]);
                    m2 = fmaxf(m2, sc[i + 2]);
                    m3 = fmaxf(m3, sc[i + 3]);
                }
                const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
                float f = 1.f;
                if ((top - m) * p.scale2 > 8.f) {
                    f = exp2_((m - top) * p.scale2);   // 0 for the first that the row sees
                    m = top;
                }
                if (__any_sync(~0u, f != 1.f)) {
                    l *= f;
                    if (j > 0) {
#pragma unroll
                        for (uint32_t q = 0; q < D / 32; ++q) {
                            uint32_t o[32];
                            tm_ld(o, t_o + 32 * q);
                            wait_ld(o);
#pragma unroll
                            for (uint32_t i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tm_st(t_o + 32 * q, o);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.f : m * p.scale2;
                float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
                for (uint32_t i = 0; i < kWideKeys; i += 4) {
                    const float a = exp2_(fmaf(sc[i], p.scale2, -base)), b = exp2_(fmaf(sc[i + 1], p.scale2, -base));
                    const float d = exp2_(fmaf(sc[i + 2], p.scale2, -base)), e = exp2_(fmaf(sc[i + 3], p.scale2, -base));
                    l0 += a;
                    l1 += b;
                    l2 += d;
                    l3 += e;
                    // the weights in the cache's type, as the tensor cores take them
                    raw[i / 2] = Pack2<T>::pack(a, b);
                    raw[i / 2 + 1] = Pack2<T>::pack(d, e);
                }
                l += (l0 + l1) + (l2 + l3);
                tm_st(t_s, raw);
                tm_st(t_s + 32, raw + 32);
                wait_st();
                fence_before();
                mbar_arrive(p_full(x));
            }
            mbar_wait(o_full(x), pieces & 1, gave_up, p.status);
            ++pieces;
            fence_after();
            const bool whole = w.whole(), on = r < rows;
            const uint32_t rr = w.k.row0 + 128 * x + (on ? r : 0);
            const uint64_t tok = (uint64_t)(w.k.token0 + rr / p.G);
            const uint32_t h = w.head * p.G + rr % p.G;
            const uint64_t part = whole ? 0 : w.part_row(p) + 128 * x + r;
            const float inv = l > 0.f ? 1.f / l : 0.f;
            char *dst = p.o + tok * p.o_token + h * p.o_head;
#pragma unroll
            for (uint32_t q = 0; q < D / 32; ++q) {
                uint32_t o[32];
                tm_ld(o, t_o + 32 * q);
                wait_ld(o);
                if (on && whole) {
#pragma unroll
                    for (uint32_t i = 0; i < 32; i += 8) {
                        uint4 v;
                        v.x = Pack2<T>::pack(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
                        v.y = Pack2<T>::pack(__uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
                        v.z = Pack2<T>::pack(__uint_as_float(o[i + 4]) * inv, __uint_as_float(o[i + 5]) * inv);
                        v.w = Pack2<T>::pack(__uint_as_float(o[i + 6]) * inv, __uint_as_float(o[i + 7]) * inv);
                        *reinterpret_cast<uint4 *>(dst + q * 64 + i * 2) = v;
                    }
                } else if (on) {
                    uint4 *to = reinterpret_cast<uint4 *>(p.w.part[0] + part * D + q * 32);
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) to[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
                __syncwarp();
            }
            if (on) {
                const float m2 = m * p.scale2;   // minus infinity where the row saw nothing
                if (!whole) p.w.ml[0][part] = make_float2(m2, l);
                else if (p.lse) p.lse[tok * p.q_heads + h] = l > 0.f ? (m2 + log2f(l)) * 0.69314718056f : -INFINITY;
            }
            __syncwarp();
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (wid == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <class T, int D>
cudaError_t launch(const AttendArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st) {
    static SmemOptIn opt;
    DM_TRY(opt_in_smem(opt, Wide<D>::kBytes, k_attend_wide<T, D>));
    k_attend_wide<T, D><<<p.ctas[0], kWideT, Wide<D>::kBytes, st>>>(mk, mv, p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_wide(const dm_cache *c, const AttendArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st) {
    if (c->dtype == DM_BF16) return c->head_dim == 64 ? launch<__nv_bfloat16, 64>(p, mk, mv, st) : launch<__nv_bfloat16, 128>(p, mk, mv, st);
    return c->head_dim == 64 ? launch<__half, 64>(p, mk, mv, st) : launch<__half, 128>(p, mk, mv, st);
}

}  // namespace dm
