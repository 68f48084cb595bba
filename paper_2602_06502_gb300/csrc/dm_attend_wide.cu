// dm_attend_wide.cu -- attention over the paged cache for many rows per key
// head: a group's rows against its shared prefix, prompts, drafts.
//
// One CTA per SM walks its units (dm_attend.cuh).  Rows come in two tiles of
// 128 (A and B) that read the same keys:
//   warps 0-3, 4-7  softmax of A and of B, a row per thread
//   warps 8, 10, 11 TMA: keys and values page by page into a ring of stages
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
// there are 256 rows; memory where there are few.  16 prompts' 100-1,000 new
// tokens behind 2,048-8,192 cached ones, 32 heads over 8, D = 128: 550 us, 1.6
// PFLOP/s (the tensor pipe busy for 72% of the cycles).
#include <algorithm>

#include "dm_attend.cuh"

namespace dm {
namespace {

constexpr uint32_t kWideT = 384;   // three warpgroups: softmax of A, of B, and the issuing warps

template <int D>
struct Wide {
    static constexpr uint32_t kTile = 128 * D * 2;                  // bytes of 128 rows
    static constexpr uint32_t kStages = D == 128 ? 5 : 10;
    static constexpr uint32_t kRing = 2 * kTile;                    // after Q of A and B
    static constexpr uint32_t kBars = kRing + kStages * kTile;
    // full, empty per stage; then per tile: q, s, p (two halves), o; then done
    static constexpr uint32_t kWord = kBars + 16 * kStages + 8 * 11; // give-up word, tensor memory address
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

// 32 bytes, 32-byte aligned.
__device__ __forceinline__ void store32(void *to, const uint32_t *r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

// True in one thread of the warp.
__device__ __forceinline__ bool elect() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

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

// 64 scores of this thread's row; minus infinity from the `seen`-th on.
__device__ __forceinline__ void scores64(uint32_t *raw, uint32_t at, int32_t seen) {
    tm_ld(raw, at);
    tm_ld(raw + 32, at + 32);
    wait_ld(raw, 64);
    if (seen < 64)
#pragma unroll
        for (int32_t i = 0; i < 64; ++i)
            if (i >= seen) raw[i] = 0xFF800000u;
    __syncwarp();
}

template <class T, int D>
__global__ void __launch_bounds__(kWideT, 1)
    k_attend_wide(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, AttendArgs p) {
    using W = Wide<D>;
    extern __shared__ char s_raw[];
    char *s = reinterpret_cast<char *>(align_up(reinterpret_cast<uint64_t>(s_raw), 1024));
    const uint32_t s_at = smem_addr(s), bars = s_at + W::kBars, more = bars + 16 * W::kStages;
    volatile uint32_t *gave_up = reinterpret_cast<uint32_t *>(s + W::kWord);
    const uint32_t tid = threadIdx.x, wid = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    auto full = [&](uint32_t i) { return bars + 16 * i; };
    auto empty = [&](uint32_t i) { return bars + 16 * i + 8; };
    auto q_full = [&](uint32_t x) { return more + 8 * x; };
    auto s_full = [&](uint32_t x) { return more + 16 + 8 * x; };
    auto p_full = [&](uint32_t x, uint32_t half) { return more + 32 + 16 * x + 8 * half; };
    auto o_full = [&](uint32_t x) { return more + 64 + 8 * x; };
    const uint32_t done = more + 80;
    if (tid == 0) {
        for (uint32_t i = 0; i < W::kStages; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
        }
        for (uint32_t x = 0; x < 2; ++x) {
            mbar_init(q_full(x), 128);
            mbar_init(s_full(x), 1);
            mbar_init(p_full(x, 0), 128);
            mbar_init(p_full(x, 1), 128);
            mbar_init(o_full(x), 1);
        }
        mbar_init(done, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // first the wait, then the leave for the next kernel: the narrow one relies
    // on all before this kernel being complete
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (__syncthreads_or(has_err(p.status) || p.w.head->key != p.key || blockIdx.x >= p.w.head->ctas[0])) return;
    if (wid == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s_at + W::kWord + 4) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(s + W::kWord + 4);
    Walk<0> w(p);

    // 384 x 168 registers at the start; 2 x 128 x 200 + 128 x 104 are as many
    if (wid >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (wid != 9) {
            const uint32_t pw = wid == 8 ? 0 : wid - 9;
            uint32_t c = 0;   // stages so far: K of unit 0, V of unit 0, K of unit 1, ...
            bool stop = false;
            for (Slots<0, D, kWideKeys, 3> next(p, w, pw); next.more && !stop; next.step(p)) {
                for (uint32_t v = 0; v < 2; ++v, ++c) {
                    const uint32_t i = c % W::kStages, round = c / W::kStages;
                    if (round) mbar_wait(empty(i), (round - 1) & 1, gave_up, p);
                    if ((stop = __any_sync(~0u, *gave_up))) break;
                    if (withheld(p, c)) continue;
                    if (pw == 0 && lane == 0) mbar_expect(full(i), W::kTile);   // the phase ends with this and all the bytes
                    __syncwarp();
                    next.boxes.load(p, v ? &mv : &mk, s_at + W::kRing + i * W::kTile, full(i), next.tok, next.head);
                }
            }
            // no copy may be in flight when the CTA ends
            for (uint32_t i = c > W::kStages ? c - W::kStages : 0; i < c; ++i)
                mbar_drain(full(i % W::kStages), (i / W::kStages) & 1);
        } else {
            constexpr uint32_t kType = Pack2<T>::kMmaType;
            // f32 accumulators, the operands' type, N, M = 128; V's rows (dims) are contiguous
            constexpr uint32_t desc_s = 1u << 4 | kType << 7 | kType << 10 | (kWideKeys / 8) << 17 | 8u << 24;
            constexpr uint32_t desc_o = 1u << 4 | kType << 7 | kType << 10 | 1u << 16 | (D / 8) << 17 | 8u << 24;
            // The tensor cores' operands are in uniform registers: one thread
            // elected by the whole warp issues, and what it issues is the same
            // in every lane, so that no value has to be moved there first.
            const bool one = elect();
            const uint32_t tm = __shfl_sync(~0u, tmem, 0);
            const uint64_t q_op = operand(s_at, 16), k_op = operand(s_at + W::kRing, 16), v_op = operand(s_at + W::kRing, 16384);
            auto scores = [&](uint32_t x, uint32_t stage) {   // S_x = Q_x K^T
                const uint64_t qa = q_op + x * (W::kTile >> 4), ka = k_op + stage * (W::kTile >> 4);
                if (one) {
#pragma unroll
                    for (uint32_t kk = 0; kk < D / 16; ++kk) {
                        const uint32_t at = (kk / 4 * 16384 + kk % 4 * 32) >> 4;
                        mma_ss(tm + W::kS + x * 128, qa + at, ka + at, desc_s, kk > 0);
                    }
                    mma_commit(s_full(x));
                }
                __syncwarp();
            };
            auto product = [&](uint32_t x, uint32_t stage, uint32_t half, bool first) {   // O_x += P_x V, over half the keys
                const uint64_t va = v_op + stage * (W::kTile >> 4) + half * 512;
                if (one) {
#pragma unroll
                    for (uint32_t kk = 0; kk < 4; ++kk)
                        mma_ts(tm + W::kO + x * D, tm + W::kS + x * 128 + half * 32 + kk * 8, va + kk * 128, desc_o, !first || half || kk > 0);
                }
                __syncwarp();
            };
            auto release = [&](uint32_t bar) {
                if (one) mma_commit(bar);
                __syncwarp();
            };
            uint32_t c = 0, pieces[2] = {0, 0}, ps[2] = {0, 0};   // stages; pieces and weight tiles of A and B
            while (w.next(p)) {
                const uint32_t X = w.k.rows > 128 ? 2 : 1;
                for (uint32_t x = 0; x < X; ++x) mbar_wait(q_full(x), pieces[x] & 1, gave_up, p);
                mbar_wait(full(c % W::kStages), (c / W::kStages) & 1, gave_up, p);
                fence_after();
                for (uint32_t x = 0; x < X; ++x) scores(x, c % W::kStages);
                release(empty(c % W::kStages));
                for (uint32_t j = 0; j < w.units; ++j) {
                    const uint32_t v = c + 1, vs = v % W::kStages, nk = c + 2, ns = nk % W::kStages;
                    const bool last = j + 1 == w.units;
                    mbar_wait(full(vs), (v / W::kStages) & 1, gave_up, p);
                    const int32_t left = w.k.kv1 - (w.k.kv0 + (int32_t)((w.j0 + j) * kWideKeys));
                    if (left > 0 && left < (int32_t)kWideKeys && (left & ((1 << p.B_log) - 1))) {
                        // slots of the last page behind the end hold whatever was
                        // there; a weight of zero does not silence an infinity
                        const uint32_t to = (uint32_t)align_up(left, 1u << p.B_log), chunks = (to - left) * (D / 8);
                        for (uint32_t e = lane; e < chunks; e += 32) {
                            const uint32_t row = left + e / (D / 8), ch = e % (D / 8);
                            *reinterpret_cast<uint4 *>(s + W::kRing + vs * W::kTile + ch / 8 * 16384 + row * 128 + ((ch % 8) ^ (row % 8)) * 16) =
                                make_uint4(0, 0, 0, 0);
                        }
                        fence_async();
                        __syncwarp();
                    }
                    for (uint32_t x = 0; x < X; ++x) {
                        for (uint32_t half = 0; half < 2; ++half) {
                            mbar_wait(p_full(x, half), ps[x] & 1, gave_up, p);
                            fence_after();
                            product(x, vs, half, j == 0);
                        }
                        ++ps[x];
                        if (last) {
                            release(o_full(x));
                        } else {
                            if (x == 0) mbar_wait(full(ns), (nk / W::kStages) & 1, gave_up, p);
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
            release(done);
            mbar_drain(done, 0);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const uint32_t x = wid >> 2, r = tid & 127;   // tile, row (= tensor memory lane)
        const uint32_t lanes = (wid & 3) << 21;       // this warp's lanes of tensor memory
        const uint32_t t_s = tmem + W::kS + x * 128 + lanes, t_o = tmem + W::kO + x * D + lanes;
        uint32_t ss = 0, pieces = 0;
        // The next piece that has rows in this tile.
        auto next = [&](Walk<0> &k) {
            while (k.next(p))
                if (k.k.rows > 128 * x) return true;
            return false;
        };
        // A piece's Q, 16 bytes a thread and step, zeros for the rows that are
        // not there.  Begun when the last scores of the piece before are done,
        // so that the next piece's first product need not wait for it.
        auto fetch = [&](const Walk<0> &k) {
            const uint32_t rows = min(128u, k.k.rows - 128 * x), ch = r % (D / 8);
#pragma unroll 4
            for (uint32_t row = r / (D / 8); row < 128; row += 1024 / D) {
                const Row at = row_at(p, k.k, 128 * x + min(row, rows - 1));
                const char *src = p.q + (uint64_t)(k.k.token + at.token) * p.q_token + (uint64_t)(k.head * p.G + at.head) * p.q_head + ch * 16;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s_at + x * W::kTile + ch / 8 * 16384 + row * 128 + ((ch % 8) ^ (row % 8)) * 16),
                             "l"(src), "r"(row < rows ? 16 : 0)
                             : "memory");
            }
        };
        auto fetched = [&] {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async();
            mbar_arrive(q_full(x));
        };
        bool more = next(w);
        if (more) {
            fetch(w);
            fetched();
        }
        while (more) {
            const uint32_t rows = min(128u, w.k.rows - 128 * x);
            const Row mine = row_at(p, w.k, 128 * x + min(r, rows - 1));
            // rows that are not there (their Q is zero) see everything: a row that
            // is masked costs its warp the masking of every tile
            const int32_t limit = r < rows ? row_limit(w.k, mine.token) : INT32_MAX;
            Walk<0> ahead = w;
            more = next(ahead);
            float m = -INFINITY, l = 0.f;   // the maximum in the scores' own unit
            for (uint32_t j = 0; j < w.units; ++j, ++ss) {
                mbar_wait(s_full(x), ss & 1, gave_up, p);
                fence_after();
                if (j + 1 == w.units && more) fetch(ahead);
                const int32_t seen = limit - (w.k.kv0 + (int32_t)((w.j0 + j) * kWideKeys));
                // 64 scores at a time: the maximum over the second half, then
                // over the first, which stays in registers
                uint32_t raw[64];
                float top = -INFINITY;
#pragma unroll
                for (uint32_t half = 2; half-- > 0;) {
                    scores64(raw, t_s + 64 * half, seen - 64 * (int32_t)half);
                    float m0 = top, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
                    for (uint32_t i = 0; i < 64; i += 8) {
                        m0 = fmaxf(fmaxf(m0, __uint_as_float(raw[i])), __uint_as_float(raw[i + 1]));
                        m1 = fmaxf(fmaxf(m1, __uint_as_float(raw[i + 2])), __uint_as_float(raw[i + 3]));
                        m2 = fmaxf(fmaxf(m2, __uint_as_float(raw[i + 4])), __uint_as_float(raw[i + 5]));
                        m3 = fmaxf(fmaxf(m3, __uint_as_float(raw[i + 6])), __uint_as_float(raw[i + 7]));
                    }
                    top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
                }
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
                const float2 scale2 = make_float2(p.scale2, p.scale2), minus = make_float2(-base, -base);
                float2 la = make_float2(0.f, 0.f), lb = la;
                // the weights in the cache's type, as the tensor cores take
                // them; the product over the first half of the keys begins
                // while the second half is computed
#pragma unroll
                for (uint32_t half = 0; half < 2; ++half) {
                    if (half) scores64(raw, t_s + 64, seen - 64);
#pragma unroll
                    for (uint32_t i = 0; i < 64; i += 4) {
                        const float2 a = fma2(make_float2(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), scale2, minus);
                        const float2 b = fma2(make_float2(__uint_as_float(raw[i + 2]), __uint_as_float(raw[i + 3])), scale2, minus);
                        const float2 ea = make_float2(exp2_(a.x), exp2_(a.y)), eb = make_float2(exp2_(b.x), exp2_(b.y));
                        la = add2(la, ea);
                        lb = add2(lb, eb);
                        raw[i / 2] = Pack2<T>::pack(ea.x, ea.y);
                        raw[i / 2 + 1] = Pack2<T>::pack(eb.x, eb.y);
                    }
                    tm_st(t_s + 32 * half, raw);
                    wait_st();
                    fence_before();
                    mbar_arrive(p_full(x, half));
                }
                l += (la.x + la.y) + (lb.x + lb.y);
            }
            if (more) fetched();
            mbar_wait(o_full(x), pieces & 1, gave_up, p);
            ++pieces;
            fence_after();
            const bool whole = w.whole(), on = r < rows;
            const uint64_t tok = (uint64_t)(w.k.token + mine.token);
            const uint32_t h = w.head * p.G + mine.head;
            const uint64_t part = whole ? 0 : w.part_row(p) + 128 * x + r;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            char *dst = p.o + tok * p.o_token + h * p.o_head;
#pragma unroll
            for (uint32_t q = 0; q < D / 32; ++q) {
                uint32_t o[32];
                tm_ld(o, t_o + 32 * q);
                wait_ld(o);
                // A row per thread is 32 lines per store, so the widest store
                // there is; 16 bytes where the caller's rows allow no more.
                if (on && whole) {
                    uint32_t y[16];
#pragma unroll
                    for (uint32_t i = 0; i < 16; ++i) y[i] = Pack2<T>::pack(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
#pragma unroll
                    for (uint32_t i = 0; i < 16; i += 8) {
                        if (p.o_wide) {
                            store32(dst + q * 64 + i * 4, y + i);
                        } else {
                            *reinterpret_cast<uint4 *>(dst + q * 64 + i * 4) = make_uint4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                            *reinterpret_cast<uint4 *>(dst + q * 64 + i * 4 + 16) = make_uint4(y[i + 4], y[i + 5], y[i + 6], y[i + 7]);
                        }
                    }
                } else if (on) {
                    float *to = p.w.part[0] + part * D + q * 32;
#pragma unroll
                    for (uint32_t i = 0; i < 32; i += 8) store32(to + i, o + i);
                }
                __syncwarp();
            }
            if (on) {
                const float m2 = m * p.scale2;   // minus infinity where the row saw nothing
                if (!whole) p.w.ml[0][part] = make_float2(m2, l);
                else if (p.lse) p.lse[tok * p.q_heads + h] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * 0.69314718056f;
            }
            __syncwarp();
            fence_before();   // O has been read; the next product may write it
            w = ahead;
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
    return launch_pdl(k_attend_wide<T, D>, p.ctas[0], kWideT, Wide<D>::kBytes, st, mk, mv, p);
}

}  // namespace

cudaError_t launch_attend_wide(const dm_cache *c, const AttendArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st) {
    if (c->dtype == DM_BF16) return c->head_dim == 64 ? launch<__nv_bfloat16, 64>(p, mk, mv, st) : launch<__nv_bfloat16, 128>(p, mk, mv, st);
    return c->head_dim == 64 ? launch<__half, 64>(p, mk, mv, st) : launch<__half, 128>(p, mk, mv, st);
}

}  // namespace dm
