// dm_attend.cu -- attention over the paged cache: the step's plan
// (dm_cache_plan), the kernel for few rows per key head, and the joining of
// parts; dm_attend_wide.cu has the kernel for many rows.
//
// Softmax in one pass over the keys: per row a running maximum m (scores in
// base 2), l = sum 2^(s - m) and O = sum 2^(s - m) v; two such triples over
// different keys join with M = max(m, m'): O 2^(m - M) + O' 2^(m' - M).  A
// shared prefix and a sequence's own keys are two such parts, so the prefix is
// read for all the rows of the group together.
#include <algorithm>
#include <cooperative_groups.h>

#include "dm_attend.cuh"

namespace cg = cooperative_groups;

namespace dm {
namespace {

// -- the plan ----------------------------------------------------------------------

constexpr uint32_t kPlanCl = 8, kPlanT = 1024;

struct PlanArgs {
    PlanWork w;
    const int32_t *tables, *lengths, *seqs, *offsets, *group_offsets, *group_prefix;
    uint32_t *status;
    uint32_t n, groups, tokens, G, kv_heads, B, max_seqs, max_blocks, blocks[2];
};

__device__ __forceinline__ uint64_t scan_incl(uint64_t x) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint64_t y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
    }
    return x;
}

__device__ uint64_t block_scan(uint64_t x, uint64_t *s_warp, uint64_t &total) {
    const uint32_t wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t in = scan_incl(x);
    __syncthreads();
    if (lane == 31) s_warp[wid] = in;
    __syncthreads();
    if (wid == 0) s_warp[lane] = scan_incl(s_warp[lane]);
    __syncthreads();
    total = s_warp[kPlanT / 32 - 1];
    return in - x + (wid ? s_warp[wid - 1] : 0);
}

// The group of sequence i: the last g with group_offsets[g] <= i, -1 if i is
// outside them all or the group shares nothing.
__device__ __forceinline__ int32_t group_at(const PlanArgs &p, uint32_t i) {
    if (p.groups == 0 || (int32_t)i < p.group_offsets[0] || (int32_t)i >= p.group_offsets[p.groups]) return -1;
    uint32_t lo = 0, hi = p.groups;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (p.group_offsets[mid] <= (int32_t)i) lo = mid;
        else hi = mid;
    }
    return p.group_prefix[lo] > 0 ? (int32_t)lo : -1;
}

// CTA 0 lays the work out; the others see that a group's sequences begin with
// the same pages.
__global__ void __cluster_dims__(kPlanCl, 1, 1) __launch_bounds__(kPlanT) k_plan(PlanArgs p) {
    __shared__ uint64_t s_warp[32];
    __shared__ uint32_t s_bad;
    cg::cluster_group cl = cg::this_cluster();
    const uint32_t rank = cl.block_rank(), tid = threadIdx.x;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    bool bad = false;
    // every CTA: groups and sequences in range (the page check below relies on it)
    for (uint32_t g = tid; g < p.groups; g += kPlanT) {
        const int32_t a = p.group_offsets[g], b = p.group_offsets[g + 1], P = p.group_prefix[g];
        bad |= a < 0 || b < a || b > (int32_t)p.n || P < 0 || P % (int32_t)p.B || (uint32_t)P > p.max_blocks * p.B;
    }
    if (__syncthreads_or(bad)) s_bad = 1;
    if (!s_bad) {
        for (uint32_t i = tid; i < p.n; i += kPlanT) {
            const int32_t s = p.seqs[i], a = p.offsets[i], b = p.offsets[i + 1];
            if ((uint32_t)s >= p.max_seqs || a < 0 || b < a || b > (int32_t)p.tokens) {
                bad = true;
                continue;
            }
            const int64_t len = p.lengths[s], used = b - a;
            const int32_t g = group_at(p, i);
            bad |= len < 0 || len > (int64_t)p.max_blocks * p.B || (g >= 0 && used > 0 && p.group_prefix[g] > len - used);
        }
        // a group's prefix is read through its first sequence's row, so that
        // one's id has to be in range too (it is one of the n)
        if (__syncthreads_or(bad)) s_bad = 1;
    }
    __syncthreads();
    if (rank > 0 && !s_bad && p.groups) {   // a warp per sequence
        const uint32_t lane = tid & 31, warps = (kPlanCl - 1) * kPlanT / 32;
        for (uint32_t i = (rank - 1) * (kPlanT / 32) + tid / 32; i < p.n; i += warps) {
            const int32_t g = group_at(p, i);
            if (g < 0 || p.offsets[i + 1] == p.offsets[i]) continue;
            const int32_t *mine = p.tables + (uint64_t)p.seqs[i] * p.max_blocks;
            const int32_t *lead = p.tables + (uint64_t)p.seqs[p.group_offsets[g]] * p.max_blocks;
            const uint32_t nb = (uint32_t)p.group_prefix[g] / p.B;
#pragma unroll 4
            for (uint32_t j = lane; j < nb; j += 32) bad |= mine[j] != lead[j];
        }
        if (bad) s_bad = 1;
    }
    if (rank == 0 && !s_bad) {
        for (uint32_t g = tid; g < p.groups; g += kPlanT) p.w.group_max[g] = p.w.group_n[g] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < p.n; i += kPlanT) {
            const int32_t g = group_at(p, i);
            const uint32_t rows = (uint32_t)(p.offsets[i + 1] - p.offsets[i]) * p.G;
            if (g >= 0 && rows) {
                atomicMax(p.w.group_max + g, rows);
                atomicAdd(p.w.group_n + g, 1u);
            }
        }
        __syncthreads();
        auto shares = [&](int32_t g) { return g >= 0 && __ldcg(p.w.group_max + g) < kShareRows && __ldcg(p.w.group_n + g) >= 2; };
        auto rows_of = [&](uint32_t e) -> uint32_t {   // of an entity: groups, then sequences
            if (e < p.groups) {
                if (!shares(p.group_prefix[e] > 0 ? (int32_t)e : -1)) return 0;
                return (uint32_t)(p.offsets[p.group_offsets[e + 1]] - p.offsets[p.group_offsets[e]]) * p.G;
            }
            return (uint32_t)(p.offsets[e - p.groups + 1] - p.offsets[e - p.groups]) * p.G;
        };
        for (uint32_t i = tid; i < p.n; i += kPlanT) {
            const int32_t g = group_at(p, i);
            p.w.group_of[i] = shares(g) ? g : -1;
        }
        const uint32_t ents = p.groups + p.n;
        uint64_t carry = 0;   // wide blocks in the low half, narrow ones above
        for (uint32_t e0 = 0; e0 < ents; e0 += kPlanT) {
            const uint32_t e = e0 + tid, rows = e < ents ? rows_of(e) : 0;
            const uint64_t mine = rows == 0 ? 0 : rows <= kNarrowRows ? 1ull << 32 : (rows + kWideRows - 1) / kWideRows;
            uint64_t total;
            const uint64_t before = carry + block_scan(mine, s_warp, total);
            if (e < ents) {
                p.w.first[0][e] = (uint32_t)before;
                p.w.first[1][e] = (uint32_t)(before >> 32);
            }
            carry += total;
        }
        const uint32_t count[2] = {(uint32_t)carry, (uint32_t)(carry >> 32)};
        __syncthreads();
        for (int kind = 0; kind < 2; ++kind) {
            const uint32_t cap = kind == 0 ? kWideRows : kNarrowRows, keys = kind == 0 ? kWideKeys : kNarrowKeys;
            uint64_t units0 = 0, parts0 = 0;
            for (uint32_t b0 = 0; b0 < count[kind]; b0 += kPlanT) {
                const uint32_t b = b0 + tid;
                AttendBlock k{};
                if (b < count[kind]) {
                    uint32_t lo = 0, hi = ents;   // the last entity with first <= b; those without blocks come before it
                    while (hi - lo > 1) {
                        const uint32_t mid = (lo + hi) / 2;
                        if (__ldcg(p.w.first[kind] + mid) <= b) lo = mid;
                        else hi = mid;
                    }
                    const uint32_t e = lo, rows = rows_of(e);
                    const uint32_t row0 = (b - __ldcg(p.w.first[kind] + e)) * cap;
                    k.rows = min(rows - row0, cap);
                    k.lead = row0 % p.G;
                    if (e < p.groups) {
                        const int32_t i = p.group_offsets[e];
                        k.row = p.seqs[i];
                        k.token = p.offsets[i] + (int32_t)(row0 / p.G);
                        k.kv1 = p.group_prefix[e];
                        k.pos = 1 << 30;   // behind every key of the prefix
                        k.shared = 1;
                    } else {
                        const uint32_t i = e - p.groups;
                        const int32_t g = __ldcg(p.w.group_of + i), used = p.offsets[i + 1] - p.offsets[i];
                        k.row = p.seqs[i];
                        k.token = p.offsets[i] + (int32_t)(row0 / p.G);
                        k.shared = g >= 0;
                        k.kv0 = g >= 0 ? p.group_prefix[g] : 0;
                        k.pos = p.lengths[k.row] - used + (int32_t)(row0 / p.G);
                        k.kv1 = max(k.kv0, k.pos + (int32_t)((k.lead + k.rows - 1) / p.G) + 1);
                    }
                    k.units = max(1u, ((uint32_t)(k.kv1 - k.kv0) + keys - 1) / keys);
                }
                uint64_t units, parts;
                const uint64_t at = units0 + block_scan((uint64_t)k.units * p.kv_heads, s_warp, units);
                const uint64_t part = parts0 + block_scan(k.shared ? (uint64_t)k.rows * p.kv_heads : 0, s_warp, parts);
                if (b < count[kind]) {
                    k.part0 = (uint32_t)part;
                    p.w.block[kind][b] = k;
                    p.w.cum[kind][b] = at;
                }
                units0 += units;
                parts0 += parts;
            }
            if (tid == 0) {
                p.w.head->units[kind] = units0;
                p.w.head->blocks[kind] = count[kind];
            }
        }
    }
    cl.sync();
    if (rank == 0 && tid < 32) {
        const bool any = tid < kPlanCl && *cl.map_shared_rank(&s_bad, tid);
        const bool failed = __any_sync(~0u, any) || has_err(p.status);
        if (tid == 0) {
            p.w.head->ok = !failed;
            if (failed) set_err(p.status, DM_ERR_INVALID_ARG);
        }
    }
    cl.sync();
}

// -- few rows: up to 16 per key head ------------------------------------------------
//
// Memory's kernel: every key and value is used by at most 16 rows, so the
// tensor work is small and mma.sync's rate is enough; what counts is bytes in
// flight.  A producer warp keeps a ring of 32-key slots (keys and values, 8 KB
// or 16 KB) full through TMA, two CTAs per SM; each of four warps takes the 16
// keys of its half of every other slot, with its own running maximum and sum,
// and the four join once per tile.

constexpr uint32_t kSlotKeys = 32;

template <int D>
struct Narrow {
    static constexpr uint32_t kHalf = kSlotKeys * D * 2;            // bytes of a slot's keys, or values
    // Even, so that a ring place always belongs to the same pair of warps: a
    // pair that skipped a round could take the phase before it for its own.
    static constexpr uint32_t kSlots = D == 128 ? 4 : 8;
    static_assert(kSlots % 2 == 0, "each ring place has one pair of readers");
    static constexpr uint32_t kRed = kSlots * 2 * kHalf;            // 2 x 16 x D floats
    static constexpr uint32_t kMl = kRed + 2 * 16 * D * 4;          // 4 x 16 float2
    static constexpr uint32_t kBars = kMl + 4 * 16 * 8;             // full, empty per slot, then the give-up word
    static constexpr uint32_t kBytes = kBars + 16 * kSlots + 16 + 1024;   // with room to align
};

__device__ __forceinline__ void ldsm4(uint32_t *r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t *r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <class T, int D>
__global__ void __launch_bounds__(160, kNarrowPerSm)
    k_attend_narrow(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, AttendArgs p) {
    using N = Narrow<D>;
    extern __shared__ char s_raw[];
    char *s = reinterpret_cast<char *>(align_up(reinterpret_cast<uint64_t>(s_raw), 1024));
    const uint32_t s_at = smem_addr(s), bars = s_at + N::kBars;
    volatile uint32_t *gave_up = reinterpret_cast<uint32_t *>(s + N::kBars + 16 * N::kSlots);
    const uint32_t tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    auto full = [&](uint32_t slot) { return bars + 16 * slot; };
    auto empty = [&](uint32_t slot) { return bars + 16 * slot + 8; };
    if (tid == 0) {
        for (uint32_t i = 0; i < N::kSlots; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 2);   // two warps read a slot
        }
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (__syncthreads_or(has_err(p.status))) return;
    Walk<1> w(p);
    if (wid == 4) {
        uint32_t c = 0;   // slots so far
        KeyBoxes<D, kSlotKeys, 1> boxes(0);
        bool more = w.next(p);
        const int32_t *table = nullptr;
        uint32_t blocks = 0, tok = 0, left = 0, head = 0;   // the next slot; slots left of the piece
        auto piece = [&] {
            table = p.tables + (uint64_t)w.k.row * p.max_blocks;
            blocks = ((uint32_t)w.k.kv1 + (1u << p.B_log) - 1) >> p.B_log;
            tok = (uint32_t)w.k.kv0 + w.j0 * kNarrowKeys;
            left = 2 * w.units;
            head = w.head;
        };
        if (more) {
            piece();
            boxes.find(p, table, tok, blocks);
        }
        while (more) {
            const uint32_t slot = c % N::kSlots, round = c / N::kSlots, at = s_at + slot * 2 * N::kHalf;
            if (round) mbar_wait(empty(slot), (round - 1) & 1, gave_up, p.status);
            if (__any_sync(~0u, *gave_up)) break;
            if (lane == 0) mbar_expect(full(slot), 2 * N::kHalf);
            __syncwarp();
            boxes.load(p, &mk, at, full(slot), tok, head);
            boxes.load(p, &mv, at + N::kHalf, full(slot), tok, head);
            ++c;
            tok += kSlotKeys;
            if (--left == 0 && (more = w.next(p))) piece();
            if (more) boxes.find(p, table, tok, blocks);
        }
        // no copy may be in flight when the CTA ends
        for (uint32_t i = c > N::kSlots ? c - N::kSlots : 0; i < c; ++i)
            mbar_drain(full(i % N::kSlots), (i / N::kSlots) & 1);
        return;
    }
    float *red = reinterpret_cast<float *>(s + N::kRed);
    float2 *s_ml = reinterpret_cast<float2 *>(s + N::kMl);
    const uint32_t g = lane >> 2, t4 = lane & 3, pair = wid >> 1, key0 = (wid & 1) * 16;
    uint32_t c = 0;
    while (w.next(p)) {
        // this thread's rows are g and g + 8
        uint32_t qf[D / 16][4];
        int32_t limit[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint32_t row = g + 8 * r;
            const bool on = row < w.k.rows;
            const Row at = row_at(p, w.k, on ? row : 0);
            limit[r] = on ? row_limit(w.k, at.token) : 0;
            const char *src = p.q + (uint64_t)(w.k.token + at.token) * p.q_token + (uint64_t)(w.head * p.G + at.head) * p.q_head;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                qf[kk][r] = on ? __ldg(reinterpret_cast<const uint32_t *>(src + kk * 32 + t4 * 4)) : 0;
                qf[kk][r + 2] = on ? __ldg(reinterpret_cast<const uint32_t *>(src + kk * 32 + 16 + t4 * 4)) : 0;
            }
        }
        float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        for (uint32_t j = pair; j < 2 * w.units; j += 2) {
            const uint32_t slot = (c + j) % N::kSlots, round = (c + j) / N::kSlots, at = s_at + slot * 2 * N::kHalf;
            mbar_wait(full(slot), round & 1, gave_up, p.status);
            const int32_t first = w.k.kv0 + (int32_t)(w.j0 * kNarrowKeys + j * kSlotKeys + key0);
            if (first < w.k.kv1) {
                // scores: 16 rows x 16 keys
                float sc[2][4] = {};
                {
                    const uint32_t row = key0 + (lane & 7) + (lane >> 4) * 8, ch = (lane >> 3) & 1;
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t chunk = kk * 2 + ch, half = chunk >> 3;
                        uint32_t b[4];
                        ldsm4(b, at + half * kSlotKeys * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
                        Pack2<T>::mma(sc[0], qf[kk], b[0], b[1]);
                        Pack2<T>::mma(sc[1], qf[kk], b[2], b[3]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (first + i * 8 + (int32_t)t4 * 2 + (e & 1) >= limit[e >> 1]) sc[i][e] = -INFINITY;
                float mx[2], f[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    mx[r] = fmaxf(fmaxf(sc[0][2 * r], sc[0][2 * r + 1]), fmaxf(sc[1][2 * r], sc[1][2 * r + 1]));
                    mx[r] = fmaxf(mx[r], __shfl_xor_sync(~0u, mx[r], 1));
                    mx[r] = fmaxf(mx[r], __shfl_xor_sync(~0u, mx[r], 2));
                    const float now = fmaxf(m[r], mx[r] * p.scale2);
                    f[r] = now == -INFINITY ? 1.f : exp2_(m[r] - now);
                    m[r] = now;
                }
                if (__any_sync(~0u, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        o[i][0] *= f[0];
                        o[i][1] *= f[0];
                        o[i][2] *= f[1];
                        o[i][3] *= f[1];
                    }
                    l[0] *= f[0];
                    l[1] *= f[1];
                }
                const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[i][e] = exp2_(sc[i][e] * p.scale2 - base[e >> 1]);
                        l[e >> 1] += sc[i][e];
                    }
                // the weights in the cache's type, as the tensor cores take them
                const uint32_t a[4] = {Pack2<T>::pack(sc[0][0], sc[0][1]), Pack2<T>::pack(sc[0][2], sc[0][3]),
                                       Pack2<T>::pack(sc[1][0], sc[1][1]), Pack2<T>::pack(sc[1][2], sc[1][3])};
                const uint32_t row = key0 + (lane & 7) + ((lane >> 3) & 1) * 8, ch = lane >> 4;
                // values behind the end are whatever the page holds: a weight
                // of zero does not silence an infinity
                const int32_t left = w.k.kv1 - first;
                uint32_t keep0 = ~0u, keep1 = ~0u;
                if (left < 16) {
                    const int32_t k0 = (int32_t)t4 * 2;
                    keep0 = (k0 < left ? 0xFFFFu : 0u) | (k0 + 1 < left ? 0xFFFF0000u : 0u);
                    keep1 = (k0 + 8 < left ? 0xFFFFu : 0u) | (k0 + 9 < left ? 0xFFFF0000u : 0u);
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t chunk = i * 2 + ch, half = chunk >> 3;
                    uint32_t b[4];
                    ldsm4t(b, at + N::kHalf + half * kSlotKeys * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
                    Pack2<T>::mma(o[2 * i], a, b[0] & keep0, b[1] & keep1);
                    Pack2<T>::mma(o[2 * i + 1], a, b[2] & keep0, b[3] & keep1);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(slot));
        }
        c += 2 * w.units;
        // the four warps' parts: maxima and sums first, then the outputs in a fixed order
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(~0u, l[r], 1);
            l[r] += __shfl_xor_sync(~0u, l[r], 2);
            if (t4 == 0) s_ml[wid * 16 + g + 8 * r] = make_float2(m[r], l[r]);
        }
        bar_consumers();
        float M[2], L[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float2 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = s_ml[i * 16 + g + 8 * r];
            M[r] = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
            const float base = M[r] == -INFINITY ? 0.f : M[r];
            L[r] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) L[r] += x[i].y * exp2_(x[i].x - base);
            const float f = exp2_(m[r] - base);
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                o[i][2 * r] *= f;
                o[i][2 * r + 1] *= f;
            }
        }
        auto cell = [&](uint32_t part, int i, int r) { return reinterpret_cast<float2 *>(red + part * 16 * D + (g + 8 * r) * D + i * 8 + t4 * 2); };
        if (wid >= 2)
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) *cell(wid - 2, i, r) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
        bar_consumers();
        if (wid < 2)
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float2 x = *cell(wid, i, r);
                    o[i][2 * r] += x.x;
                    o[i][2 * r + 1] += x.y;
                    if (wid == 1) *cell(1, i, r) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
                }
        bar_consumers();
        if (wid == 0) {
            const bool whole = w.whole();
            const uint64_t part = whole ? 0 : w.part_row(p);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint32_t row = g + 8 * r;
                if (row >= w.k.rows) continue;
                const Row at = row_at(p, w.k, row);
                const uint64_t tok = (uint64_t)(w.k.token + at.token);
                const uint32_t h = w.head * p.G + at.head;
                if (whole) {
                    const float inv = L[r] > 0.f ? 1.f / L[r] : 0.f;
                    char *dst = p.o + tok * p.o_token + h * p.o_head;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const float2 x = *cell(1, i, r);
                        *reinterpret_cast<uint32_t *>(dst + i * 16 + t4 * 4) =
                            Pack2<T>::pack((o[i][2 * r] + x.x) * inv, (o[i][2 * r + 1] + x.y) * inv);
                    }
                    if (p.lse && t4 == 0) p.lse[tok * p.q_heads + h] = L[r] > 0.f ? (M[r] + log2f(L[r])) * 0.69314718056f : -INFINITY;
                } else {
                    float *dst = p.w.part[1] + (part + row) * D;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const float2 x = *cell(1, i, r);
                        *reinterpret_cast<float2 *>(dst + i * 8 + t4 * 2) = make_float2(o[i][2 * r] + x.x, o[i][2 * r + 1] + x.y);
                    }
                    if (t4 == 0) p.w.ml[1][part + row] = make_float2(M[r], L[r]);
                }
            }
        }
    }
}

// -- joining parts --------------------------------------------------------------------

// A warp per token and head: its parts from the group's prefix and from its
// own keys, in the order of the CTAs that left them.  A token whose only part
// went straight to the output has nothing to do.
template <class T, int D>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs p) {
    constexpr int V = D / 32;
    const uint64_t warp = (uint64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t tok = (uint32_t)(warp / p.q_heads), h = (uint32_t)(warp % p.q_heads);
    if (tok >= p.tokens || has_err(p.status) || !p.w.head->ok) return;
    if ((int32_t)tok < p.offsets[0] || (int32_t)tok >= p.offsets[p.n]) return;
    uint32_t i = 0, hi = p.n;
    while (hi - i > 1) {
        const uint32_t mid = (i + hi) / 2;
        if (p.offsets[mid] <= (int32_t)tok) i = mid;
        else hi = mid;
    }
    const int32_t g = p.w.group_of[i];
    const uint32_t kvh = h / p.G;
    float acc[V], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.f;
    // parts of entity e whose first query token is t0; false: it went straight out
    auto join = [&](uint32_t e, uint32_t t0, uint32_t rows_all) {
        const uint32_t row = (tok - t0) * p.G + h % p.G;
        const int kind = rows_all <= kNarrowRows;
        const uint32_t cap = kind ? kNarrowRows : kWideRows, b = p.w.first[kind][e] + row / cap, r = row % cap;
        const AttendBlock k = p.w.block[kind][b];
        const uint64_t u0 = p.w.cum[kind][b] + (uint64_t)kvh * k.units, U = p.w.head->units[kind];
        const uint32_t S = (uint32_t)min((uint64_t)p.ctas[kind], U);
        const uint32_t c0 = cta_of(u0, U, S), c1 = cta_of(u0 + k.units - 1, U, S);
        if (!k.shared && c0 == c1) return false;
        for (uint32_t c = c0; c <= c1; ++c) {
            const uint64_t at = k.shared ? k.part0 + (uint64_t)kvh * k.rows + (uint64_t)cap * c + r
                                         : p.w.shared_rows[kind] + (uint64_t)cap * (2 * c + (c == c0 ? 1 : 0)) + r;
            const float2 ml = p.w.ml[kind][at];
            const float *src = p.w.part[kind] + at * D + lane * V;
            float x[V];
            if constexpr (V == 4) *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(src);
            else *reinterpret_cast<float2 *>(x) = *reinterpret_cast<const float2 *>(src);
            const float now = fmaxf(M, ml.x), base = now == -INFINITY ? 0.f : now;
            const float f = exp2_(M - base), fx = exp2_(ml.x - base);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = acc[v] * f + x[v] * fx;
            L = L * f + ml.y * fx;
            M = now;
        }
        return true;
    };
    if (g >= 0) {
        const uint32_t a = (uint32_t)p.offsets[p.group_offsets[g]], b = (uint32_t)p.offsets[p.group_offsets[g + 1]];
        join((uint32_t)g, a, (b - a) * p.G);
    }
    const uint32_t t0 = (uint32_t)p.offsets[i];
    if (!join(p.groups + i, t0, ((uint32_t)p.offsets[i + 1] - t0) * p.G)) return;
    const float inv = L > 0.f ? 1.f / L : 0.f;
    char *dst = p.o + tok * p.o_token + h * p.o_head + lane * V * 2;
    if constexpr (V == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(Pack2<T>::pack(acc[0] * inv, acc[1] * inv), Pack2<T>::pack(acc[2] * inv, acc[3] * inv));
    else *reinterpret_cast<uint32_t *>(dst) = Pack2<T>::pack(acc[0] * inv, acc[1] * inv);
    if (p.lse && lane == 0) p.lse[(uint64_t)tok * p.q_heads + h] = L > 0.f ? (M + log2f(L)) * 0.69314718056f : -INFINITY;
}

// -- launches -----------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return EncodeTiled(nullptr);
        return reinterpret_cast<EncodeTiled>(fn);
    }();
    return f;
}

// A pool's pages of one layer as (dim, token, head, page); a box is 64 dims of
// `box` tokens.
bool page_map(CUtensorMap *m, const dm_cache *c, void *pool, uint32_t layer, uint32_t box) {
    const PageShape ps = page_shape(c);
    const cuuint64_t dims[4] = {c->head_dim, c->page_tokens, c->kv_heads, c->pages};
    const cuuint64_t strides[3] = {2ull * ps.token_step, 2ull * ps.head_step, 2ull * c->page_stride};
    const cuuint32_t boxes[4] = {64, box, 1, 1}, steps[4] = {1, 1, 1, 1};
    const EncodeTiled f = encode_tiled();
    return f && f(m, c->dtype == DM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                  static_cast<char *>(pool) + layer * c->layer_stride * 2, dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int D>
cudaError_t launch_rest(const AttendArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st) {
    static SmemOptIn opt;
    DM_TRY(opt_in_smem(opt, Narrow<D>::kBytes, k_attend_narrow<T, D>));
    k_attend_narrow<T, D><<<p.ctas[1], 160, Narrow<D>::kBytes, st>>>(mk, mv, p);
    DM_TRY(cudaGetLastError());
    const uint64_t warps = (uint64_t)p.tokens * p.q_heads;
    k_attend_join<T, D><<<(uint32_t)((warps + 7) / 8), 256, 0, st>>>(p);
    return cudaGetLastError();
}

uint32_t log2_of(uint32_t x) { return 31 - (uint32_t)__builtin_clz(x); }

bool plan_ok(const dm_cache *c, const dm_plan *p, PlanShape &s, PlanWork &w) {
    if (!cache_ok(c) || !p || !plan_shape(c, p->n, p->groups, p->tokens, p->q_heads, s)) return false;
    if ((p->n && (!p->seqs || !p->offsets)) || (p->groups && (!p->group_offsets || !p->group_prefix))) return false;
    return p->work && aligned(p->work, 256) && plan_work(s, p->work, w) <= p->work_bytes;
}

}  // namespace
}  // namespace dm

extern "C" uint64_t dm_plan_bytes(const dm_cache *c, uint32_t n, uint32_t groups, uint32_t tokens, uint32_t q_heads) {
    dm::PlanShape s;
    dm::PlanWork w;
    return dm::plan_shape(c, n, groups, tokens, q_heads, s) ? dm::plan_work(s, nullptr, w) : 0;
}

extern "C" dm_status dm_cache_plan(const dm_cache *c, const dm_plan *pl, void *stream) {
    using namespace dm;
    PlanShape s;
    PlanArgs p{};
    if (!plan_ok(c, pl, s, p.w)) return DM_ERR_INVALID_ARG;
    if (pl->n == 0 || pl->tokens == 0) return DM_OK;
    p.tables = c->tables, p.lengths = c->lengths, p.status = c->status;
    p.seqs = pl->seqs, p.offsets = pl->offsets, p.group_offsets = pl->group_offsets, p.group_prefix = pl->group_prefix;
    p.n = pl->n, p.groups = pl->groups, p.tokens = pl->tokens, p.G = s.G, p.kv_heads = c->kv_heads, p.B = c->page_tokens;
    p.max_seqs = c->max_seqs, p.max_blocks = c->max_blocks;
    k_plan<<<kPlanCl, kPlanT, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cudaGetLastError() == cudaSuccess ? DM_OK : DM_ERR_CUDA;
}

extern "C" dm_status dm_cache_attend(const dm_cache *c, const dm_plan *pl, const dm_attend_args *a, void *stream) {
    using namespace dm;
    PlanShape s;
    AttendArgs p{};
    if (!plan_ok(c, pl, s, p.w) || !a || a->layer >= c->layers) return DM_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !(a->scale <= 3.4e38f)) return DM_ERR_INVALID_ARG;
    if (pl->n == 0 || pl->tokens == 0) return DM_OK;
    if (!a->q || !a->o || !aligned(a->q, 16) || !aligned(a->o, 16) || !aligned(a->lse, 4)) return DM_ERR_INVALID_ARG;
    if ((a->q_token | a->q_head | a->o_token | a->o_head) % 8) return DM_ERR_INVALID_ARG;
    p.tables = c->tables, p.status = c->status;
    p.q = static_cast<const char *>(a->q), p.o = static_cast<char *>(a->o), p.lse = a->lse;
    p.q_token = a->q_token * 2, p.q_head = a->q_head * 2, p.o_token = a->o_token * 2, p.o_head = a->o_head * 2;
    const uint32_t box = std::min(c->page_tokens, kSlotKeys);
    p.max_blocks = c->max_blocks, p.pages = c->pages, p.B_log = log2_of(c->page_tokens), p.box_log = log2_of(box);
    p.G_mul = (uint32_t)((0xFFFFFFFFull + s.G) / s.G);   // 2^32 / G, rounded up
    p.G = s.G, p.kv_heads = c->kv_heads, p.q_heads = s.q_heads, p.scale2 = a->scale * 1.44269504089f;
    p.ctas[0] = s.ctas[0], p.ctas[1] = s.ctas[1];
    p.offsets = pl->offsets, p.group_offsets = pl->group_offsets;
    p.n = pl->n, p.groups = pl->groups, p.tokens = pl->tokens;
    if (((uint64_t)p.tokens * p.q_heads + 7) / 8 > 0x7FFFFFFFull) return DM_ERR_INVALID_ARG;
    CUtensorMap mk, mv;
    if (!page_map(&mk, c, c->k, a->layer, box) || !page_map(&mv, c, c->v, a->layer, box)) return DM_ERR_CUDA;
    const auto st = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_attend_wide(c, p, mk, mv, st);
    if (e == cudaSuccess) {
        if (c->dtype == DM_BF16)
            e = c->head_dim == 64 ? launch_rest<__nv_bfloat16, 64>(p, mk, mv, st) : launch_rest<__nv_bfloat16, 128>(p, mk, mv, st);
        else
            e = c->head_dim == 64 ? launch_rest<__half, 64>(p, mk, mv, st) : launch_rest<__half, 128>(p, mk, mv, st);
    }
    return e == cudaSuccess ? DM_OK : DM_ERR_CUDA;
}
