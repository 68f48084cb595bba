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
#include <atomic>
#include <cooperative_groups.h>

#include "dm_attend.cuh"

namespace cg = cooperative_groups;

namespace dm {
namespace {

// -- the plan ----------------------------------------------------------------------

// 256 threads a CTA for a few sequences (10.7 -> 9.2 us for four; with 256
// sequences the page check needs them all).
constexpr uint32_t kPlanCl = 8, kPlanT = 1024, kPlanFew = 32;

struct PlanArgs {
    PlanWork w;
    const int32_t *tables, *lengths, *seqs, *offsets, *group_offsets, *group_prefix;
    uint32_t *status;
    uint32_t n, groups, tokens, G, kv_heads, B, max_seqs, max_blocks, key, ctas[2];
    PlanCosts costs;
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
    total = s_warp[blockDim.x / 32 - 1];
    return in - x + (wid ? s_warp[wid - 1] : 0);
}

// Measured with 256 single tokens of 64 heads behind 12 prefixes (D = 128), and
// with drafts of up to 8 tokens and 12 heads for 96 sequences (D = 64): the
// times of CTAs with units of one sort, in cycles / 100.  They share the SMs out
// between the kernels and even the CTAs' ends out; for prompts, whose units
// arithmetic bounds, they are the same.
constexpr PlanCosts kCosts128 = {23, 20, 75, 24, 8}, kCosts64 = {20, 17, 38, 15, 6};
constexpr uint32_t kFewGroups = 512, kFewBlocks = 2048;   // kept in shared memory

// The group of sequence i: the last g with offsets[g] <= i, -1 if i is outside
// them all or the group shares nothing.
__device__ __forceinline__ int32_t group_at(const int32_t *offsets, const int32_t *prefix, uint32_t groups, uint32_t i) {
    if (groups == 0 || (int32_t)i < offsets[0] || (int32_t)i >= offsets[groups]) return -1;
    uint32_t lo = 0, hi = groups;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (offsets[mid] <= (int32_t)i) lo = mid;
        else hi = mid;
    }
    return prefix[lo] > 0 ? (int32_t)lo : -1;
}

// CTA 0 lays the wide blocks out and CTA 1 the narrow ones (both work out the
// entities, writing the same); the others see that a group's sequences begin
// with the same pages.  Bound: latency, a chain of small steps, so what is
// searched is kept in shared memory.  9 us for four sequences, 13 to 16 for 96
// to 256 in five to twelve groups.
__global__ void __cluster_dims__(kPlanCl, 1, 1) __launch_bounds__(kPlanT) k_plan(PlanArgs p) {
    __shared__ uint64_t s_warp[32], s_cum[kFewBlocks];
    __shared__ int32_t s_offsets[kFewGroups + 1], s_prefix[kFewGroups];
    __shared__ uint32_t s_max[kFewGroups], s_n[kFewGroups];
    __shared__ uint32_t s_bad, s_cuts, s_rows;
    pdl_enter();
    cg::cluster_group cl = cg::this_cluster();
    const uint32_t rank = cl.block_rank(), tid = threadIdx.x, T = blockDim.x;
    const bool few = p.groups <= kFewGroups;
    const int32_t *go = few ? s_offsets : p.group_offsets, *gp = few ? s_prefix : p.group_prefix;
    uint32_t *gmax = few ? s_max : p.w.group_max + (rank & 1) * p.groups, *gn = few ? s_n : p.w.group_n + (rank & 1) * p.groups;
    __shared__ uint64_t s_sum[4];   // cost and units of each kind
    __shared__ uint32_t s_any;      // rank 0: some CTA found the step wrong
    __shared__ uint32_t s_stood;    // an earlier call's error
    if (tid < 4) s_sum[tid] = 0;
    if (tid == 0) s_bad = s_any = s_stood = has_err(p.status);
    if (few)
        for (uint32_t g = tid; p.groups && g <= p.groups; g += T) {
            s_offsets[g] = p.group_offsets[g];
            if (g < p.groups) s_prefix[g] = p.group_prefix[g];
        }
    if (rank < 2)
        for (uint32_t g = tid; g < p.groups; g += T) gmax[g] = gn[g] = 0;
    cl.sync();   // rank 0's s_any is set before another writes it
    bool bad = false;
    // every CTA: groups and sequences in range (the page check below relies on it)
    for (uint32_t g = tid; g < p.groups; g += T) {
        const int32_t a = go[g], b = go[g + 1], P = gp[g];
        bad |= a < 0 || b < a || b > (int32_t)p.n || P < 0 || P % (int32_t)p.B || (uint32_t)P > p.max_blocks * p.B;
    }
    if (__syncthreads_or(bad)) s_bad = 1;
    if (!s_bad) {
        for (uint32_t i = tid; i < p.n; i += T) {
            const int32_t s = p.seqs[i], a = p.offsets[i], b = p.offsets[i + 1];
            if ((uint32_t)s >= p.max_seqs || a < 0 || b < a || b > (int32_t)p.tokens) {
                bad = true;
                continue;
            }
            const int64_t len = p.lengths[s], used = b - a;
            const int32_t g = group_at(go, gp, p.groups, i);
            bad |= len < 0 || len > (int64_t)p.max_blocks * p.B || (g >= 0 && used > 0 && gp[g] > len - used);
            if (rank < 2 && g >= 0 && used) {
                atomicMax(gmax + g, (uint32_t)used * p.G);
                atomicAdd(gn + g, 1u);
            }
        }
        if (__syncthreads_or(bad)) s_bad = 1;
    }
    __syncthreads();
    if (rank > 1 && !s_bad && p.groups) {   // a warp per sequence, against its group's first
        const uint32_t lane = tid & 31, warps = (kPlanCl - 2) * T / 32;
        for (uint32_t i = (rank - 2) * (T / 32) + tid / 32; i < p.n; i += warps) {
            const int32_t g = group_at(go, gp, p.groups, i);
            if (g < 0 || p.offsets[i + 1] == p.offsets[i]) continue;
            const int32_t *mine = p.tables + (uint64_t)p.seqs[i] * p.max_blocks;
            const int32_t *lead = p.tables + (uint64_t)p.seqs[go[g]] * p.max_blocks;
            const uint32_t nb = (uint32_t)gp[g] / p.B;
#pragma unroll 8
            for (uint32_t j = lane; j < nb; j += 32) bad |= mine[j] != lead[j];
        }
        if (bad) s_bad = 1;
    }
    if (rank < 2 && !s_bad) {
        const uint32_t ents = p.groups + p.n;
        uint64_t carry = 0;   // wide blocks in the low half, narrow ones above
        for (uint32_t e0 = 0; e0 < ents; e0 += T) {
            const uint32_t e = e0 + tid;
            PlanEntity x{};
            if (e < ents) {
                const uint32_t i = e < p.groups ? (uint32_t)go[e] : e - p.groups;
                const int32_t g = e < p.groups ? (gp[e] > 0 ? (int32_t)e : -1) : group_at(go, gp, p.groups, i);
                const bool shares = g >= 0 && gmax[g] < kShareRows && gn[g] >= 2;
                x.group = shares ? g : -1;
                if (e >= p.groups || shares) {
                    const int32_t last = e < p.groups ? p.offsets[go[e + 1]] : p.offsets[i + 1];
                    x.row = p.seqs[i];
                    x.token = p.offsets[i];
                    x.rows = (uint32_t)(last - x.token) * p.G;
                    x.shared = e < p.groups ? kPrefix : shares ? kOwn : 0;
                    x.kv0 = e < p.groups || !shares ? 0 : gp[g];
                    x.pos = e < p.groups ? gp[e] - 1 : p.lengths[x.row] - (last - x.token);
                }
            }
            const uint64_t mine = x.rows == 0 ? 0 : x.rows <= kNarrowRows ? 1ull << 32 : (x.rows + kWideRows - 1) / kWideRows;
            uint64_t total;
            const uint64_t before = carry + block_scan(mine, s_warp, total);
            if (e < ents) {
                const int kind = x.rows <= kNarrowRows;
                x.first = (uint32_t)(kind ? before >> 32 : before);
                p.w.entity[e] = x;
                for (uint32_t j = 0; j < (uint32_t)(kind ? mine >> 32 : mine); ++j) p.w.owner[kind][x.first + j] = e;
            }
            carry += total;
        }
        const uint32_t count[2] = {(uint32_t)carry, (uint32_t)(carry >> 32)};
        __syncthreads();
        // block b of a kind, but for its place in the line and in the parts
        auto block_at = [&](int kind, uint32_t b) {
            const uint32_t cap = kind == 0 ? kWideRows : kNarrowRows, keys = kind == 0 ? kWideKeys : kNarrowKeys;
            AttendBlock k{};
            const uint32_t e = p.w.owner[kind][b];
            const PlanEntity x = p.w.entity[e];
            const uint32_t row0 = (b - x.first) * cap;
            k.row = x.row;
            k.rows = min(x.rows - row0, cap);
            k.lead = row0 % p.G;
            k.token = x.token + (int32_t)(row0 / p.G);
            k.kv0 = x.kv0;
            k.shared = x.shared;
            k.pos = x.pos + (x.shared == kPrefix ? 0 : (int32_t)(row0 / p.G));
            k.kv1 = x.shared == kPrefix ? gp[e] : max(k.kv0, k.pos + (int32_t)((k.lead + k.rows - 1) / p.G) + 1);
            k.units = max(1u, ((uint32_t)(k.kv1 - k.kv0) + keys - 1) / keys);
            k.cost = kind ? p.costs.narrow : k.rows > 128 ? p.costs.two : p.costs.one;
            k.over = kind ? p.costs.narrow_over : p.costs.wide_over;
            if (x.shared == kOwn) {
                const PlanEntity pre = p.w.entity[x.group];
                k.pre = pre.first;
                k.pre_kind = pre.rows <= kNarrowRows;
                k.pre_row = (uint32_t)(x.token - pre.token) * p.G + row0;
            }
            return k;
        };
        // What each kind costs, and its units.  A thread keeps the first block
        // that it lays out.
        const int kind = (int)rank;
        AttendBlock mine{};
        for (int kd = 0; kd < 2; ++kd) {
            uint64_t c = 0, u = 0;
            for (uint32_t b = tid; b < count[kd]; b += T) {
                const AttendBlock k = block_at(kd, b);
                if (kd == kind && b == tid) mine = k;
                c += (uint64_t)(k.units * (uint64_t)k.cost + k.over) * p.kv_heads;
                u += (uint64_t)k.units * p.kv_heads;
            }
            if (count[kd] > tid / 32 * 32) {   // the warp has some
                c = scan_incl(c);
                u = scan_incl(u);
                if ((tid & 31) == 31) {
                    atomicAdd(reinterpret_cast<unsigned long long *>(s_sum + 2 * kd), (unsigned long long)c);
                    atomicAdd(reinterpret_cast<unsigned long long *>(s_sum + 2 * kd + 1), (unsigned long long)u);
                }
            }
        }
        __syncthreads();
        const uint64_t cost[2] = {s_sum[0], s_sum[2]}, units[2] = {s_sum[1], s_sum[3]};
        // The SMs are shared out so that both kernels, which run side by side,
        // take about as long; kNarrowPerSm narrow CTAs share an SM.
        uint32_t sms = 0;
        if (units[0]) {
            const uint64_t wide = cost[0] * kNarrowPerSm, all = wide + cost[1];
            sms = (uint32_t)((wide * p.ctas[0] + all / 2) / all);
            sms = max(1u, min(sms, units[1] ? p.ctas[0] - 1 : p.ctas[0]));
        }
        PlanHead *h = p.w.head;
        const uint32_t mine_n = kind ? count[1] : count[0];
        const uint64_t mine_cost = kind ? cost[1] : cost[0], mine_units = kind ? units[1] : units[0];
        AttendBlock *block = kind ? p.w.block[1] : p.w.block[0];
        PlanStart *start = kind ? p.w.start[1] : p.w.start[0];
        uint64_t *all_cum = kind ? p.w.cum[1] : p.w.cum[0];
        if (mine_units == 0) {
            if (tid == 0) h->cost[kind] = h->inv[kind] = h->ctas[kind] = h->own[kind] = h->own_rows[kind] = h->cuts[kind] = 0;
        } else {
            // Each CTA has a unit where its share is not less than the widest
            // gap between two units' beginnings.  So little work that this
            // would leave CTAs idle goes a unit at a time.
            const uint32_t most = kind == 0 ? sms : (p.ctas[0] - sms) * kNarrowPerSm;
            const uint32_t gap = kind == 0 ? max(p.costs.two, p.costs.one) + p.costs.wide_over : p.costs.narrow + p.costs.narrow_over;
            const bool even = mine_cost / gap < most;
            const uint64_t C = even ? mine_units : mine_cost;
            const uint32_t S = (uint32_t)min((uint64_t)most, C);
            uint64_t *cum = mine_n <= kFewBlocks ? s_cum : all_cum;
            uint64_t at0 = 0, parts0 = 0;   // parts: rows below, blocks of their own from bit 40 on
            if (tid == 0) s_cuts = s_rows = 0;
            for (uint32_t b0 = 0; b0 < mine_n; b0 += T) {
                const uint32_t b = b0 + tid;
                AttendBlock k{};
                if (b < mine_n) {
                    k = b0 ? block_at(kind, b) : mine;
                    if (even) k.cost = 1, k.over = 0;
                }
                uint64_t length, parts;
                const uint64_t at = at0 + block_scan((uint64_t)(k.units * (uint64_t)k.cost + k.over) * p.kv_heads, s_warp, length);
                at0 += length;
                uint64_t part = 0;
                if (p.groups) {
                    part = parts0 + block_scan((k.shared ? (uint64_t)k.rows * p.kv_heads : 0) | (uint64_t)(k.shared == kOwn) << 40, s_warp, parts);
                    parts0 += parts;
                }
                if (b < mine_n) {
                    if (k.shared == kOwn) {
                        (kind ? p.w.own[1] : p.w.own[0])[part >> 40] = b;
                        atomicMax(&s_rows, k.rows);
                    }
                    k.part0 = (uint32_t)part;
                    block[b] = k;
                    all_cum[b] = at;
                    cum[b] = at;
                }
            }
            __syncthreads();
            for (uint32_t c = tid; c < S; c += T) {
                const uint64_t from = c * C / S;
                uint32_t lo = 0, hi = mine_n;   // the last block that begins by then
                while (hi - lo > 1) {
                    const uint32_t mid = (lo + hi) / 2;
                    if (cum[mid] <= from) lo = mid;
                    else hi = mid;
                }
                const AttendBlock k = block[lo];
                const uint64_t tile = (uint64_t)k.units * k.cost + k.over, inside = from - cum[lo];
                PlanStart x{0, lo, (uint32_t)(inside / tile), 0, 0};
                const uint64_t begin = cum[lo] + x.head * tile, rest = from - begin;   // of the tile; into it
                if (rest) x.unit = rest <= k.over + k.cost ? 1 : (uint32_t)((rest - k.over + k.cost - 1) / k.cost);
                x.at = begin + (x.unit ? k.over + (uint64_t)x.unit * k.cost : 0);
                if (x.unit == k.units) {   // the next tile
                    x.unit = 0;
                    if (++x.head == p.kv_heads) x.head = 0, ++x.block;
                }
                start[c] = x;
                // the first boundary inside a tile
                if (!k.shared && x.unit && (c - 1) * C / S <= begin) (kind ? p.w.cut[1] : p.w.cut[0])[atomicAdd(&s_cuts, 1u)] = c;
            }
            __syncthreads();
            if (tid == 0) {
                h->cost[kind] = C;
                h->inv[kind] = ~0ull / C;
                h->ctas[kind] = S;
                h->own[kind] = (uint32_t)(parts0 >> 40);
                h->own_rows[kind] = s_rows;
                h->cuts[kind] = s_cuts;
            }
        }
    }
    __syncthreads();
    if (tid == 0 && s_bad) *cl.map_shared_rank(&s_any, 0) = 1;
    cl.sync();
    const bool failed = rank == 0 ? s_any != 0 : s_bad != 0;
    if (rank == 0 && tid == 0) {
        // a step that was not looked at leaves no plan: once that error has been
        // read, attention on the buffer says so
        p.w.head->key = !failed ? p.key : s_stood ? 0 : kRefused;
        if (failed) set_err(p.status, DM_ERR_INVALID_ARG);
    }
    if (s_bad || !p.groups) return;
    // what joining needs of the shared groups' own blocks, all CTAs
    const uint32_t own0 = __ldcg(p.w.head->own), owns = own0 + __ldcg(p.w.head->own + 1);
    for (uint32_t i = tid * kPlanCl + rank; i < owns; i += kPlanCl * T) {
        const int kd = i >= own0;
        const uint32_t j = kd ? i - own0 : i, b = __ldcg((kd ? p.w.own[1] : p.w.own[0]) + j);
        JoinOwn x;
        auto side = [&](int from, uint32_t blk, uint32_t row) {
            const AttendBlock k = load_block(from ? p.w.block[1] : p.w.block[0], blk);
            return JoinSide{__ldcg((from ? p.w.cum[1] : p.w.cum[0]) + blk), k.units, k.cost, k.over, k.rows, k.part0, row};
        };
        const AttendBlock k = load_block(kd ? p.w.block[1] : p.w.block[0], b);
        const uint32_t cap = k.pre_kind ? kNarrowRows : kWideRows;
        x.own = side(kd, b, 0);
        x.pre_kind = k.pre_kind;
        x.pre_block = k.pre + k.pre_row / cap;
        x.pre = side((int)k.pre_kind, x.pre_block, k.pre_row % cap);
        x.token = k.token;
        x.lead = k.lead;
        (kd ? p.w.join[1] : p.w.join[0])[j] = x;
    }
}

// -- few rows: up to 16 per key head ------------------------------------------------
//
// Memory's kernel: every key and value is used by at most 16 rows, so the
// tensor work is small and mma.sync's rate is enough; what counts is bytes in
// flight.  Two warps keep a ring of 32-key slots (keys and values, 8 KB or 16 KB)
// full through TMA, two CTAs per SM; each of four warps takes the 16
// keys of its half of every other slot, with its own running maximum and sum,
// and the four join once per tile.  16 sequences of up to 100,000 keys of their
// own, two key heads, D = 128: 171 us at 6.1 TB/s from HBM, beside 153 us of the
// wide kernel's SMs.

constexpr uint32_t kSlotKeys = 32, kNarrowT = 192;

template <int D>
struct Narrow {
    static constexpr uint32_t kHalf = kSlotKeys * D * 2;            // bytes of a slot's keys, or values
    // Even, so that a ring place always belongs to the same pair of warps: a
    // pair that skipped a round could take the phase before it for its own.
    static constexpr uint32_t kSlots = D == 128 ? 4 : 8;
    static_assert(kSlots % 2 == 0, "each ring place has one pair of readers");
    static constexpr uint32_t kRow = D + 8;                         // floats, no two of a half warp's stores in one bank
    static constexpr uint32_t kRed = kSlots * 2 * kHalf;            // four warps' 8 rows
    static constexpr uint32_t kQ = kRed + 4 * 8 * kRow * 4;         // two pieces' queries, 16 rows each
    static constexpr uint32_t kMl = kQ + 2 * 16 * D * 2;            // 4 x 16 float2
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
__global__ void __launch_bounds__(kNarrowT, kNarrowPerSm)
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
    // After a wide kernel this one runs beside it: that one's CTAs have seen the
    // plan and everything before it complete before they let this one begin,
    // and this one ends after it, for what follows.  What the plan wrote is
    // therefore read through L2.
    if (p.beside) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    else pdl_enter();
    if (__syncthreads_or(has_err(p.status))) {
        if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    Walk<1> w(p);
    if (wid >= 4) {
        // one warp the keys, one the values
        const bool keys = wid == 4;
        uint32_t c = 0;   // slots so far
        for (Slots<1, D, kSlotKeys, 1> next(p, w, 0); next.more; next.step(p), ++c) {
            const uint32_t slot = c % N::kSlots, round = c / N::kSlots, at = s_at + slot * 2 * N::kHalf;
            if (round) mbar_wait(empty(slot), (round - 1) & 1, gave_up, p);
            if (__any_sync(~0u, *gave_up)) break;
            if (withheld(p, c)) continue;
            if (keys && lane == 0) mbar_expect(full(slot), 2 * N::kHalf);   // the phase ends with this and all the bytes
            __syncwarp();
            next.boxes.load(p, keys ? &mk : &mv, keys ? at : at + N::kHalf, full(slot), next.tok, next.head);
        }
        // no copy may be in flight when the CTA ends
        for (uint32_t i = c > N::kSlots ? c - N::kSlots : 0; i < c; ++i)
            mbar_drain(full(i % N::kSlots), (i / N::kSlots) & 1);
        if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    float *red = reinterpret_cast<float *>(s + N::kRed);
    float2 *s_ml = reinterpret_cast<float2 *>(s + N::kMl);
    const uint32_t g = lane >> 2, t4 = lane & 3, pair = wid >> 1, key0 = (wid & 1) * 16;
    uint32_t c = 0, buf = 0;
    // A piece's queries to shared memory, zeros for the rows that are not there.
    auto fetch = [&](const Walk<1> &k, uint32_t to) {
#pragma unroll
        for (uint32_t e = tid; e < 16 * D / 8; e += 128) {
            const uint32_t row = e / (D / 8), ch = e % (D / 8);
            const Row at = row_at(p, k.k, min(row, k.k.rows - 1));
            const char *src = p.q + (uint64_t)(k.k.token + at.token) * p.q_token + (uint64_t)(k.head * p.G + at.head) * p.q_head + ch * 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s_at + N::kQ + to * 32 * D + ch / 8 * 2048 + row * 128 + ((ch % 8) ^ (row % 8)) * 16),
                         "l"(src), "r"(row < k.k.rows ? 16 : 0)
                         : "memory");
        }
    };
    bool more = w.next(p);
    if (more) fetch(w, 0);
    while (more) {
        // this thread's rows are g and g + 8
        uint32_t qf[D / 16][4];
        int32_t limit[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint32_t row = g + 8 * r;
            limit[r] = row < w.k.rows ? row_limit(w.k, row_at(p, w.k, row).token) : 0;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        bar_consumers();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t row = lane & 15, chunk = kk * 2 + (lane >> 4);
            ldsm4(qf[kk], s_at + N::kQ + buf * 32 * D + (chunk >> 3) * 2048 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
        }
        Walk<1> ahead = w;
        float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        for (uint32_t j = pair; j < 2 * w.units; j += 2) {
            const uint32_t slot = (c + j) % N::kSlots, round = (c + j) / N::kSlots, at = s_at + slot * 2 * N::kHalf;
            mbar_wait(full(slot), round & 1, gave_up, p);
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
            if (j == pair && (more = ahead.next(p))) fetch(ahead, buf ^ 1);   // while the ring is full
        }
        c += 2 * w.units;
        buf ^= 1;
        // The four warps' parts, eight rows at a time: each warp leaves its
        // own, then adds up a quarter of the dims, in the order of the warps.
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(~0u, l[r], 1);
            l[r] += __shfl_xor_sync(~0u, l[r], 2);
            if (t4 == 0) s_ml[wid * 16 + g + 8 * r] = make_float2(m[r], l[r]);
        }
        const bool whole = w.whole();
        const uint64_t part = whole ? 0 : w.part_row(p);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (8u * r >= w.k.rows) break;
            if (r) bar_consumers();   // the first eight have been added up
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                *reinterpret_cast<float2 *>(red + (wid * 8 + g) * N::kRow + i * 8 + t4 * 2) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
            bar_consumers();
            constexpr uint32_t kMine = D / 16;   // dims of a thread
            const uint32_t row = 8 * r + g, col = wid * (D / 4) + t4 * kMine;
            float2 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = s_ml[i * 16 + row];
            const float M = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x)), base = M == -INFINITY ? 0.f : M;
            float L = 0.f, acc[kMine];
#pragma unroll
            for (uint32_t e = 0; e < kMine; ++e) acc[e] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = exp2_(x[i].x - base);
                L += x[i].y * f;
#pragma unroll
                for (uint32_t e = 0; e < kMine; e += 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(red + (i * 8 + g) * N::kRow + col + e);
                    acc[e] += y.x * f;
                    acc[e + 1] += y.y * f;
                    acc[e + 2] += y.z * f;
                    acc[e + 3] += y.w * f;
                }
            }
            if (row < w.k.rows) {
                if (whole) {
                    const Row at = row_at(p, w.k, row);
                    const uint64_t tok = (uint64_t)(w.k.token + at.token);
                    const uint32_t h = w.head * p.G + at.head;
                    const float inv = L == 0.f ? 0.f : 1.f / L;
                    char *dst = p.o + tok * p.o_token + h * p.o_head + col * 2;
#pragma unroll
                    for (uint32_t e = 0; e < kMine; e += 4)
                        *reinterpret_cast<uint2 *>(dst + e * 2) =
                            make_uint2(Pack2<T>::pack(acc[e] * inv, acc[e + 1] * inv), Pack2<T>::pack(acc[e + 2] * inv, acc[e + 3] * inv));
                    if (p.lse && wid == 0 && t4 == 0) p.lse[tok * p.q_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718056f;
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < kMine; e += 4)
                        *reinterpret_cast<float4 *>(p.w.part[1] + (part + row) * D + col + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
                    if (wid == 0 && t4 == 0) p.w.ml[1][part + row] = make_float2(M, L);
                }
            }
        }
        w = ahead;
    }
    if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// -- joining parts --------------------------------------------------------------------

// A warp takes kRows rows of a tile: of a shared group's sequence (their parts of
// the prefix, then those of its own keys) or of another tile that CTAs share,
// parts in the order of the CTAs that left them.  32 parts' maxima and sums are
// looked at together, so that the parts themselves are independent loads,
// kAhead of each row at once.  Bound: latency, then L2 (4 D + 8 bytes a row and
// part).  Finding a tile's parts takes a warp longer than adding a few up, so
// four rows go together once the GPU's warps all have four; with fewer rows
// more warps are worth more.  Where the GPU has a warp for each row anyway, one
// CTA an SM has 16 parts in flight (27 parts a row: 5.5 us with four).
template <class T, int D, uint32_t kRows, uint32_t kAhead, uint32_t kCtas>
__global__ void __launch_bounds__(256, kCtas) k_attend_join(AttendArgs p) {
    constexpr int V = D / 32;
    static_assert(kNarrowRows % kRows == 0 && kWideRows % kRows == 0);
    pdl_enter();
    const PlanHead h = *p.w.head;
    const uint32_t lane = threadIdx.x & 31;
    if (has_err(p.status)) return;
    if (h.key != p.key) {   // no plan, or one of another step's shape: the kernels before this one did nothing either
        if (h.key != kRefused && blockIdx.x == 0 && threadIdx.x == 0) set_err(p.status, DM_ERR_INVALID_ARG);
        return;
    }
    // A sequence's rows are taken in fours of its group's, none of which is in
    // two blocks of the prefix; where its first is not the first of a four, it
    // may need one more.
    const uint32_t more = p.G % kRows ? kRows - 1 : 0;
    const uint32_t fours[2] = {(h.own_rows[0] + more + kRows - 1) / kRows, (h.own_rows[1] + more + kRows - 1) / kRows};
    const uint64_t own1 = (uint64_t)h.own[1] * p.kv_heads * fours[1], own0 = own1 + (uint64_t)h.own[0] * p.kv_heads * fours[0];
    const uint64_t cut0 = own0 + (uint64_t)h.cuts[0] * (kWideRows / kRows), jobs = cut0 + (uint64_t)h.cuts[1] * (kNarrowRows / kRows);
    for (uint64_t t = blockIdx.x * 8ull + threadIdx.x / 32; t < jobs; t += gridDim.x * 8ull) {
        // a tile's parts: how many, and where its row 0 is in the i-th
        struct Parts {
            const float *part;
            const float2 *ml;
            uint32_t n, step, odd;   // a cut tile's first part is `odd` rows off
            uint64_t at;
            __device__ uint64_t row(uint32_t i) const { return at + (uint64_t)i * step + (i == 0 ? odd : 0); }
        };
        auto parts = [&](int kd, const JoinSide &x, uint32_t head, bool shared) {
            const uint64_t C = kd ? h.cost[1] : h.cost[0], begin = x.cum + head * ((uint64_t)x.units * x.cost + x.over);
            const uint64_t last = begin + (x.units > 1 ? x.over + (x.units - 1ull) * x.cost : 0);   // its last unit
            const uint32_t cap = kd ? kNarrowRows : kWideRows, S = kd ? h.ctas[1] : h.ctas[0];
            const uint64_t inv = kd ? h.inv[1] : h.inv[0];
            const uint32_t c0 = cta_of(begin, C, inv, S), c1 = cta_of(last, C, inv, S);
            Parts q{kd ? p.w.part[1] : p.w.part[0], kd ? p.w.ml[1] : p.w.ml[0], c1 - c0 + 1, cap, 0, 0};
            if (shared) {
                q.at = x.part0 + (uint64_t)head * x.rows + (uint64_t)cap * c0;
            } else {
                q.at = (kd ? p.w.shared_rows[1] : p.w.shared_rows[0]) + (uint64_t)cap * 2 * c0;
                q.step = 2 * cap;
                q.odd = cap;
            }
            return q;
        };
        uint32_t head, lead;
        int32_t token, r0, rows;   // the first row, of `rows`
        Parts pre{}, own;
        if (t < own0) {
            const int kind = t < own1;
            const uint64_t x = kind ? t : t - own1;
            const uint32_t per = kind ? fours[1] : fours[0], tile = (uint32_t)(x / per);
            head = tile % p.kv_heads;
            const JoinOwn &k = (kind ? p.w.join[1] : p.w.join[0])[tile / p.kv_heads];
            rows = (int32_t)k.own.rows;
            r0 = (int32_t)((uint32_t)(x % per) * kRows) - (int32_t)(k.pre.row % kRows);
            if (r0 >= rows) continue;
            token = k.token;
            lead = k.lead;
            own = parts(kind, k.own, head, true);
            JoinSide side = k.pre;
            int32_t at = (int32_t)side.row;   // of row 0 among the rows of the prefix's block
            const int32_t pre_cap = k.pre_kind ? kNarrowRows : kWideRows;
            if (at + max(r0, 0) >= pre_cap) {   // in the prefix's next block
                at -= pre_cap;
                const AttendBlock y = (k.pre_kind ? p.w.block[1] : p.w.block[0])[k.pre_block + 1];
                side = {(k.pre_kind ? p.w.cum[1] : p.w.cum[0])[k.pre_block + 1], y.units, y.cost, y.over, y.rows, y.part0, 0};
            }
            pre = parts((int)k.pre_kind, side, head, true);
            pre.at += at;   // row 0 may lie before the block; the rows taken do not
        } else {
            const int kind = t >= cut0;
            const uint64_t x = kind ? t - cut0 : t - own0;
            const uint32_t per = kind ? kNarrowRows / kRows : kWideRows / kRows;
            const PlanStart &from = (kind ? p.w.start[1] : p.w.start[0])[(kind ? p.w.cut[1] : p.w.cut[0])[x / per]];
            const AttendBlock y = (kind ? p.w.block[1] : p.w.block[0])[from.block];
            rows = (int32_t)y.rows;
            r0 = (int32_t)((uint32_t)(x % per) * kRows);
            if (r0 >= rows) continue;
            head = from.head;
            token = y.token;
            lead = y.lead;
            own = parts(kind, {(kind ? p.w.cum[1] : p.w.cum[0])[from.block], y.units, y.cost, y.over, y.rows, y.part0, 0}, head, false);
        }
        const uint32_t N = pre.n + own.n;
        const int32_t lo = max(r0, 0), hi = min(r0 + (int32_t)kRows, rows);
        float acc[kRows][V], M[kRows], L[kRows];
        uint32_t r[kRows];   // rows outside lo .. hi are read as the nearest inside
#pragma unroll
        for (uint32_t q = 0; q < kRows; ++q) {
            r[q] = (uint32_t)min(max(r0 + (int32_t)q, lo), hi - 1);
            M[q] = -INFINITY;
            L[q] = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) acc[q][v] = 0.f;
        }
        for (uint32_t i0 = 0; i0 < N; i0 += 32) {
            const uint32_t i = i0 + lane, n = min(N - i0, 32u);
            const float *mine = nullptr;   // row 0 of part i
            float2 ml[kRows];
#pragma unroll
            for (uint32_t q = 0; q < kRows; ++q) ml[q] = make_float2(-INFINITY, 0.f);
            if (i < N) {
                const bool first = i < pre.n;
                const uint64_t row = first ? pre.row(i) : own.row(i - pre.n);
                const float2 *src = (first ? pre.ml : own.ml) + row;
                mine = (first ? pre.part : own.part) + row * D;
#pragma unroll
                for (uint32_t q = 0; q < kRows; ++q) ml[q] = src[r[q]];
            }
            __syncwarp();
            float y[kAhead][kRows][V];
            auto load = [&](uint32_t j0) {
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    if (j0 + j >= n) break;
                    const float *src = reinterpret_cast<const float *>(__shfl_sync(~0u, reinterpret_cast<uint64_t>(mine), j0 + j)) + lane * V;
#pragma unroll
                    for (uint32_t q = 0; q < kRows; ++q) {
                        if constexpr (V == 4) *reinterpret_cast<float4 *>(y[j][q]) = *reinterpret_cast<const float4 *>(src + r[q] * D);
                        else *reinterpret_cast<float2 *>(y[j][q]) = *reinterpret_cast<const float2 *>(src + r[q] * D);
                    }
                }
            };
            load(0);
            float fi[kRows];
#pragma unroll
            for (uint32_t q = 0; q < kRows; ++q) {
                float now = ml[q].x;
#pragma unroll
                for (int d = 16; d; d /= 2) now = fmaxf(now, __shfl_xor_sync(~0u, now, d));
                now = fmaxf(now, M[q]);
                const float base = now == -INFINITY ? 0.f : now, f = exp2_(M[q] - base);
                fi[q] = exp2_(ml[q].x - base);
                float l = ml[q].y * fi[q];
#pragma unroll
                for (int d = 16; d; d /= 2) l += __shfl_xor_sync(~0u, l, d);
                L[q] = L[q] * f + l;
                M[q] = now;
#pragma unroll
                for (int v = 0; v < V; ++v) acc[q][v] *= f;
            }
            for (uint32_t j0 = 0; j0 < n; j0 += kAhead) {
                if (j0) load(j0);
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    if (j0 + j >= n) break;
#pragma unroll
                    for (uint32_t q = 0; q < kRows; ++q) {
                        const float fj = __shfl_sync(~0u, fi[q], j0 + j);
#pragma unroll
                        for (int v = 0; v < V; ++v) acc[q][v] += y[j][q][v] * fj;
                    }
                }
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < kRows; ++q) {
            if (r0 + (int32_t)q < lo || r0 + (int32_t)q >= hi) continue;
            const Row at = row_at(p, lead, r[q]);
            const uint64_t tok = (uint64_t)(token + at.token);
            const uint32_t qh = head * p.G + at.head;
            const float inv = L[q] == 0.f ? 0.f : 1.f / L[q];
            char *dst = p.o + tok * p.o_token + qh * p.o_head + lane * V * 2;
            if constexpr (V == 4)
                *reinterpret_cast<uint2 *>(dst) =
                    make_uint2(Pack2<T>::pack(acc[q][0] * inv, acc[q][1] * inv), Pack2<T>::pack(acc[q][2] * inv, acc[q][3] * inv));
            else *reinterpret_cast<uint32_t *>(dst) = Pack2<T>::pack(acc[q][0] * inv, acc[q][1] * inv);
            if (p.lse && lane == 0) p.lse[tok * p.q_heads + qh] = L[q] == 0.f ? -INFINITY : (M[q] + log2f(L[q])) * 0.69314718056f;
        }
    }
}

// -- launches -----------------------------------------------------------------------------

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
cudaError_t launch_rest(const AttendArgs &p, uint64_t q_rows, uint64_t rows, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st) {
    static SmemOptIn opt;
    DM_TRY(opt_in_smem(opt, Narrow<D>::kBytes, k_attend_narrow<T, D>));
    DM_TRY(launch_pdl(k_attend_narrow<T, D>, p.ctas[1], kNarrowT, Narrow<D>::kBytes, st, mk, mv, p));
    // Four rows a warp from 64 rows an SM on, about four for each warp that the
    // GPU then holds.  Attention of 256 tokens with 64 heads: 182 us one row at a
    // time, 178 by fours; 8,000 tokens of prompts with 32 heads: 584 and 573; two
    // layers of 128 tokens with 32 heads (27 rows an SM): 200 and 206.
    const bool four = q_rows >= p.ctas[0] * 64ull;
    const auto join = four ? k_attend_join<T, D, 4, 2, 2> : rows <= p.ctas[0] * 8ull ? k_attend_join<T, D, 1, 16, 1> : k_attend_join<T, D, 1, 4, 4>;
    // a warp per row or four, or twice as many as the GPU holds
    const uint64_t warps = std::min<uint64_t>(rows, p.ctas[0] * (four ? 32ull : 64ull));
    return launch_pdl(join, (uint32_t)((warps + 7) / 8), 256, 0, st, p);
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
    p.max_seqs = c->max_seqs, p.max_blocks = c->max_blocks, p.ctas[0] = s.ctas[0], p.ctas[1] = s.ctas[1], p.key = s.key;
    p.costs = c->head_dim == 128 ? kCosts128 : kCosts64;
    return status_of(launch_pdl(k_plan, kPlanCl, pl->n <= kPlanFew ? 256 : kPlanT, 0, static_cast<cudaStream_t>(stream), p));
}

#ifdef DM_DEBUG
static std::atomic<uint64_t> g_test_wait_ns{0};
#endif

extern "C" dm_status dm_test_attend_wait(uint64_t ns) {
#ifdef DM_DEBUG
    g_test_wait_ns = ns;
    return DM_OK;
#else
    return ns ? DM_ERR_INVALID_ARG : DM_OK;
#endif
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
    p.ctas[0] = s.ctas[0], p.ctas[1] = s.ctas[1], p.key = s.key;
    p.o_wide = aligned(a->o, 32) && (a->o_token | a->o_head) % 16 == 0;
    CUtensorMap mk, mv;
    if (!page_map(&mk, c, c->k, a->layer, box) || !page_map(&mv, c, c->v, a->layer, box)) return DM_ERR_CUDA;
#ifdef DM_DEBUG
    p.test_wait_ns = g_test_wait_ns;
#endif
    const auto st = static_cast<cudaStream_t>(stream);
    p.beside = (uint64_t)pl->tokens * s.G > kNarrowRows;   // else so few rows that no block of them is wide
    cudaError_t e = p.beside ? launch_attend_wide(c, p, mk, mv, st) : cudaSuccess;
    if (e == cudaSuccess) {
        // narrow tiles count 16 rows in the joining
        const uint64_t q_rows = (uint64_t)pl->tokens * s.q_heads, rows = q_rows + (uint64_t)pl->n * c->kv_heads * kNarrowRows;
        if (c->dtype == DM_BF16)
            e = c->head_dim == 64 ? launch_rest<__nv_bfloat16, 64>(p, q_rows, rows, mk, mv, st) : launch_rest<__nv_bfloat16, 128>(p, q_rows, rows, mk, mv, st);
        else
            e = c->head_dim == 64 ? launch_rest<__half, 64>(p, q_rows, rows, mk, mv, st) : launch_rest<__half, 128>(p, q_rows, rows, mk, mv, st);
    }
    return status_of(e);
}
