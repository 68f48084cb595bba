// dm_attend.cuh -- what the attention kernels over the paged cache share: the
// division of a step's work (dm_cache_plan), and how their parts are joined.
//
// Rows.  A query row is a token and one of the G = q_heads / kv_heads heads
// that read the same keys; a sequence's rows against one key head, or a whole
// group's against its shared prefix, go through the tensor cores together.
//
// Work.  A block is up to 256 rows (wide: the tcgen05 kernel) or up to 16
// (narrow) of one sequence or group and a range of keys; with a key head it is
// a tile, cut into units of 128 (wide) or 64 (narrow) keys.  All tiles of a
// kind stand in one line, each as long as it costs (`cost` a unit and `over`
// besides, which the first unit has), and CTA i of S takes the units that begin
// from i C / S to (i + 1) C / S of the line's length C.  S is small enough that
// each has some: every CTA is busy for about as long whatever the lengths.
// A tile that a boundary cuts, and every tile of a shared group, leaves
// (maximum, sum, unnormalised output) per row and CTA; k_attend_join adds them
// up.  A CTA and tile meet in one place of a staircase through (tiles x CTAs),
// so `first row + 256 CTA` (16 for narrow) is a place of its own for each.
#pragma once

#include <cuda.h>

#include "dm_cache.cuh"

namespace dm {

constexpr uint32_t kWideRows = 256, kWideKeys = 128, kNarrowRows = 16, kNarrowKeys = 64;
constexpr uint32_t kShareRows = 128;   // a sequence with as many rows fills a tile by itself
constexpr uint32_t kNarrowPerSm = 2;

// The plan's records are read and written 16 bytes at a time (a thread each: a
// word at a time is a line per lane and word).
struct alignas(16) AttendBlock {
    int32_t row;          // of tables
    int32_t token;        // query token of its first row
    uint32_t lead, rows;  // that row's head within G; its rows
    int32_t kv0, kv1;     // keys; no row sees one from kv1 on
    int32_t pos;          // the first token's position; a group's prefix, all of which all rows see: its last key
    uint32_t units;       // per key head, >= 1
    uint32_t cost, over;
    uint32_t part0;       // shared: its first row in the parts
    uint32_t shared;      // kPrefix, kOwn, or 0
    // kOwn: where the rows' parts of the prefix are, a block of kind pre_kind
    // and on, and the first row's place among the group's
    uint32_t pre, pre_kind, pre_row;
};
constexpr uint32_t kOwn = 1, kPrefix = 2;

struct PlanHead {
    uint64_t cost[2];     // wide, narrow
    uint64_t inv[2];      // 2^64 / cost
    uint32_t ctas[2];     // that have units
    uint32_t own[2];      // blocks of shared groups' sequences
    uint32_t own_rows[2]; // the most rows of one
    uint32_t cuts[2];     // other tiles that more than one CTA has part of
    uint32_t key, pad;    // the step's shape (PlanShape.key), kRefused, or 0: no plan
};

constexpr uint32_t kRefused = 2;   // PlanHead.key of a step that was found wrong

// A CTA's first unit.
struct alignas(16) PlanStart {
    uint64_t at;          // along the line
    uint32_t block, head, unit, pad;
};

// What the parts of a block cost, in 100 cycles of a CTA.
struct PlanCosts {
    uint32_t two, one, wide_over;     // a wide unit with two tiles of rows, with one; a wide tile besides
    uint32_t narrow, narrow_over;
};

// Where a block's parts are, and all that k_attend_join needs of a block of a
// shared group's sequence.
struct JoinSide {
    uint64_t cum;
    uint32_t units, cost, over, rows, part0, row;   // row: of the block's first row among that block's
};
struct alignas(16) JoinOwn {
    JoinSide own, pre;
    uint32_t pre_kind, pre_block;
    int32_t token;
    uint32_t lead;
};

// A sequence or a group of the step.
struct alignas(16) PlanEntity {
    int32_t row, token, group, kv0, pos;
    uint32_t rows, shared;
    uint32_t first;       // its first block of its kind
};

// The plan's work buffer.
struct PlanWork {
    PlanHead *head;
    AttendBlock *block[2];    // wide, narrow
    uint64_t *cum[2];         // where each block begins along the line
    PlanStart *start[2];      // per CTA
    uint32_t *owner[2];       // per block: its entity
    uint32_t *own[2];         // the blocks of shared groups' sequences
    JoinOwn *join[2];         // and what joining them needs
    uint32_t *cut[2];         // per other cut tile: the second CTA that has part of it
    PlanEntity *entity;       // groups, then sequences
    uint32_t *group_max, *group_n;   // most rows of a sequence; sequences with rows (two copies)
    float *part[2];           // rows x D
    float2 *ml[2];            // rows: maximum (base 2), sum
    uint64_t shared_rows[2];  // the parts' rows before the cut tiles' (two per CTA)
};

struct PlanShape {
    uint32_t n, groups, tokens, q_heads, G, D, sms;
    uint32_t ctas[2], blocks[2];
    uint64_t rows[2], shared_rows[2];
    uint32_t key;         // of the sizes that a plan holds for, odd
};

inline bool plan_shape(const dm_cache *c, uint32_t n, uint32_t groups, uint32_t tokens, uint32_t q_heads, PlanShape &s) {
    if (!cache_shape_ok(c) || q_heads == 0 || q_heads % c->kv_heads || q_heads > 65535u * 32) return false;
    if (n > c->max_seqs || groups > n || tokens > 0x7FFFFFFFu) return false;
    s.n = n, s.groups = groups, s.tokens = tokens, s.q_heads = q_heads;
    if (q_heads / c->kv_heads > 32768) return false;   // row_at's division
    s.G = q_heads / c->kv_heads, s.D = c->head_dim, s.sms = (uint32_t)sm_count();
    s.ctas[0] = s.sms, s.ctas[1] = s.sms * kNarrowPerSm;
    const uint32_t cap[2] = {kWideRows, kNarrowRows};
    // a sequence of a shared group has fewer than kShareRows rows, a narrow
    // one at most kNarrowRows; each of its rows has a part of the prefix and one of its own keys
    const uint32_t most[2] = {kShareRows - 1, kNarrowRows};
    for (int k = 0; k < 2; ++k) {
        const uint64_t t = std::min<uint64_t>(tokens, (uint64_t)n * (most[k] / s.G));
        s.shared_rows[k] = (groups ? 2 * t * q_heads : 0) + (uint64_t)cap[k] * s.ctas[k];
        s.rows[k] = s.shared_rows[k] + 2ull * cap[k] * s.ctas[k];
        if (s.rows[k] > 0xFFFFFFFFull) return false;
    }
    const uint64_t wide = (uint64_t)n + groups + 2 * ((uint64_t)tokens * s.G / kWideRows);
    if (wide > 0x7FFFFFFFull || (uint64_t)tokens * s.G > 0x7FFFFFFFull) return false;
    s.blocks[0] = (uint32_t)wide;
    s.blocks[1] = n + groups;
    s.key = 0;
    for (uint32_t x : {n, groups, tokens, q_heads, c->kv_heads, c->head_dim, c->page_tokens, c->max_seqs, c->max_blocks})
        s.key = (s.key ^ x) * 0x9E3779B1u, s.key ^= s.key >> 15;
    s.key |= 1;
    return true;
}

// Lays the buffer out from `base` (which may be null, for its size).
inline uint64_t plan_work(const PlanShape &s, void *base, PlanWork &w) {
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        char *p = static_cast<char *>(base) + at;
        at += align_up(bytes, 256);
        return p;
    };
    w.head = (PlanHead *)take(sizeof(PlanHead));
    for (int k = 0; k < 2; ++k) {
        w.block[k] = (AttendBlock *)take(sizeof(AttendBlock) * s.blocks[k]);
        w.cum[k] = (uint64_t *)take(8ull * s.blocks[k]);
        w.start[k] = (PlanStart *)take(sizeof(PlanStart) * s.ctas[k]);
        w.owner[k] = (uint32_t *)take(4ull * s.blocks[k]);
        w.own[k] = (uint32_t *)take(4ull * s.blocks[k]);
        w.join[k] = (JoinOwn *)take(s.groups ? sizeof(JoinOwn) * s.blocks[k] : 0);
        w.cut[k] = (uint32_t *)take(4ull * s.ctas[k]);
    }
    w.entity = (PlanEntity *)take(sizeof(PlanEntity) * (s.n + (uint64_t)s.groups));
    w.group_max = (uint32_t *)take(8ull * s.groups);
    w.group_n = (uint32_t *)take(8ull * s.groups);
    for (int k = 0; k < 2; ++k) {
        w.part[k] = (float *)take(4ull * s.D * s.rows[k]);
        w.ml[k] = (float2 *)take(8ull * s.rows[k]);
        w.shared_rows[k] = s.shared_rows[k];
    }
    return at;
}

struct AttendArgs {
    PlanWork w;
    const int32_t *tables;
    uint32_t *status;
    const char *q;
    char *o;
    float *lse;
    uint64_t q_token, q_head, o_token, o_head;   // bytes
    uint32_t max_blocks, pages, G, G_mul, kv_heads, q_heads;   // x / G = x * G_mul >> 32 for x <= G + 256
    uint32_t B_log, box_log;                     // log2 of a page's tokens and of a TMA box's
    float scale2;                                // scale * log2(e)
    uint32_t ctas[2];                            // launched
    uint32_t o_wide;                             // rows of o begin on 32 bytes
    uint32_t key;                                // the plan's
    uint32_t beside;                             // the narrow kernel runs beside a wide one
#ifdef DM_DEBUG
    uint64_t test_wait_ns;                       // dm_test_attend_wait: 0, or how long waits last
#endif
};

// Whether a test has slot c of this CTA's keys never arrive.
__device__ __forceinline__ bool withheld(const AttendArgs &p, uint32_t c) {
#ifdef DM_DEBUG
    return p.test_wait_ns && blockIdx.x == 0 && c == 0;
#else
    return false;
#endif
}

// The CTA of S whose units begin at `at` of a line of length C, the last i with
// i C / S <= at: ((at + 1) S - 1) / C.  inv = 2^64 / C rounded down gives that
// or one less ((at + 1) S <= C S < 2^64).
__device__ __forceinline__ uint32_t cta_of(uint64_t at, uint64_t C, uint64_t inv, uint32_t S) {
    const uint64_t x = (at + 1) * S - 1, i = __umul64hi(x, inv);
    return (uint32_t)(x - i * C >= C ? i + 1 : i);
}

// A block through L2: it may have been written by another CTA of this kernel, or
// before a kernel that this one runs beside.
__device__ __forceinline__ AttendBlock load_block(const AttendBlock *blocks, uint32_t b) {
    AttendBlock k;
    const uint4 *src = reinterpret_cast<const uint4 *>(blocks + b);
    uint4 *dst = reinterpret_cast<uint4 *>(&k);
#pragma unroll
    for (uint32_t i = 0; i < sizeof(AttendBlock) / 16; ++i) dst[i] = __ldcg(src + i);
    return k;
}

// Walks the tiles of a CTA's units.
template <int kKind>
struct Walk {
    uint64_t at, end;           // of the next unit along the line; of this CTA's share
    uint32_t b, next_head, next_unit;
    // of the present piece
    AttendBlock k;
    uint32_t head, j0, units;   // units j0 .. j0 + units of the tile
    bool in, out;               // another CTA has units before, behind

    __device__ Walk(const AttendArgs &p) {
        const PlanHead *h = p.w.head;
        const uint64_t C = __ldcg(&h->cost[kKind]);
        const uint32_t S = __ldcg(&h->key) == p.key ? __ldcg(&h->ctas[kKind]) : 0;
        at = end = 0;
        b = next_head = next_unit = 0;
        if (blockIdx.x < S) {
            const PlanStart *s = p.w.start[kKind] + blockIdx.x;
            at = __ldcg(&s->at);
            b = __ldcg(&s->block);
            next_head = __ldcg(&s->head);
            next_unit = __ldcg(&s->unit);
            end = (blockIdx.x + 1) * C / S;
        }
    }
    __device__ bool next(const AttendArgs &p) {
        if (at >= end) return false;
        k = load_block(p.w.block[kKind], b);
        head = next_head;
        j0 = next_unit;
        in = j0 > 0;
        // units of the tile that begin before `end`; the second begins `over` later
        const uint32_t over = in ? 0 : k.over, room = (uint32_t)min(end - at, (uint64_t)0x7FFFFFFF);
        units = room <= over + k.cost ? 1 : (room - over + k.cost - 1) / k.cost;
        units = min(units, k.units - j0);
        out = j0 + units < k.units;
        if (out) {
            at = end;
        } else {
            at += over + (uint64_t)units * k.cost;
            next_unit = 0;
            if (++next_head == p.kv_heads) {
                next_head = 0;
                ++b;
            }
        }
        return true;
    }
    // Whether the rows go straight to the output, and if not their first row
    // in the parts.
    __device__ bool whole() const { return !k.shared && !in && !out; }
    __device__ uint64_t part_row(const AttendArgs &p) const {
        constexpr uint32_t cap = kKind == 0 ? kWideRows : kNarrowRows;
        if (k.shared) return k.part0 + (uint64_t)head * k.rows + (uint64_t)cap * blockIdx.x;
        return p.w.shared_rows[kKind] + (uint64_t)cap * (2 * blockIdx.x + (in ? 0 : 1));
    }
};

// Row r of a block: its token, counted from the block's first, and its head.
struct Row {
    uint32_t token, head;
};
__device__ __forceinline__ Row row_at(const AttendArgs &p, uint32_t lead, uint32_t r) {
    const uint32_t x = lead + r, t = p.G == 1 ? x : __umulhi(x, p.G_mul);
    return {t, x - t * p.G};
}
__device__ __forceinline__ Row row_at(const AttendArgs &p, const AttendBlock &k, uint32_t r) { return row_at(p, k.lead, r); }
// One past the last key that a token of a block sees.
__device__ __forceinline__ int32_t row_limit(const AttendBlock &k, uint32_t token) {
    return min(k.kv1, k.pos + (int32_t)token + 1);
}

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ float exp2_(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// -- mbarriers and TMA ---------------------------------------------------------

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
constexpr uint32_t kWaits = 1u << 24;
constexpr uint64_t kWaitNs = 2'000'000'000;
// Waits for the phase, at most `ns` and kWaits tries.
__device__ __forceinline__ bool mbar_drain(uint32_t bar, uint32_t parity, const volatile uint32_t *gave_up = nullptr, uint64_t ns = kWaitNs) {
    if (mbar_try(bar, parity)) return true;
    const uint64_t t0 = now_ns();
    for (uint32_t i = 0; i < kWaits; ++i) {
        if (mbar_try(bar, parity)) return true;
        if (gave_up && *gave_up) return true;
        if ((i & 63) == 63 && now_ns() - t0 > ns) break;
    }
    return false;
}
// The same by a whole warp; a wait that gives up says so in `gave_up` (shared
// memory), and the CTA's others then return at once.  The caller goes on
// either way: every loop is as long as its data says, so the CTA ends.
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up, const AttendArgs &p) {
    uint64_t ns = kWaitNs;
#ifdef DM_DEBUG
    if (p.test_wait_ns) ns = p.test_wait_ns;
#endif
    if (!mbar_drain(bar, parity, gave_up, ns)) {
        *gave_up = 1;
        set_err(p.status, DM_ERR_TIMEOUT);
    }
    __syncwarp();
}

__device__ __forceinline__ void tma_load4(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}

// Key rows tok .. tok + keys of a sequence into shared memory, as D / 64 halves
// of 128-byte rows (128-byte swizzle): TMA boxes of up to a page, shared out to
// the lanes of kWarps warps (a warp issues its lanes' boxes one after another,
// about 55 cycles each).  A page that does not exist (a block from `blocks` on,
// an id out of range) reads as zeros.  find() loads the ids some time before
// load() needs them.
template <int D, int kKeys, uint32_t kWarps>
struct KeyBoxes {
    static constexpr uint32_t kHalves = D / 64;
    static constexpr uint32_t kEach = (kKeys / 4 * kHalves + 32 * kWarps - 1) / (32 * kWarps);   // a lane's, with 4-token pages
    uint32_t first, page[kEach];

    __device__ __forceinline__ explicit KeyBoxes(uint32_t warp) : first((threadIdx.x & 31) * kWarps + warp) {}

    __device__ __forceinline__ void find(const AttendArgs &p, const int32_t *table, uint32_t tok, uint32_t blocks) {
        const uint32_t boxes = kKeys * kHalves >> p.box_log;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t x = first + 32 * kWarps * i, blk = (tok + (x / kHalves << p.box_log)) >> p.B_log;
            page[i] = x < boxes && blk < blocks ? min((uint32_t)__ldcg(table + blk), p.pages) : p.pages;
        }
    }
    __device__ __forceinline__ void load(const AttendArgs &p, const CUtensorMap *map, uint32_t dst, uint32_t bar, uint32_t tok,
                                         uint32_t head) const {
        const uint32_t boxes = kKeys * kHalves >> p.box_log;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t x = first + 32 * kWarps * i, half = x % kHalves, at = x / kHalves << p.box_log;
            if (x < boxes)
                tma_load4(dst + half * kKeys * 128 + at * 128, map, bar, (int)half * 64, (int)((tok + at) & ((1u << p.B_log) - 1)),
                          (int)head, (int)page[i]);
        }
    }
};

// A CTA's key slots of kKeys, one after another over its pieces, and the pages
// of the next.
template <int kKind, int D, int kKeys, uint32_t kWarps>
struct Slots {
    static constexpr uint32_t kUnit = kKind == 0 ? kWideKeys : kNarrowKeys;
    Walk<kKind> w;
    KeyBoxes<D, kKeys, kWarps> boxes;
    const int32_t *table;
    uint32_t blocks, tok, left, head;   // left: of the piece
    bool more;

    __device__ __forceinline__ Slots(const AttendArgs &p, const Walk<kKind> &from, uint32_t warp) : w(from), boxes(warp) {
        left = 1;
        tok = 0;
        more = true;
        step(p);
    }
    __device__ __forceinline__ void step(const AttendArgs &p) {
        tok += kKeys;
        if (--left == 0) {
            more = w.next(p);
            if (!more) return;
            table = p.tables + (uint64_t)w.k.row * p.max_blocks;
            blocks = ((uint32_t)w.k.kv1 + (1u << p.B_log) - 1) >> p.B_log;
            tok = (uint32_t)w.k.kv0 + w.j0 * kUnit;
            left = w.units * (kUnit / kKeys);
            head = w.head;
        }
        boxes.find(p, table, tok, blocks);
    }
};

template <class T>
struct Pack2;
template <>
struct Pack2<__nv_bfloat16> {
    static constexpr uint32_t kMmaType = 1;   // of the tcgen05 instruction descriptor
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <>
struct Pack2<__half> {
    static constexpr uint32_t kMmaType = 0;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

cudaError_t launch_attend_wide(const dm_cache *c, const AttendArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st);

}  // namespace dm
