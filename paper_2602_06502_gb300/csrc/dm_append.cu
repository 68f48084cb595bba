// dm_append.cu -- new tokens enter an instance's prefix cache
// (dm_cache_append): each head's query and key is divided by its root mean
// square, weighted and rotated by its position; queries go to the caller's
// buffer, keys and values to their slots in the pages.
//
// One pass: a head's D values lie in D / 8 lanes, 16 bytes each, so the mean
// square is a few shuffles, and the partner of a value that turns is either in
// the same lane (pairs side by side) or a fixed number of lanes away.  All
// arithmetic is in 32 bits; the only rounding is the store.
//
// Bound: HBM bandwidth, 2 bytes read and 2 written per value (46,000 tokens of
// 48 heads, D = 128: 177 us, 6.4 TB/s); a few tokens alone, the latency of one
// launch (61 tokens: 5.6 us).
#include <algorithm>
#include <type_traits>

#include "dm_cache.cuh"

namespace dm {
namespace {

struct AppendArgs {
    const int32_t *seqs, *offsets, *tables, *lengths;
    uint32_t *status;
    int32_t *mark;            // per sequence: which of the call's named it last
    const uint4 *q, *k, *v;
    uint4 *q_out, *kc, *vc;   // kc, vc: this layer's pages
    uint64_t qt, qh, kt, kh, vt, vh, ot, oh, page_stride;   // 16-byte units
    uint32_t head_step, token_step;                         // within a page, 16-byte units
    const uint4 *qw, *kw;
    const float *cos, *sin;
    uint32_t n, tokens, q_heads, kv_heads, B, pages, max_seqs, max_blocks, rope_rows, rope_dim, per_warp;
    float eps;
};

template <class T>
struct Two;
template <>
struct Two<__nv_bfloat16> {
    using type = __nv_bfloat162;
    static __device__ float2 up(type x) { return __bfloat1622float2(x); }
    static __device__ type down(float a, float b) { return __floats2bfloat162_rn(a, b); }
};
template <>
struct Two<__half> {
    using type = __half2;
    static __device__ float2 up(type x) { return __half22float2(x); }
    static __device__ type down(float a, float b) { return __floats2half2_rn(a, b); }
};

template <class T>
__device__ __forceinline__ void unpack(uint4 x, float *f) {
    const auto *p = reinterpret_cast<const typename Two<T>::type *>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = Two<T>::up(p[i]);
        f[2 * i] = y.x;
        f[2 * i + 1] = y.y;
    }
}

template <class T>
__device__ __forceinline__ uint4 pack(const float *f) {
    uint4 x;
    auto *p = reinterpret_cast<typename Two<T>::type *>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = Two<T>::down(f[2 * i], f[2 * i + 1]);
    return x;
}

// A warp: per_warp heads of one token (its heads in the order queries, keys,
// values), 32 / (D / 8) of them at a time and kAhead such rounds in flight.  The
// first are loaded before the token's sequence is known.  Instructions are the
// next bound after HBM (3,600 a token of 48 heads in a form that chose between
// queries, keys and values head by head; 228 us at 46,000 tokens against 178
// so), hence a loop for each of the three.
constexpr uint32_t kAhead = 4, kThreads = 128;

template <class T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, 6) k_append(AppendArgs p) {
    constexpr uint32_t L = D / 8, H = 32 / L;
    const uint32_t lane = threadIdx.x & 31, l = lane % L, sub = lane / L;
    const uint32_t heads = p.q_heads + 2 * p.kv_heads, parts = (heads + p.per_warp - 1) / p.per_warp;
    const uint64_t warp = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const uint32_t t = (uint32_t)(warp / parts), h0 = (uint32_t)(warp % parts) * p.per_warp;
    pdl_enter();
    if (t >= p.tokens || has_err(p.status)) return;
    const uint32_t h1 = min(heads, h0 + p.per_warp), k0 = p.q_heads, v0 = k0 + p.kv_heads;
    uint4 raw[kAhead];
    // heads h .. end of a segment from here on, this lane's first being h + sub
    auto load = [&](const uint4 *src, uint64_t step, uint32_t h, uint32_t end) {
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
            if (h + u * H + sub < end) raw[u] = __ldcs(src + u * H * step);
    };
    const uint4 *src_q = p.q + t * p.qt + (h0 + sub) * p.qh + l;
    const uint32_t hk = max(h0, k0), hv = max(h0, v0);
    const uint4 *src_k = p.k + t * p.kt + (hk - k0 + sub) * p.kh + l, *src_v = p.v + t * p.vt + (hv - v0 + sub) * p.vh + l;
    if (h0 < k0) load(src_q, p.qh, h0, min(h1, k0));
    else if (h0 < v0) load(src_k, p.kh, h0, min(h1, v0));
    else load(src_v, p.vh, h0, h1);
    // the token's sequence: the last i with offsets[i] <= t
    const int32_t first = p.offsets[0], last = p.offsets[p.n];
    if (first < 0 || last < first || (uint32_t)last > p.tokens) {
        if (lane == 0) set_err(p.status, DM_ERR_INVALID_ARG);
        return;
    }
    if ((int32_t)t < first || (int32_t)t >= last) return;
    uint32_t lo = 0, hi = p.n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (p.offsets[mid] <= (int32_t)t) lo = mid;
        else hi = mid;
    }
    const int32_t s = p.seqs[lo], end = p.offsets[lo + 1];
    bool bad = (uint32_t)s >= p.max_seqs || end <= (int32_t)t || (uint32_t)end > p.tokens;
    const int64_t pos = bad ? 0 : (int64_t)p.lengths[s] - (end - (int32_t)t);
    bad = bad || pos < 0 || pos / p.B >= p.max_blocks || (p.rope_dim && pos >= p.rope_rows);
    const uint32_t page = bad ? 0 : (uint32_t)p.tables[(uint64_t)s * p.max_blocks + (uint32_t)pos / p.B];
    if (bad || page >= p.pages) {
        if (lane == 0) set_err(p.status, DM_ERR_INVALID_ARG);
        return;
    }
    // A sequence named twice would have two writers in its slots.  Of the two
    // that have tokens the later one here finds the other; a mark that an
    // earlier call left is checked against this call's sequences, so it says
    // nothing wrong.
    uint32_t named = lo;
    if (h0 == 0 && lane == 0 && (int32_t)t == p.offsets[lo]) named = (uint32_t)atomicExch(p.mark + s, (int32_t)lo);
    const uint64_t slot = page * p.page_stride + (uint32_t)pos % p.B * p.token_step;
    // this lane's cosines and sines: of its own values' frequencies
    constexpr int F = kInterleaved ? 4 : 8;
    float c[F], sn[F];
    const uint32_t e0 = l * 8, half = p.rope_dim / 2;
    const bool turns = e0 < p.rope_dim, low = e0 < half;
    if (turns) {
        const uint64_t at = (uint64_t)pos * half + (kInterleaved ? e0 / 2 : low ? e0 : e0 - half);
#pragma unroll
        for (int i = 0; i < F; i += 4) {
            *reinterpret_cast<float4 *>(c + i) = *reinterpret_cast<const float4 *>(p.cos + at + i);
            *reinterpret_cast<float4 *>(sn + i) = *reinterpret_cast<const float4 *>(p.sin + at + i);
        }
        if (!kInterleaved && low)   // a cos - b sin below, b cos + a sin above
#pragma unroll
            for (int i = 0; i < F; ++i) sn[i] = -sn[i];
    }
    if (named != lo && named < p.n && p.seqs[named] == s && p.offsets[named + 1] > p.offsets[named]) set_err(p.status, DM_ERR_INVALID_ARG);
    const uint32_t partner = sub * L + (low ? l + half / 8 : l - half / 8) % L;
    // heads h .. end: normed and rotated (kTurn) or as they are, loads ahead
    auto run = [&](auto turn, const uint4 *src, uint64_t step, uint4 *dst, uint64_t dst_step, uint32_t h, uint32_t end, const uint4 *weight,
                   bool loaded) {
        constexpr bool kTurn = decltype(turn)::value;
        if (h >= end) return;
        if (!loaded) load(src, step, h, end);
        float w[8];
        if (kTurn && weight) unpack<T>(weight[l], w);
        for (; h < end; h += H * kAhead) {
            uint4 now[kAhead];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) now[u] = raw[u];
            src += kAhead * H * step;
            load(src, step, h + H * kAhead, end);
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                if (h + u * H >= end) break;   // the whole warp
                uint4 y = now[u];
                if constexpr (kTurn) {
                    float x[8];
                    unpack<T>(y, x);
                    if (weight) {
                        float ss = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
                        for (uint32_t d = 1; d < L; d *= 2) ss += __shfl_xor_sync(~0u, ss, d);
                        const float r = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
                    }
                    if (kInterleaved) {
                        if (turns)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float a = x[2 * i], b = x[2 * i + 1];
                                x[2 * i] = a * c[i % F] - b * sn[i % F];
                                x[2 * i + 1] = b * c[i % F] + a * sn[i % F];
                            }
                    } else if (p.rope_dim) {
                        float z[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[i] = __shfl_sync(~0u, x[i], partner);
                        if (turns)
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i % F] + z[i] * sn[i % F];
                    }
                    y = pack<T>(x);
                }
                if (h + u * H + sub < end) __stcs(dst + u * H * dst_step, y);
            }
            dst += kAhead * H * dst_step;
        }
    };
    run(std::true_type{}, src_q, p.qh, p.q_out + t * p.ot + (h0 + sub) * p.oh + l, p.oh, h0, min(h1, k0), p.qw, true);
    run(std::true_type{}, src_k, p.kh, p.kc + slot + (uint64_t)(hk - k0 + sub) * p.head_step + l, p.head_step, hk, min(h1, v0), p.kw, h0 >= k0);
    run(std::false_type{}, src_v, p.vh, p.vc + slot + (uint64_t)(hv - v0 + sub) * p.head_step + l, p.head_step, hv, h1, nullptr, h0 >= v0);
}

template <class T, int D>
cudaError_t append_launch(const AppendArgs &p, bool interleaved, uint32_t grid, cudaStream_t st) {
    return launch_pdl(interleaved ? k_append<T, D, true> : k_append<T, D, false>, grid, kThreads, 0, st, p);
}

}  // namespace
}  // namespace dm

extern "C" dm_status dm_cache_append(const dm_cache *c, const dm_append_args *a, void *stream) {
    using namespace dm;
    if (!cache_ok(c) || !a || a->layer >= c->layers || a->tokens > 0x7FFFFFFFu) return DM_ERR_INVALID_ARG;
    if (a->q_heads % c->kv_heads || a->q_heads > 65535 * 32u || !(a->eps >= 0.f)) return DM_ERR_INVALID_ARG;
    if (a->rope_dim % 16 || a->rope_dim > c->head_dim || (a->rope_dim && (!a->cos || !a->sin || !a->rope_rows)))
        return DM_ERR_INVALID_ARG;
    if (a->n > c->max_seqs || a->interleaved > 1) return DM_ERR_INVALID_ARG;
    if (a->n == 0 || a->tokens == 0) return DM_OK;
    if (!a->seqs || !a->offsets || !a->k || !a->v || (a->q_heads && (!a->q || !a->q_out))) return DM_ERR_INVALID_ARG;
    for (const void *x : {a->q, a->k, a->v, (const void *)a->q_out, a->q_weight, a->k_weight, (const void *)a->cos,
                          (const void *)a->sin})
        if (!aligned(x, 16)) return DM_ERR_INVALID_ARG;
    if ((a->q_token | a->q_head | a->k_token | a->k_head | a->v_token | a->v_head | a->q_out_token | a->q_out_head) % 8)
        return DM_ERR_INVALID_ARG;
    const PageShape ps = page_shape(c);
    AppendArgs p{};
    p.seqs = a->seqs, p.offsets = a->offsets, p.tables = c->tables, p.lengths = c->lengths, p.status = c->status;
    p.mark = cache_work(c).mark;
    p.q = (const uint4 *)a->q, p.k = (const uint4 *)a->k, p.v = (const uint4 *)a->v, p.q_out = (uint4 *)a->q_out;
    p.kc = (uint4 *)c->k + a->layer * (c->layer_stride / 8);
    p.vc = (uint4 *)c->v + a->layer * (c->layer_stride / 8);
    p.qt = a->q_token / 8, p.qh = a->q_head / 8, p.kt = a->k_token / 8, p.kh = a->k_head / 8;
    p.vt = a->v_token / 8, p.vh = a->v_head / 8, p.ot = a->q_out_token / 8, p.oh = a->q_out_head / 8;
    p.page_stride = c->page_stride / 8, p.head_step = ps.head_step / 8, p.token_step = ps.token_step / 8;
    p.qw = (const uint4 *)a->q_weight, p.kw = (const uint4 *)a->k_weight, p.cos = a->cos, p.sin = a->sin;
    p.n = a->n, p.tokens = a->tokens, p.q_heads = a->q_heads, p.kv_heads = c->kv_heads, p.B = c->page_tokens;
    p.pages = c->pages, p.max_seqs = c->max_seqs, p.max_blocks = c->max_blocks;
    p.rope_rows = a->rope_rows, p.rope_dim = a->rope_dim, p.eps = a->eps;
    // heads of a token per warp: all of them, fewer while the warps would not
    // fill the SMs (48 heads of 64 tokens: 8 warps a token)
    const uint32_t heads = a->q_heads + 2 * c->kv_heads, once = 32 / (c->head_dim / 8);
    p.per_warp = (heads + once - 1) / once * once;
    const uint64_t enough = (uint64_t)sm_count() * 24;
    while (p.per_warp > once && (uint64_t)a->tokens * ((heads + p.per_warp - 1) / p.per_warp) < enough)
        p.per_warp = (p.per_warp / 2 + once - 1) / once * once;
    const uint64_t warps = (uint64_t)a->tokens * ((heads + p.per_warp - 1) / p.per_warp);
    constexpr uint32_t kWarps = kThreads / 32;
    if ((warps + kWarps - 1) / kWarps > 0x7FFFFFFFu) return DM_ERR_INVALID_ARG;
    const uint32_t grid = (uint32_t)((warps + kWarps - 1) / kWarps);
    const auto st = static_cast<cudaStream_t>(stream);
    const bool il = a->interleaved != 0;
    if (c->dtype == DM_BF16)
        return status_of(c->head_dim == 64 ? append_launch<__nv_bfloat16, 64>(p, il, grid, st)
                                           : append_launch<__nv_bfloat16, 128>(p, il, grid, st));
    return status_of(c->head_dim == 64 ? append_launch<__half, 64>(p, il, grid, st) : append_launch<__half, 128>(p, il, grid, st));
}
