// dm_product.cuh -- what the product kernels share: their arguments, the
// checks of rows on the device, types and the epilogue.
//
// Rows.  Expert e's rows are offsets[e] .. offsets[e + 1]) of y; row r reads
// row sources[r] / per of x.  Channels are rows of the weights; a gated product
// has a gate's channel c and its partner n + c, n being y's channels.
//
// 8-bit values are whole numbers up to 128 in size, which f16 holds exactly, as
// its tensor products do: 8-bit products run at the f16 rate, with sums in 32
// bits (sm_103a's own 8-bit rate is far below that).
#pragma once

#include "dm_cache.cuh"

namespace dm {

struct ProductArgs {
    const char *w, *x;
    const float *w_scale, *x_scale;
    void *y;
    const int32_t *offsets, *sources;
    uint32_t *status;
    uint64_t w_row, w_expert, x_row;   // bytes
    uint64_t y_row;                    // elements
    uint32_t rows, x_rows, per, experts;
    uint32_t n, k;                     // channels of y; elements of a row of x
    uint32_t y_dtype, gated;
    uint32_t x_halves;                 // 8-bit: x holds halves, row r in row r; sources name the scales alone
                                       // (for the kernel for many rows)
    float eps;                         // of rows that the product quantises itself
    uint32_t most;                     // rows of an expert that the kernel for few rows has, the other has the rest; 0: one has all
};

// Expert e's rows [a, b); none, and an error, where the offsets are wrong.
struct Rows {
    int32_t a, b;
};
__device__ __forceinline__ Rows expert_rows(const ProductArgs &p, uint32_t e) {
    if (!p.offsets) return {0, (int32_t)p.rows};
    const int32_t a = __ldcg(p.offsets + e), b = __ldcg(p.offsets + e + 1);
    if (a < 0 || b < a || b > (int32_t)p.rows) {
        set_err(p.status, DM_ERR_INVALID_ARG);
        return {0, 0};
    }
    return {a, b};
}
// The row of x that row r reads; 0, and an error, where there is none.
__device__ __forceinline__ uint32_t source_row(const ProductArgs &p, uint32_t r) {
    if (p.sources) {
        const int32_t s = __ldcg(p.sources + r);
        r = s < 0 ? ~0u : (uint32_t)s / p.per;
    }
    if (r < p.x_rows) return r;
    set_err(p.status, DM_ERR_INVALID_ARG);
    return 0;
}

// Four bytes as four halves: 0x6400 + b is the half 1024 + b, and b is the
// signed byte + 128.
__device__ __forceinline__ void bytes_to_halves(uint32_t v, uint32_t &lo, uint32_t &hi) {
    v ^= 0x80808080u;
    const __half2 minus = __half2half2(__ushort_as_half(0x6480));   // 1152
    const uint32_t a = __byte_perm(v, 0x64646464u, 0x4140), b = __byte_perm(v, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), minus), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), minus);
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}

// In 32 bits.  The fast exponential is off by (2 + 1.2 |g|) 2^-23 of its size, and
// so is silu at most: for the sizes that matter far less than y's own rounding.
__device__ __forceinline__ float gate(float g, float u) { return g / (1.f + __expf(-g)) * u; }

__device__ __forceinline__ void store_y(const ProductArgs &p, uint64_t at, float v) {
    if (p.y_dtype == DM_BF16) static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(v);
    else if (p.y_dtype == DM_F16) static_cast<__half *>(p.y)[at] = __float2half_rn(v);
    else static_cast<float *>(p.y)[at] = v;
}

inline uint32_t dtype_size(uint32_t t) { return t == DM_I8 ? 1 : t == DM_F32 ? 4 : 2; }

inline bool status_ok(const uint32_t *status) { return status && aligned(status, 4); }

inline bool weights_ok(const dm_weights *w) {
    if (!w || !w->w || !aligned(w->w, 16) || w->dtype > DM_I8) return false;
    if (w->dtype == DM_I8 && (!w->scale || !aligned(w->scale, 4))) return false;
    if (w->experts < 1 || w->experts > 1024 || w->n < 1 || w->n > (1u << 24) || w->k < 1 || w->k > (1u << 24)) return false;
    const uint64_t step = 16 / dtype_size(w->dtype);
    if (w->row % step || w->row < w->k || w->row > (1ull << 32) || w->expert % step) return false;
    return w->experts == 1 || w->expert >= (w->n - 1) * w->row + w->k;
}

// How the kernel for many rows takes a product: tiles across the channels,
// parts of k and the stages they share out, and its work buffer: rows laid out
// for it, then the parts' sums.
struct WideShape {
    uint32_t blocks, splits, steps;
    uint64_t x_row, x_bytes, part_bytes;
};
// Where a product's rows are: as they came, named by sources, or halves of 8-bit values.
enum RowsAre { kPlain, kGathered, kHalves };
WideShape wide_shape(const dm_weights *w, uint32_t rows, uint32_t gated, RowsAre are);
uint64_t product_bytes(const dm_weights *w, uint32_t rows, uint32_t gated, RowsAre are);
bool takes_raw(const dm_weights *w, uint32_t rows);   // a projection quantises its rows within the product
cudaError_t launch_product_raw(const ProductArgs &p, uint32_t dtype, cudaStream_t st);
bool takes_halves(const dm_weights *w, uint32_t rows);   // 8-bit values as halves are worth having
// Where the rows of a layer's or a projection's product are: their quantising kernel
// writes halves where they are worth having, and bytes else.  What a product
// lays out in its work buffer follows from this, for its size and its launch.
inline RowsAre rows_are(const dm_weights *w, uint32_t rows, bool gathered) {
    return takes_halves(w, rows) ? kHalves : gathered ? kGathered : kPlain;
}
cudaError_t launch_product_wide(const dm_weights *w, const ProductArgs &p, const WideShape &s, void *work, cudaStream_t st);

// A product whose arguments are known to be right; a work buffer that is too small is refused.
cudaError_t launch_product(const dm_weights *w, const ProductArgs &p, void *work, uint64_t work_bytes, cudaStream_t st);
ProductArgs product_args(const dm_weights *w, const dm_product_args *a);

}  // namespace dm
