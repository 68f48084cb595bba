// dm_product.cu -- products of rows with 16-bit or 8-bit weights, of one
// expert or of many (dm_product), and the kernel for few rows.
#include <algorithm>

#include "dm_product.cuh"
#include "dm_quantize.cuh"

namespace dm {
namespace {

// -- few rows ---------------------------------------------------------------------
//
// The weights' bytes are all there is to it: each is read once from memory and
// used for at most 32 rows, so mma.sync's rate is enough and no weight goes
// through shared memory.  The product's sum may be taken in any order, as long
// as both operands agree on it: lane (g, t) of a warp loads 16 consecutive bytes
// of channel g (and g + 8), and of row g, and what the tensor cores take for
// their columns 2 t .. are the values that the lane has.  A warp's load is so 64
// consecutive bytes of eight rows.
//
// A CTA has 16 channels (gated: and their 16 partners); its eight warps share
// out k, 64 bytes at a time, and add their sums up in the order of the warps.
//
// Bound: memory.  One expert of 6,144 x 4,096, 8 rows, bf16: 10.3 us, 4.9 TB/s; 64
// of 2,048 x 2,048, 8 rows each: 88 us, 6.1 TB/s; in 8 bits, half the bytes, 7.3
// us, 3.4 TB/s, and 64 us, 4.2: a CTA's beginning and end weigh twice as much.
// (Sets of weights in turn, so they come from memory.)

constexpr uint32_t kFewT = 256, kFewWarps = 8;
constexpr int kFewShared = 35;   // percent of an SM's memory as shared memory

template <class T>
struct Few;   // T: of the weights and rows
template <>
struct Few<__nv_bfloat16> {
    static constexpr int kMmas = 2;
    static __device__ __forceinline__ void operand(const uint4 &x, int i, uint32_t &lo, uint32_t &hi) { lo = i ? x.z : x.x, hi = i ? x.w : x.y; }
    static __device__ __forceinline__ void mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <>
struct Few<__half> {
    static constexpr int kMmas = 2;
    static __device__ __forceinline__ void operand(const uint4 &x, int i, uint32_t &lo, uint32_t &hi) { lo = i ? x.z : x.x, hi = i ? x.w : x.y; }
    static __device__ __forceinline__ void mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <>
struct Few<int8_t> {
    static constexpr int kMmas = 4;
    static __device__ __forceinline__ void operand(const uint4 &x, int i, uint32_t &lo, uint32_t &hi) {
        bytes_to_halves(i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w, lo, hi);
    }
    static __device__ __forceinline__ void mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) { Few<__half>::mma(c, a, b0, b1); }
};

// 16 bytes.  In the order of the program: the compiler would else move a load
// down to its use, and the next would wait for it.
__device__ __forceinline__ uint4 load16(const char *p) {
    uint4 x;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}
__device__ __forceinline__ uint4 load16_kept(const char *p) {   // that other warps of the SM want too
    uint4 x;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}
// Zeros in the place of what lies `left` bytes and more from the first.
__device__ __forceinline__ void cut16(uint4 &x, int32_t left) {
    uint32_t *w = reinterpret_cast<uint32_t *>(&x);
#pragma unroll
    for (int32_t i = 0; i < 4; ++i) {
        const int32_t n = min(max(left - 4 * i, 0), 4);
        w[i] = n == 4 ? w[i] : w[i] & ((1u << 8 * n) - 1);
    }
}

// kTiles: 8-row tiles at a time; kM: 16-channel tiles (2: gated); kU: of a warp's
// steps of k, those whose loads are on their way together.  X: of the rows; a 16-bit
// type beside 8-bit weights: the CTA quantises them itself, a warp a row to look
// for its largest value, then each value on its way to the tensor cores.
template <class T, int kTiles, int kM, uint32_t kU, class X = T>
__global__ void __launch_bounds__(kFewT, kM * kTiles <= 2 ? 3 : 2) k_product_few(ProductArgs p) {
    constexpr uint32_t kCols = 16 * kM + 4;
    constexpr bool kRaw = !std::is_same_v<T, X>;
    constexpr uint32_t kWide = kRaw ? 2 : 1;   // 16-byte loads of a row for those of a channel
    static_assert(!kRaw || kTiles == 1);
    __shared__ float s_red[kFewWarps][8 * kTiles][kCols];
    __shared__ RowStep s_step[kRaw ? 8 : 1];
    __shared__ float s_scale[kRaw ? 8 : 1];
    pdl_enter();
    if (__syncthreads_or(has_err(p.status))) return;
    const uint32_t tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t e = blockIdx.y, c0 = blockIdx.x * 16;
    const Rows rows = expert_rows(p, e);
    if (p.most && (uint32_t)(rows.b - rows.a) > p.most) return;
    const uint32_t end = p.k * (uint32_t)sizeof(T), chunks = (end + 63) / 64, last = (end - 1) / 16 * 16;
    const uint32_t x_last = (end - 1) % 16 >= 8 ? 16 : 0;   // kRaw: from where a row's bytes for those of a channel begin, its last 16
    const char *w[kM][2];
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[m][h] = p.w + e * p.w_expert + (m * (uint64_t)p.n + min(c0 + g + 8 * h, p.n - 1)) * p.w_row;
    for (int32_t r0 = rows.a; r0 < rows.b; r0 += 8 * kTiles) {
        const char *x[kTiles];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) x[j] = p.x + source_row(p, (uint32_t)min(r0 + 8 * j + (int32_t)g, rows.b - 1)) * p.x_row;
        RowStep step;   // of row g
        if constexpr (kRaw) {
            const char *row = p.x + source_row(p, (uint32_t)min(r0 + (int32_t)wid, rows.b - 1)) * p.x_row;
            uint32_t tops = 0;
            float sum = 0.f;
            for (uint32_t at = lane * 16; at < 2 * p.k; at += 512) {
                uint4 v = load16_kept(row + at);
                cut16(v, (int32_t)(2 * p.k) - (int32_t)at);
                tops = larger2(larger2(larger2(larger2(tops, v.x), v.y), v.z), v.w);
                float f[8];
                unpack<X>(v, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += f[i] * f[i];
            }
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
            float scale;
            const uint32_t bits = __reduce_max_sync(~0u, max(tops & 0xFFFFu, tops >> 16));
            const RowStep mine = row_step<X>(bits, scale);
            if (p.eps >= 0.f && plain_squares<X>(bits)) {
                scale *= rsqrtf(sum / (float)p.k + p.eps);
            } else if (p.eps >= 0.f && far_squares<X>(bits)) {
                const float shift = far_shift(bits);
                sum = 0.f;
                for (uint32_t at = lane * 16; at < 2 * p.k; at += 512) {
                    uint4 v = load16_kept(row + at);
                    cut16(v, (int32_t)(2 * p.k) - (int32_t)at);
                    float f[8];
                    unpack<X>(v, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += f[i] * shift * (f[i] * shift);
                }
#pragma unroll
                for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
                scale = far_scale(bits, sum / (float)p.k, p.eps);
            }
            __syncthreads();   // the tile before has been read
            if (lane == 0) {
                s_step[wid] = mine;
                s_scale[wid] = scale;
            }
            __syncthreads();
            step = s_step[g];
        }
        float acc[kM][kTiles][4] = {};
        for (uint32_t c = wid; c < chunks; c += kFewWarps * kU) {
            uint4 wv[kU][kM][2], xv[kU][kTiles][kWide];
#pragma unroll
            for (uint32_t u = 0; u < kU; ++u) {
                const uint32_t at = min((c + kFewWarps * u) * 64 + t * 16, last);   // what is beyond the end becomes zero below
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) wv[u][m][h] = load16(w[m][h] + at);
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
#pragma unroll
                    for (uint32_t i = 0; i < kWide; ++i) xv[u][j][i] = load16_kept(x[j] + min(kWide * at + 16 * i, kWide * last + (kRaw ? x_last : 0)));
            }
            if ((c + kFewWarps * (kU - 1) + 1) * 64 > end) {
#pragma unroll
                for (uint32_t u = 0; u < kU; ++u) {
                    const int32_t left = (int32_t)end - (int32_t)((c + kFewWarps * u) * 64 + t * 16);
#pragma unroll
                    for (int m = 0; m < kM; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) cut16(wv[u][m][h], left);
#pragma unroll
                    for (int j = 0; j < kTiles; ++j)
#pragma unroll
                        for (uint32_t i = 0; i < kWide; ++i) cut16(xv[u][j][i], (int32_t)kWide * left - 16 * (int32_t)i);
                }
            }
#pragma unroll
            for (uint32_t u = 0; u < kU; ++u) {
                if constexpr (kRaw) {
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i) {
                        uint32_t n[8];
                        steps8<X>(xv[u][0][i], step, n);
                        xv[u][0][i] = halves8(n);
                    }
                }
#pragma unroll
                for (int i = 0; i < Few<T>::kMmas; ++i) {
                    uint32_t a[kM][4];
#pragma unroll
                    for (int m = 0; m < kM; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) Few<T>::operand(wv[u][m][h], i, a[m][h], a[m][2 + h]);
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) {
                        uint32_t b0, b1;
                        if constexpr (kRaw) Few<__half>::operand(xv[u][j][i / 2], i % 2, b0, b1);
                        else Few<T>::operand(xv[u][j][0], i, b0, b1);
#pragma unroll
                        for (int m = 0; m < kM; ++m) Few<T>::mma(acc[m][j], a[m], b0, b1);
                    }
                }
            }
        }
        __syncthreads();   // the sums before have been read
#pragma unroll
        for (int m = 0; m < kM; ++m)
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) s_red[wid][8 * j + 2 * t + (i & 1)][16 * m + g + 8 * (i >> 1)] = acc[m][j][i];
        __syncthreads();
        for (uint32_t i = tid; i < 8 * kTiles * 16; i += kFewT) {
            const uint32_t row = i / 16, ch = i % 16;
            const int32_t r = r0 + (int32_t)row;
            if (r >= rows.b || c0 + ch >= p.n) continue;
            float z[kM] = {};
#pragma unroll
            for (uint32_t q = 0; q < kFewWarps; ++q)
#pragma unroll
                for (int m = 0; m < kM; ++m) z[m] += s_red[q][row][16 * m + ch];
            if constexpr (sizeof(T) == 1) {
                const float sx = kRaw ? s_scale[row] : p.x_scale[source_row(p, (uint32_t)r)];
#pragma unroll
                for (int m = 0; m < kM; ++m) z[m] *= sx * p.w_scale[(uint64_t)e * kM * p.n + m * p.n + c0 + ch];
            }
            store_y(p, (uint64_t)r * p.y_row + c0 + ch, kM == 2 ? gate(z[0], z[kM - 1]) : z[0]);
        }
    }
}

// What is on its way lies in L1, which a kernel with much shared memory before
// this one would leave small: this one asks for its own division of the SM (64
// experts of 2,048 x 2,048, 8 rows each, behind k_product_wide: 158 us without).
template <class T, int kTiles, int kM, uint32_t kU, class X = T>
cudaError_t launch_few_one(const ProductArgs &p, cudaStream_t st) {
    static SmemOptIn asked;
    int dev = 0;
    DM_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kDevices) return cudaErrorInvalidDevice;
    const auto k = k_product_few<T, kTiles, kM, kU, X>;
    DM_TRY(static_cast<cudaError_t>(asked.raise(dev, 1, [&] { return (int)cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, kFewShared); })));
    return launch_pdl(k, dim3((p.n + 15) / 16, p.experts), kFewT, 0, st, p);
}

template <class T, int kTiles, uint32_t kU>
cudaError_t launch_few_tiles(const ProductArgs &p, cudaStream_t st) {
    return p.gated ? launch_few_one<T, kTiles, 2, kU>(p, st) : launch_few_one<T, kTiles, 1, kU>(p, st);
}

template <class T>
cudaError_t launch_few(const ProductArgs &p, cudaStream_t st) {
    const uint32_t each = (p.rows + p.experts - 1) / p.experts;
    if (each > 16) return launch_few_tiles<T, 4, 2>(p, st);
    if (each > 8) return launch_few_tiles<T, 2, 2>(p, st);
    // Two steps are all that a warp has of short rows (1,536 x 1,024 in 8 bits:
    // 3.4 us; with four, half of which are thrown away, 5.3), and as many as
    // registers hold of gated ones (eight experts' 4,096 x 1,024: 8.7 us, 9.9
    // with four); else four (6,144 x 4,096 in 8 bits: 7.7 us, 8.1 with two).
    if (p.gated || p.k * sizeof(T) <= 64 * kFewWarps * 2) return launch_few_tiles<T, 1, 2>(p, st);
    return launch_few_one<T, 1, 1, 4>(p, st);
}

}  // namespace

ProductArgs product_args(const dm_weights *w, const dm_product_args *a) {
    ProductArgs p{};
    const uint32_t size = dtype_size(w->dtype);
    p.w = static_cast<const char *>(w->w), p.w_scale = w->scale, p.w_row = w->row * size, p.w_expert = w->expert * size;
    p.experts = w->experts, p.k = w->k, p.n = a->gated ? w->n / 2 : w->n, p.gated = a->gated;
    p.x = static_cast<const char *>(a->x), p.x_scale = a->x_scale, p.x_row = a->x_row * size;
    p.y = a->y, p.y_row = a->y_row, p.y_dtype = a->y_dtype;
    p.offsets = a->offsets, p.sources = a->sources, p.per = a->per_source, p.status = a->status;
    p.rows = a->rows, p.x_rows = a->x_rows;
    return p;
}

// Which kernel has a product.  An expert's weights are read again for every 32
// rows by the one for few rows, and through more hands by the other.  With 64
// experts of 2,048 x 2,048 and 16 rows each 105 and 92 us (bf16), 77 and 78 (8
// bits), with 8 rows 88 and 90, 64 and 77; where some experts have many more
// rows than others, an average of 16 is 127 and 92, 95 and 78 us.  One of 6,144 x 4,096 with 16 rows 11.6
// and 14.7, 8.6 and 20, with 32 rows 20 and 15, 15 and 21 us; one of 1,536 x 1,024
// with 64 rows 7.0 and 8.1, 6.7 and 13.
// Where many experts have few rows on average, one may yet have hundreds, which
// the kernel for few rows takes eight at a time.  From kBothRows on the other
// kernel runs behind it, for experts with more than kMostFew.  The kernel for few
// rows alone, both, and the other alone (us; one expert has all rows; then each
// has as many): 2,048 rows of 256 experts of 2,048 x 2,048 410, 143, 25; 328, 332,
// 326 in bf16, 320, 141, 39; 238, 248, 252 in 8 bits; 2,048 rows of 64 experts
// of 512 x 512 83, 22, 14; 21, 24, 12, and 150, 25, 18; 30, 36, 17.  So both cost 3 to 10 us
// where no expert has many rows (14 where 8-bit rows are named by sources) and
// save much where one does; the other alone would save more in most of this range.
// Up to kBothRows one expert may have them all: 512 rows of 64 of 2,048 x 2,048,
// bf16, are 129 us then, 90 where they are even.
constexpr uint32_t kMostFew = 64, kBothRows = 1024;
enum Kernels { kFew, kBoth, kWide };
static Kernels kernels_of(const dm_weights *w, uint32_t rows) {
    const uint64_t bytes = (uint64_t)w->experts * w->n * w->k * dtype_size(w->dtype);
    const uint64_t most = bytes <= (4u << 20) ? 64 : bytes <= (32u << 20) ? 32 : w->experts == 1 ? 16 : 8;
    if (rows > w->experts * most) return kWide;
    return w->experts > 1 && rows > kBothRows ? kBoth : kFew;
}

// One launch and no work buffer: 4 rows of 1,536 x 1,024 take 13.3 us of the host
// for 18, and 5.2 of the GPU for 4.4.  Each CTA quantises all rows again, so only
// where the weights are few.
bool takes_raw(const dm_weights *w, uint32_t rows) {
    return w->dtype == DM_I8 && w->experts == 1 && rows <= 8 && (uint64_t)w->n * w->k <= (4u << 20);
}

cudaError_t launch_product_raw(const ProductArgs &p, uint32_t dtype, cudaStream_t st) {
    return dtype == DM_BF16 ? launch_few_one<int8_t, 1, 1, 2, __nv_bfloat16>(p, st) : launch_few_one<int8_t, 1, 1, 2, __half>(p, st);
}

bool takes_halves(const dm_weights *w, uint32_t rows) { return w->dtype == DM_I8 && kernels_of(w, rows) == kWide; }

uint64_t product_bytes(const dm_weights *w, uint32_t rows, uint32_t gated, RowsAre are) {
    if (kernels_of(w, rows) == kFew) return 1;
    const WideShape s = wide_shape(w, rows, gated, are);
    return std::max<uint64_t>(s.x_bytes + s.part_bytes, 1);
}

cudaError_t launch_product(const dm_weights *w, const ProductArgs &from, void *work, uint64_t work_bytes, cudaStream_t st) {
    ProductArgs p = from;
    const Kernels k = kernels_of(w, p.rows);
    WideShape s{};
    if (k != kFew) s = wide_shape(w, p.rows, p.gated, p.x_halves ? kHalves : p.sources ? kGathered : kPlain);
    if (s.x_bytes + s.part_bytes > work_bytes) return cudaErrorInvalidValue;
    p.most = k == kBoth ? kMostFew : 0;
    const auto few = w->dtype == DM_BF16 ? launch_few<__nv_bfloat16> : w->dtype == DM_F16 ? launch_few<__half> : launch_few<int8_t>;
    if (k != kWide) DM_TRY(few(p, st));
    if (k == kFew) return cudaSuccess;
    return launch_product_wide(w, p, s, work, st);
}

}  // namespace dm

extern "C" uint64_t dm_product_bytes(const dm_weights *w, uint32_t rows, uint32_t gated, uint32_t gathered) {
    using namespace dm;
    if (!weights_ok(w) || rows > 0x7FFFFFFFu || gated > 1 || gathered > 1 || (gated && w->n % 2)) return 0;
    return product_bytes(w, rows, gated, gathered ? kGathered : kPlain);
}

extern "C" dm_status dm_product(const dm_weights *w, const dm_product_args *a, void *stream) {
    using namespace dm;
    if (!a) return DM_ERR_INVALID_ARG;
    const uint64_t need = dm_product_bytes(w, a->rows, a->gated, a->sources != nullptr);
    if (!need || a->reserved0 || !status_ok(a->status)) return DM_ERR_INVALID_ARG;
    if (need > 1 && (a->work_bytes < need || !a->work || !aligned(a->work, 256))) return DM_ERR_INVALID_ARG;
    const uint32_t size = dtype_size(w->dtype), n = a->gated ? w->n / 2 : w->n;
    if (a->y_dtype > DM_F32 || a->y_dtype == DM_I8 || a->x_rows > 0x7FFFFFFFu) return DM_ERR_INVALID_ARG;
    if (!a->offsets && w->experts != 1) return DM_ERR_INVALID_ARG;
    if (a->sources ? a->per_source < 1 : a->x_rows < a->rows) return DM_ERR_INVALID_ARG;
    if (a->rows == 0) return DM_OK;
    if (a->x_rows == 0 || !a->x || !a->y || !aligned(a->x, 16) || !aligned(a->y, dtype_size(a->y_dtype))) return DM_ERR_INVALID_ARG;
    if (a->x_row * size % 16 || a->x_row > (1ull << 32) || (a->x_rows > 1 && a->x_row < w->k)) return DM_ERR_INVALID_ARG;
    if (a->y_row > (1ull << 32) || (a->rows > 1 && a->y_row < n)) return DM_ERR_INVALID_ARG;
    if (w->dtype == DM_I8 && (!a->x_scale || !aligned(a->x_scale, 4))) return DM_ERR_INVALID_ARG;
    if (!aligned(a->offsets, 4) || !aligned(a->sources, 4)) return DM_ERR_INVALID_ARG;
    return status_of(launch_product(w, product_args(w, a), a->work, a->work ? a->work_bytes : 0, static_cast<cudaStream_t>(stream)));
}
