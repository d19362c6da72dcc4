// Declarations shared by the layers' translation units: arguments of the matrix product, its epilogue, activations.
#pragma once
#include <atomic>
#include <type_traits>
#include "fc_dma_util.hpp"
#include "focused_layers.h"

namespace fc {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

// The exponential and the reciprocal are the hardware's, good to a unit of the last place: 2^-20 of the argument is what the activations are off by at most,
// below half a step of the 16-bit types by far.  (With expf, erff and the exact division they were a third of a large group norm's time, 149 of 252 us.)
// erfc(z) for z >= 0 is formula 7.1.26 of Abramowitz and Stegun, 1.5e-7 off at most; the side of zero is taken by the sign, so nothing cancels.
template <int ACT> __device__ __forceinline__ float activate(float y)
{
    if constexpr (ACT == FC_ACT_RELU) return relu_keep_nan(y);
    if constexpr (ACT == FC_ACT_SILU) return y * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * -1.44269504088896f));
    if constexpr (ACT == FC_ACT_GELU) {
        const float z = fabsf(y) * 0.707106781186547524f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
        float p = fmaf(1.061405429f, t, -1.453152027f);
        p = fmaf(p, t, 1.421413741f);
        p = fmaf(p, t, -0.284496736f);
        p = fmaf(p, t, 0.254829592f);
        const float half = 0.5f * (p * t) * __builtin_amdgcn_exp2f(z * z * -1.44269504088896f);    // erfc(z) / 2
        return y * (y < 0.f ? half : 1.f - half);
    }
    return y;
}
__device__ __forceinline__ float activate(float y, int act)
{
    switch (act) {
    case FC_ACT_RELU: return activate<FC_ACT_RELU>(y);
    case FC_ACT_SILU: return activate<FC_ACT_SILU>(y);
    case FC_ACT_GELU: return activate<FC_ACT_GELU>(y);
    default: return y;
    }
}
// N values at once: one branch, then the values' arithmetic side by side.
template <int N> __device__ __forceinline__ void activate_all(float (&v)[N], int act)
{
    if (act == FC_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<FC_ACT_RELU>(v[i]);
    } else if (act == FC_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<FC_ACT_SILU>(v[i]);
    } else if (act == FC_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<FC_ACT_GELU>(v[i]);
    }
}

// The carrier of a storage type.
template <int DT> struct CarrierOf { typedef float type; };
template <> struct CarrierOf<FC_BF16> { typedef bf16_t type; };
template <> struct CarrierOf<FC_F16> { typedef f16_t type; };

// Eight values next to each other (16 or 32 bytes, aligned so) and the way back with one rounding.
__device__ __forceinline__ void load8_float(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
template <typename T> __device__ __forceinline__ void unpack8(const uint4 &x, float (&v)[8])
{
    static_assert(sizeof(T) == 2, "16-bit values");
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = to_float(T{(uint16_t)w[i]});
        v[2 * i + 1] = to_float(T{(uint16_t)(w[i] >> 16)});
    }
}
template <typename T> __device__ __forceinline__ void load8_float(const T *p, float (&v)[8]) { unpack8<T>(*reinterpret_cast<const uint4 *>(p), v); }
__device__ __forceinline__ uint32_t pack2_of(bf16_t, float a, float b)
{
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}
__device__ __forceinline__ uint32_t pack2_of(f16_t, float a, float b)
{
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}
template <typename T> __device__ __forceinline__ uint4 pack8(const float (&v)[8])
{
    return make_uint4(pack2_of(T{}, v[0], v[1]), pack2_of(T{}, v[2], v[3]), pack2_of(T{}, v[4], v[5]), pack2_of(T{}, v[6], v[7]));
}
__device__ __forceinline__ f32x4_t load4_float(const float *p) { return *reinterpret_cast<const f32x4_t *>(p); }
template <typename T> __device__ __forceinline__ f32x4_t load4_float(const T *p)
{
    const uint2 x = *reinterpret_cast<const uint2 *>(p);
    return f32x4_t{to_float(T{(uint16_t)x.x}), to_float(T{(uint16_t)(x.x >> 16)}), to_float(T{(uint16_t)x.y}), to_float(T{(uint16_t)(x.y >> 16)})};
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]) { *reinterpret_cast<uint4 *>(p) = pack8<T>(v); }

// ---- the matrix product ----

struct LinearArgs {
    const uint16_t *x, *w;
    const float *bias;
    const void *residual;
    void *out;
    const int32_t *count;
    int32_t rows, n, k, act;
    int32_t residual_first;
    int32_t wide_out;               // out's and residual's rows are pieces of 16 bytes, n of eight columns
    int64_t x_row, w_row, residual_row, out_row;
    // many rows: a grid of tiles, each in `splits` pieces of `per_split` stages of 64
    int32_t m_tiles, n_tiles, splits, per_split;
    // few rows: pieces of `per_split` chunks of 64, a wave's share `per_wave`
    int32_t per_wave;
    float *part;                    // [tile][split][what a tile has], in the registers' order
    int32_t *arrived;               // [tile]: pieces that are done; zero before and after every call
};

__device__ __forceinline__ int32_t rows_there(const LinearArgs &a)
{
    return a.count ? min(max(__builtin_amdgcn_readfirstlane(*a.count), 0), a.rows) : a.rows;
}

// A column of a row: bias, residual, activation, one rounding.  v: the sum.
template <typename TO> __device__ __forceinline__ void finish_one(const LinearArgs &a, int64_t row, int c, float v)
{
    float y = v + (a.bias ? a.bias[c] : 0.f);
    const float more = a.residual ? to_float(static_cast<const TO *>(a.residual)[row * a.residual_row + c]) : 0.f;
    if (a.residual_first) y += more;
    y = activate(y, a.act);
    if (!a.residual_first) y += more;
    from_float(y, static_cast<TO *>(a.out) + row * a.out_row + c);
}
// Eight columns of a row, before the rounding.  more: the residual's, where there is one.
__device__ __forceinline__ void finish_eight(const LinearArgs &a, const float (&bias)[8], const float (&more)[8], float (&v)[8])
{
    const bool first = a.residual && a.residual_first, after = a.residual && !a.residual_first;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
    if (first)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += more[i];
    activate_all(v, a.act);
    if (after)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += more[i];
}

// Pieces of a tile that were written past the caches by workgroups of any XCD; the workgroup that comes last adds them in their order.
constexpr int kPiecesPastCaches = 16;
__device__ __forceinline__ bool last_piece(int32_t *arrived, int pieces, int32_t *lds_flag)
{
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wave's stores have been acknowledged ...
    __syncthreads();                                        // ... and the others'
    if (threadIdx.x == 0) {
        const int32_t before = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == pieces - 1) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *lds_flag = before == pieces - 1;
    }
    __syncthreads();
    return *lds_flag;
}

// Raises a kernel's limit of dynamic LDS, once per device.
template <auto KERNEL> hipError_t raise_dynamic_lds(size_t bytes)
{
    static std::atomic<uint64_t> raised{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (raised.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) raised.fetch_or(bit, std::memory_order_release);
    return e;
}

constexpr int kLinearK = 64;        // columns of a stage, or chunk

// Eight elements c .. of a row of k elements and any alignment, zeros behind its end.  Without a branch between loads, which would wait for each of them: 16 bytes that end
// where the row does, shifted; of rows shorter than that every element by itself.
__device__ __forceinline__ uint4 row_end(const uint16_t *__restrict__ row, int c, int k)
{
    if (k >= 8) {
        const int at = min(c, k - 8), by = c - at;
        uint64_t v[2];
        __builtin_memcpy(v, row + at, 16);
        uint64_t lo = by >= 4 ? v[1] : v[0], hi = by >= 4 ? 0 : v[1];
        const int bits = (by & 3) * 16;
        lo = bits ? lo >> bits | hi << (64 - bits) : lo;
        hi >>= bits;
        lo = by >= 8 ? 0 : lo;
        hi = by >= 8 ? 0 : hi;
        return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
    }
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = row[min(c + i, k - 1)];
    loaded_together(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = c + i < k ? e[i] : 0;
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}

// The sums of a block of 16 x 16 with the products of 32 more columns of both operands.
template <int DT> __device__ __forceinline__ f32x4_t mfma16_of(const uint4 &a, const uint4 &b, const f32x4_t &c)
{
    if constexpr (DT == FC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// How a product is cut.
struct LinearPlan {
    int32_t form;                   // 0: few rows, 2: some dozens, 1: many in tiles of 128, 3: of 256; tile_m, tile_n: rows and columns of a workgroup
    int32_t tile_m, tile_n, m_tiles, n_tiles, splits, per_split, per_wave;
    bool wide, ring;                // x's and w's rows are whole 16-byte pieces (few rows); they go through LDS
    bool pad_x, pad_w;              // laid out anew (many rows)
    int64_t padded_k;
    size_t counters, at_x, at_w, at_part, workspace;
};

hipError_t launch_linear_rows(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s);
hipError_t launch_linear_tile(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s);
hipError_t launch_linear_stream(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s);
// (DT, TO: storage type, carrier of the output)
template <int DT, typename TO> hipError_t launch_large_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s);
// Rows of x, of w, or of both, as rows of padded_k elements with zeros behind k.
hipError_t launch_linear_pad(const LinearArgs &a, const LinearPlan &p, uint16_t *x, uint16_t *w, hipStream_t s);

// ---- group norm ----

struct NormArgs {
    const void *x;
    void *out;
    const float *weight, *bias;
    const uint8_t *mask;
    const int32_t *starts;
    int32_t images, rows, max_rows, channels, groups, per_group, act, keep_out;
    float eps;
    int64_t x_row, out_row;
    int32_t slices, slice, chunks, chunk_rows;      // channels of a slice (whole groups), rows of a chunk
    float4 *part;                                   // [image][slice][group of a slice][chunk]: count, mean, squared distances
};

struct NormPlan {
    bool once;                      // a workgroup holds an image's slice: read once
    bool wide;                      // pieces of 16 bytes, else elements
    int32_t threads, per_thread, slice, slices, chunks, chunk_rows;
    size_t lds, workspace;
};

hipError_t launch_group_norm(const NormArgs &a, const NormPlan &p, int dtype, hipStream_t s);

} // namespace fc
