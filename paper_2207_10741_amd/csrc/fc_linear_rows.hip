// Matrix product of few rows (one user's next token, a batch's next tokens): out = act(x w^T + bias) + residual.
//
// Every weight is needed once, so the weights' bytes bound it: they go straight from memory to the registers that the 16x16x32 matrix
// instructions read, with no LDS and no barrier between.  A workgroup of eight waves has 16 NB columns of the output (rows of w) and 16 RB rows of x; its
// waves divide the reduction among them, so that a launch of few columns still has all of its loads under way at once, and add their sums through LDS in
// order.  Where columns are fewer than the chip wants workgroups, workgroups divide the reduction as well (pieces, joined by the last in order).
//
// A lane of an operand holds eight consecutive elements of one row: lanes 0 .. 15 the rows, quarter = lane / 16 the eighths of 32 elements.
#include "fc_layers_internal.hpp"

namespace fc {

constexpr int kRowsWaves = 8, kRowsThreads = kRowsWaves * 64;

// Eight elements c .. of a row.  FULL: all are inside k; else those behind are zero.  WIDE: the row's pieces are aligned to 16 bytes.
template <bool WIDE, bool FULL> __device__ __forceinline__ uint4 row_piece(const uint16_t *__restrict__ row, int c, int k)
{
    if constexpr (FULL) {
        if constexpr (WIDE) return *reinterpret_cast<const uint4 *>(row + c);
        uint4 v;
        __builtin_memcpy(&v, row + c, 16);
        return v;
    } else if constexpr (WIDE) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + (c < k ? c : 0));
        return c < k ? v : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = c + 2 * j < k ? row[c + 2 * j] : 0, hi = c + 2 * j + 1 < k ? row[c + 2 * j + 1] : 0;
            v[j] = lo | hi << 16;
        }
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
}

template <int DT> __device__ __forceinline__ f32x4_t mfma16_of(const uint4 &a, const uint4 &b, const f32x4_t &c)
{
    if constexpr (DT == FC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// RB, NB: blocks of 16 rows and of 16 columns; U: chunks of 64 whose loads are sent for together.
template <int DT, typename TO, int RB, int NB, int U, bool WIDE>
__global__ __launch_bounds__(kRowsThreads, 2)
void k_linear_rows(LinearArgs a)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    f32x4_t *const sums = reinterpret_cast<f32x4_t *>(smem_raw);       // [wave][block][lane]
    __shared__ int32_t flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int split = (int)blockIdx.x % a.splits, tile = (int)blockIdx.x / a.splits;
    const int n0 = tile % a.n_tiles * (16 * NB), r0 = tile / a.n_tiles * (16 * RB);
    const int rows = rows_there(a);
    if (r0 >= rows) return;
    // (rows and columns that are not there: the last one's again, whose sums nobody stores)
    const uint16_t *wp[NB], *xp[RB];
#pragma unroll
    for (int b = 0; b < NB; ++b) wp[b] = a.w + (int64_t)min(n0 + b * 16 + (lane & 15), a.n - 1) * a.w_row;
#pragma unroll
    for (int b = 0; b < RB; ++b) xp[b] = a.x + (int64_t)min(r0 + b * 16 + (lane & 15), rows - 1) * a.x_row;
    const int at = (lane >> 4) * 8;

    f32x4_t acc[RB][NB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[r][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // this wave's chunks
    const int chunks = (a.k + kLinearK - 1) / kLinearK, whole = a.k / kLinearK;
    const int from = split * a.per_split + wave * a.per_wave;
    const int to = min(min(from + a.per_wave, (split + 1) * a.per_split), chunks);
    uint4 wf[U][NB][2], xf[U][RB][2];
    auto load = [&](int chunk, int u, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = chunk * kLinearK + h * 32 + at;
#pragma unroll
            for (int b = 0; b < NB; ++b) wf[u][b][h] = row_piece<WIDE, FULL>(wp[b], c, a.k);
#pragma unroll
            for (int b = 0; b < RB; ++b) xf[u][b][h] = row_piece<WIDE, FULL>(xp[b], c, a.k);
        }
    };
    auto multiply = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[r][b] = mfma16_of<DT>(wf[u][b][h], xf[u][r][h], acc[r][b]);
    };
    const int whole_to = min(to, whole);
    int c = from;
    // (each chunk's place is loaded again as soon as its products are out)
    if (c + U <= whole_to) {
#pragma unroll
        for (int u = 0; u < U; ++u) load(c + u, u, std::true_type{});
        for (; c + 2 * U <= whole_to; c += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                multiply(u);
                load(c + U + u, u, std::true_type{});
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(u);
        c += U;
    }
    for (; c < whole_to; ++c) {
        load(c, 0, std::true_type{});
        multiply(0);
    }
    for (; c < to; ++c) {
        load(c, 0, std::false_type{});
        multiply(0);
    }

#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int b = 0; b < NB; ++b) sums[(wave * (RB * NB) + r * NB + b) * 64 + lane] = acc[r][b];
    __syncthreads();
    constexpr int ITEMS = RB * NB * 64;
    auto finish = [&](int item, f32x4_t v) __attribute__((always_inline)) {
        const int l = item & 63, block = item >> 6, row = r0 + block / NB * 16 + (l & 15), col = n0 + block % NB * 16 + (l >> 4) * 4;
        if (row >= rows || col >= a.n) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < a.n) finish_one<TO>(a, row, col + i, v[i]);
    };
    __amdgpu_buffer_rsrc_t part;
    if (a.splits > 1)
        part = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)tile * a.splits * (ITEMS * 4), 0, (uint32_t)a.splits * ITEMS * 16u, 0x00020000);
    for (int item = threadIdx.x; item < ITEMS; item += kRowsThreads) {
        f32x4_t v = sums[item];
#pragma unroll
        for (int w = 1; w < kRowsWaves; ++w) v += sums[w * ITEMS + item];
        if (a.splits == 1) finish(item, v);
        else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), part, (uint32_t)(split * ITEMS + item) * 16u, 0, kPiecesPastCaches);
    }
    if (a.splits == 1 || !last_piece(a.arrived + tile, a.splits, &flag)) return;
    for (int item = threadIdx.x; item < ITEMS; item += kRowsThreads) {
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < a.splits; i += 4) {
            f32x4_t p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                p[u] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(part, (uint32_t)(min(i + u, a.splits - 1) * ITEMS + item) * 16u, 0, kPiecesPastCaches));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < a.splits) v += p[u];
        }
        finish(item, v);
    }
}

template <int DT, typename TO, int RB, int NB, int U, bool WIDE> static hipError_t launch_rows_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = (size_t)kRowsWaves * RB * NB * 1024;
    if (lds > 65536) {
        const hipError_t e = raise_dynamic_lds<&k_linear_rows<DT, TO, RB, NB, U, WIDE>>(lds);
        if (e != hipSuccess) return e;
    }
    k_linear_rows<DT, TO, RB, NB, U, WIDE><<<dim3((uint32_t)(p.m_tiles * p.n_tiles * p.splits)), dim3(kRowsThreads), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_rows_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    auto form = [&](auto wide) {
        constexpr bool W = decltype(wide)::value;
        if (p.tile_m == 16) return p.tile_n == 16 ? launch_rows_of<DT, TO, 1, 1, 6, W>(a, p, s) : launch_rows_of<DT, TO, 1, 2, 4, W>(a, p, s);
        if (p.tile_m == 32) return p.tile_n == 16 ? launch_rows_of<DT, TO, 2, 1, 4, W>(a, p, s) : launch_rows_of<DT, TO, 2, 2, 3, W>(a, p, s);
        return p.tile_n == 16 ? launch_rows_of<DT, TO, 4, 1, 3, W>(a, p, s) : launch_rows_of<DT, TO, 4, 4, 2, W>(a, p, s);
    };
    return p.wide ? form(std::true_type{}) : form(std::false_type{});
}

hipError_t launch_linear_rows(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_rows_as<FC_BF16, float>(a, p, s) : launch_rows_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_rows_as<FC_F16, float>(a, p, s) : launch_rows_as<FC_F16, f16_t>(a, p, s);
}

} // namespace fc
