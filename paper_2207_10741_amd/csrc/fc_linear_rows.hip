// Matrix product of few rows (one user's next token, a batch's next tokens): out = act(x w^T + bias) + residual.
//
// Every weight is needed once, so the weights' bytes bound it.  A workgroup has 16 NB columns of the output (rows of w) and 16 RB rows of x; its waves divide the
// reduction among them, so that a launch of few columns still has all of its loads under way at once, and add their sums through LDS in order.
//   k_linear_ring   rows of whole 16-byte pieces: both operands come in lines of 128 bytes through a ring in LDS of each wave's own.  Weights that are not in a cache:
//                   1 x 4096 x 4096 9.2 us (33 MB: 6.4 at the rate of a copy, and a launch), 1 x 4096 x 16384 29.4 (4.6 TB/s), 64 x 4096 x 16384 33.8 (with bias and GELU 36.6)
//   k_linear_rows   rows of any alignment: straight from memory to the registers that the matrix instructions read, with no LDS and no barrier between.  Where columns are
//                   fewer than the chip wants workgroups, workgroups divide the reduction as well (pieces, joined by the last in order)
//
// A lane of an operand of the 16x16x32 instructions holds eight consecutive elements of one row: lanes 0 .. 15 the rows, quarter = lane / 16 the eighths of 32 elements.
#include "fc_layers_internal.hpp"

namespace fc {

constexpr int kRowsWaves = 8, kRowsThreads = kRowsWaves * 64;

// A workgroup's tile and piece.  All row tiles and pieces of a tile of columns are an XCD's (workgroups number 0 .. 7 in turn): its L2 has the weights.
struct RowsTile {
    int tile, split, m, n;
};
template <bool SPLIT> __device__ __forceinline__ RowsTile rows_tile(const LinearArgs &a)
{
    const int slot = (int)blockIdx.x >> 3, split = SPLIT ? slot % a.splits : 0, pair = SPLIT ? slot / a.splits : slot;
    RowsTile t;
    t.split = split;
    t.m = pair % a.m_tiles;
    t.n = pair / a.m_tiles * 8 + ((int)blockIdx.x & 7);
    t.tile = t.n * a.m_tiles + t.m;
    return t;
}

// Eight elements c .. of a row of any alignment.  FULL: all are inside k; else those behind are zero.
template <bool FULL> __device__ __forceinline__ uint4 row_piece(const uint16_t *__restrict__ row, int c, int k)
{
    if constexpr (!FULL) return row_end(row, c, k);
    uint4 v;
    __builtin_memcpy(&v, row + c, 16);
    return v;
}

// From the waves' sums to the output: added in the waves' order, and with SPLIT in pieces' order where workgroups share the reduction.  sums: LDS for all of them.
template <typename TO, int RB, int NB, int WAVES, bool SPLIT>
__device__ __forceinline__ void finish_rows(const LinearArgs &a, const f32x4_t (&acc)[RB][NB], f32x4_t *sums, int32_t *flag, int rows, int r0, int n0, int tile, int split)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
    auto sum_of = [&](int item) __attribute__((always_inline)) {
        f32x4_t v = sums[item];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w * ITEMS + item];
        return v;
    };
    if (!SPLIT || a.splits == 1) {
        for (int item = threadIdx.x; item < ITEMS; item += (WAVES * 64)) finish(item, sum_of(item));
        return;
    }
    if constexpr (SPLIT) {
        const auto part = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)tile * a.splits * (ITEMS * 4), 0, (uint32_t)a.splits * ITEMS * 16u, 0x00020000);
        for (int item = threadIdx.x; item < ITEMS; item += (WAVES * 64))
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, sum_of(item)), part, (uint32_t)(split * ITEMS + item) * 16u, 0, kPiecesPastCaches);
        if (!last_piece(a.arrived + tile, a.splits, flag)) return;
        for (int item = threadIdx.x; item < ITEMS; item += (WAVES * 64)) {
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
}

// RB, NB: blocks of 16 rows and of 16 columns; U: chunks of 64 whose loads are sent for together.
template <int DT, typename TO, int RB, int NB, int U>
__global__ __launch_bounds__(kRowsThreads, 2)
void k_linear_rows(LinearArgs a)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    f32x4_t *const sums = reinterpret_cast<f32x4_t *>(smem_raw);       // [wave][block][lane]
    __shared__ int32_t flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowsTile t = rows_tile<true>(a);
    const int split = t.split, tile = t.tile, n0 = t.n * (16 * NB), r0 = t.m * (16 * RB);
    const int rows = rows_there(a);
    if (t.n >= a.n_tiles || r0 >= rows) return;
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
            for (int b = 0; b < NB; ++b) wf[u][b][h] = row_piece<FULL>(wp[b], c, a.k);
#pragma unroll
            for (int b = 0; b < RB; ++b) xf[u][b][h] = row_piece<FULL>(xp[b], c, a.k);
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

    finish_rows<TO, RB, NB, kRowsWaves, true>(a, acc, sums, &flag, rows, r0, n0, tile, split);
}

template <int DT, typename TO, int RB, int NB, int U> static hipError_t launch_rows_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = (size_t)kRowsWaves * RB * NB * 1024;
    if (lds > 65536) {
        const hipError_t e = raise_dynamic_lds<&k_linear_rows<DT, TO, RB, NB, U>>(lds);
        if (e != hipSuccess) return e;
    }
    k_linear_rows<DT, TO, RB, NB, U><<<dim3((uint32_t)((p.n_tiles + 7) / 8 * 8 * p.m_tiles * p.splits)), dim3(kRowsThreads), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_rows_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    return p.tile_m == 16 ? launch_rows_of<DT, TO, 1, 1, 6>(a, p, s) : launch_rows_of<DT, TO, 2, 1, 4>(a, p, s);
}

// Both operands through LDS.  Loads of 16 rows of 64 bytes come at 18 bytes a clock and CU, whole lines of 128 bytes at 64: with some dozens of rows, whose x is
// as many bytes as the weights that a workgroup reads, the first is slower than memory (64 x 4096 x 16384 straight into registers 44 us, so 36 when both were built).  A wave has a ring of D chunks of its own and no one to
// wait for: its loads are D - 1 chunks ahead, and the barrier comes when the sums are added.  The reduction is not divided among workgroups: with the arithmetic and the
// branches for that, which no product wanted, 1 x 1024 x 1024 took 3.86 us and 64 x 1024 x 1024 6.35, so 3.67 and 5.91.
template <int RB, int NB, int WAVES, int D> constexpr size_t kRingLds = (size_t)WAVES * D * (RB + NB) * 2048;

template <int DT, typename TO, int RB, int NB, int WAVES, int D>
__global__ __launch_bounds__(WAVES * 64)
void k_linear_ring(LinearArgs a)
{
    constexpr uint32_t CHUNK = (RB + NB) * 2048u;       // a chunk: rows of x, then of w, 128 bytes each
    constexpr int NL = 2 * (RB + NB);
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowsTile t = rows_tile<false>(a);
    const int n0 = t.n * (16 * NB), r0 = t.m * (16 * RB);
    const int rows = rows_there(a);
    if (t.n >= a.n_tiles || r0 >= rows) return;
    const int here = min(rows - r0, 16 * RB), cols = min(a.n - n0, 16 * NB);
    const u32x4_t rsrc_x = make_rsrc_words(a.x + (int64_t)r0 * a.x_row, (uint32_t)((int64_t)(here - 1) * a.x_row + a.k) * 2u);
    const u32x4_t rsrc_w = make_rsrc_words(a.w + (int64_t)n0 * a.w_row, (uint32_t)((int64_t)(cols - 1) * a.w_row + a.k) * 2u);
    // load j: rows 8 j .. 8 j + 7; a lane's slot holds the piece slot ^ swizzle(row), of even and of odd loads
    const int piece[2] = {(lane & 7) ^ FC_SWZ(lane >> 3), (lane & 7) ^ FC_SWZ(8 + (lane >> 3))};
    uint32_t xo[2 * RB], wo[2 * NB];
#pragma unroll
    for (int j = 0; j < 2 * RB; ++j) {
        const int r = j * 8 + (lane >> 3);
        xo[j] = r < here ? (uint32_t)((int64_t)r * a.x_row * 2) + (uint32_t)piece[j & 1] * 16u : kOutOfRange;
    }
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) {
        const int r = j * 8 + (lane >> 3);
        wo[j] = r < cols ? (uint32_t)((int64_t)r * a.w_row * 2) + (uint32_t)piece[j & 1] * 16u : kOutOfRange;
    }
    // this wave's chunks
    const int chunks = (a.k + kLinearK - 1) / kLinearK;
    const int from = wave * a.per_wave, to = min(from + a.per_wave, chunks), k_end = min(to * kLinearK, a.k);
    unsigned char *const ring = smem_raw + (uint32_t)wave * (D * CHUNK);
    const uint32_t ring0 = (uint32_t)reinterpret_cast<uintptr_t>(smem_raw) + (uint32_t)wave * (D * CHUNK);
    int ld_k = from * kLinearK;
    uint32_t ld_at = 0;
    // the next chunk is sent for (behind the last one: zeros)
    auto send = [&]() __attribute__((always_inline)) {
        const bool ok[2] = {ld_k + piece[0] * 8 < k_end, ld_k + piece[1] * 8 < k_end};
        const uint32_t s = ld_k < k_end ? (uint32_t)ld_k * 2u : 0u;
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) dma_load16_any(rsrc_w, ok[j & 1] ? wo[j] : kOutOfRange, s, ring0 + ld_at + RB * 2048u + (uint32_t)j * 1024u);
#pragma unroll
        for (int j = 0; j < 2 * RB; ++j) dma_load16_any(rsrc_x, ok[j & 1] ? xo[j] : kOutOfRange, s, ring0 + ld_at + (uint32_t)j * 1024u);
        ld_k += kLinearK;
        ld_at = ld_at + CHUNK == D * CHUNK ? 0 : ld_at + CHUNK;
    };
    f32x4_t acc[RB][NB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[r][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < D - 1; ++d) send();
    const uint32_t row = (uint32_t)(lane & 15), frag = row * 128u + (((uint32_t)(lane >> 4) ^ FC_SWZ(row)) * 16u);
    uint32_t at = 0;
    for (int c = from; c < to; ++c) {
        lds_reads_done();       // (of the chunk before, whose place is sent for)
        wait_vmcnt<(D - 2) * NL>();
        send();
        uint4 wf[NB][2], xf[RB][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char *const p = ring + at + (frag ^ (uint32_t)(h * 64));
#pragma unroll
            for (int b = 0; b < NB; ++b) wf[b][h] = *reinterpret_cast<const uint4 *>(p + (RB + b) * 2048);
#pragma unroll
            for (int r = 0; r < RB; ++r) xf[r][h] = *reinterpret_cast<const uint4 *>(p + r * 2048);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[r][b] = mfma16_of<DT>(wf[b][h], xf[r][h], acc[r][b]);
        at = at + CHUNK == D * CHUNK ? 0 : at + CHUNK;
    }
    lds_reads_done();
    wait_vmcnt<0>();
    __syncthreads();
    finish_rows<TO, RB, NB, WAVES, false>(a, acc, reinterpret_cast<f32x4_t *>(smem_raw), nullptr, rows, r0, n0, 0, 0);
}

template <int DT, typename TO, int RB, int NB, int WAVES, int D> static hipError_t launch_ring_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = kRingLds<RB, NB, WAVES, D>;
    static_assert(lds >= (size_t)WAVES * RB * NB * 1024, "room for the sums");
    const hipError_t e = raise_dynamic_lds<&k_linear_ring<DT, TO, RB, NB, WAVES, D>>(lds);
    if (e != hipSuccess) return e;
    k_linear_ring<DT, TO, RB, NB, WAVES, D><<<dim3((uint32_t)((p.n_tiles + 7) / 8 * 8 * p.m_tiles)), dim3(WAVES * 64), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_ring_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    if (p.tile_m == 16) return p.tile_n == 16 ? launch_ring_of<DT, TO, 1, 1, 8, 4>(a, p, s) : launch_ring_of<DT, TO, 1, 2, 8, 3>(a, p, s);
    if (p.tile_m == 32) return p.tile_n == 16 ? launch_ring_of<DT, TO, 2, 1, 8, 3>(a, p, s) : p.tile_n == 32 ? launch_ring_of<DT, TO, 2, 2, 8, 2>(a, p, s) : launch_ring_of<DT, TO, 2, 4, 4, 3>(a, p, s);
    return p.tile_n == 16 ? launch_ring_of<DT, TO, 4, 1, 4, 4>(a, p, s) : p.tile_n == 32 ? launch_ring_of<DT, TO, 4, 2, 4, 3>(a, p, s) : launch_ring_of<DT, TO, 4, 4, 4, 2>(a, p, s);
}

hipError_t launch_linear_rows(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (p.ring) {
        if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_ring_as<FC_BF16, float>(a, p, s) : launch_ring_as<FC_BF16, bf16_t>(a, p, s);
        return out_dtype == FC_F32 ? launch_ring_as<FC_F16, float>(a, p, s) : launch_ring_as<FC_F16, f16_t>(a, p, s);
    }
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_rows_as<FC_BF16, float>(a, p, s) : launch_rows_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_rows_as<FC_F16, float>(a, p, s) : launch_rows_as<FC_F16, f16_t>(a, p, s);
}

} // namespace fc
