// Matrix product of many rows: out = act(x w^T + bias) + residual.
//
// A workgroup has a tile of TM rows and TN columns, and goes over the reduction in stages of 64 (128 bytes of a row).  A stage's rows of x and of w go straight
// from memory into LDS, two stages deep, each row's 16-byte pieces exchanged by the row's number so that the reads of a fragment meet no bank
// twice.  A wave owns PB x 2 blocks of 32 x 32 sums (32x32x16 matrix instructions); with 128 x 64 a wave an instruction needs 0.75 KB of LDS reads.
// Everything that is not a product goes out between two of them: fragments a k-step ahead, across the stage's border too (its barrier stands inside
// the last k-step), a stage's loads after the barrier that frees their buffer.
//
// Bounds are explicit: a row or a piece that is not there has an offset out of every descriptor's range and comes back as zeros.
#include "fc_layers_internal.hpp"
#include <type_traits>

namespace fc {

// f(integral_constant 0) .. f(integral_constant N - 1)
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

template <int WM, int WN, int PB> constexpr size_t kTileLds = (size_t)2 * (WM * PB * 32 + WN * 64) * 128 + 16;

template <int DT, typename TO, int WM, int WN, int PB>
__global__ __launch_bounds__(WM * WN * 64, 2)
void k_linear_tile(LinearArgs a)
{
    constexpr int NT = WM * WN * 64, CB = 2, TM = WM * PB * 32, TN = WN * CB * 32;
    constexpr int RPL = NT / 8;                     // rows that the waves' loads cover side by side
    constexpr int XL = TM / RPL, WL = TN / RPL, KK = 4;
    constexpr uint32_t XB = TM * 128u, SB = (TM + TN) * 128u;      // a stage: rows of x, then of w
    static_assert(TM % RPL == 0 && TN % RPL == 0 && RPL % 16 == 0, "whole loads; the exchange is the same for all of a lane's rows");

    extern __shared__ __align__(16) unsigned char smem_raw[];
    int32_t *const flag = reinterpret_cast<int32_t *>(smem_raw + 2 * SB);
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(smem_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave % WM, wave_n = wave / WM;

    // ---- which tile: an XCD (workgroups number 0 .. 7 in turn) takes a run of the tiles, which go down eight tiles of rows before the next columns ----
    const int rows = rows_there(a);
    const int m_tiles = (rows + TM - 1) / TM, total = m_tiles * a.n_tiles * a.splits;
    const int xcd = (int)blockIdx.x & 7, first = (int)(((int64_t)total * xcd) >> 3), behind = (int)(((int64_t)total * (xcd + 1)) >> 3);
    const int number = first + ((int)blockIdx.x >> 3);
    if (number >= behind) return;
    const int split = number % a.splits, tile = number / a.splits;
    constexpr int GROUP = 8;
    const int group = tile / (GROUP * a.n_tiles), in_group = tile - group * GROUP * a.n_tiles;
    const int high = min(GROUP, m_tiles - group * GROUP);
    const int tile_m = group * GROUP + in_group % high, tile_n = in_group / high;
    const int r0 = tile_m * TM, n0 = tile_n * TN;

    const int here = min(rows - r0, TM), cols = min(a.n - n0, TN);
    const u32x4_t rsrc_x = make_rsrc_words(a.x + (int64_t)r0 * a.x_row, (uint32_t)((int64_t)(here - 1) * a.x_row + a.k) * 2u);
    const u32x4_t rsrc_w = make_rsrc_words(a.w + (int64_t)n0 * a.w_row, (uint32_t)((int64_t)(cols - 1) * a.w_row + a.k) * 2u);
    // a lane's place in a load: row (of every RPL) and slot; the slot holds the piece slot ^ swizzle(row)
    const int lrow = wave * 8 + (lane >> 3), piece = (lane & 7) ^ FC_SWZ(lrow);
    uint32_t xo[XL], wo[WL];
#pragma unroll
    for (int j = 0; j < XL; ++j) {
        const int r = j * RPL + lrow;
        xo[j] = r < here ? (uint32_t)((int64_t)r * a.x_row * 2) + (uint32_t)piece * 16u : kOutOfRange;
    }
#pragma unroll
    for (int j = 0; j < WL; ++j) {
        const int r = j * RPL + lrow;
        wo[j] = r < cols ? (uint32_t)((int64_t)r * a.w_row * 2) + (uint32_t)piece * 16u : kOutOfRange;
    }
    const int k0 = split * a.per_split * kLinearK, stages = min(a.per_split, (a.k - k0 + kLinearK - 1) / kLinearK);
    const int k_end = min(a.k, k0 + stages * kLinearK);
    // the next stage to be sent for (behind the last one: zeros)
    int ld_k = k0;
    uint32_t ld_s = 0;
    bool ld_ok = false;
    auto next_stage = [&]() __attribute__((always_inline)) {
        ld_ok = ld_k + piece * 8 < k_end;
        ld_s = ld_k < k_end ? (uint32_t)ld_k * 2u : 0u;
        ld_k += kLinearK;
    };
    const uint32_t lds_wave = lds0 + (uint32_t)wave * 1024u;
    auto issue = [&](int j, uint32_t buf) __attribute__((always_inline)) {
        if (j < XL) dma_load16_any(rsrc_x, ld_ok ? xo[j] : kOutOfRange, ld_s, lds_wave + buf * SB + (uint32_t)j * (RPL * 128u));
        else dma_load16_any(rsrc_w, ld_ok ? wo[j - XL] : kOutOfRange, ld_s, lds_wave + buf * SB + XB + (uint32_t)(j - XL) * (RPL * 128u));
    };

    // where this lane's fragments are: row of the block, half of the k-step
    const uint32_t frow = (uint32_t)(lane & 31);
    const uint32_t fx = (uint32_t)(wave_m * (PB * 32)) * 128u + frow * 128u, fw = XB + (uint32_t)(wave_n * (CB * 32)) * 128u + frow * 128u;
    const uint32_t ft = (uint32_t)((lane >> 5) ^ FC_SWZ(frow)) * 16u;       // (blocks begin at multiples of 32 rows: the exchange is the row's in the block)

    f32x16_t acc[PB][CB];
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[p][b][i] = 0.f;

    next_stage();
#pragma unroll
    for (int j = 0; j < XL + WL; ++j) issue(j, 0);
    next_stage();
#pragma unroll
    for (int j = 0; j < XL + WL; ++j) issue(j, 1);
    wait_vmcnt<XL + WL>();
    __syncthreads();

    Frag<DT> wf[2][CB], xf[2][PB];
    constexpr int NM = PB * CB, NR = PB + CB, NL = XL + WL;
    // fragment r of a k-step, in the order the products need them: w0, x0, w1, x1 ..
    auto read_frag = [&](int r, int set, uint32_t buf, int kk) __attribute__((always_inline)) {
        const uint32_t o = buf * SB + (((uint32_t)kk * 32u) ^ ft);
        if (r == 1 || r > CB) {
            const int p = r == 1 ? 0 : r - CB;
            xf[set][p].load(smem_raw, o + fx + (uint32_t)p * 4096u);
        } else {
            const int b = r == 0 ? 0 : r - 1;
            wf[set][b].load(smem_raw, o + fw + (uint32_t)b * 4096u);
        }
    };
#pragma unroll
    for (int r = 0; r < NR; ++r) read_frag(r, 0, 0, 0);
    auto stage = [&](auto buf_c) __attribute__((always_inline)) {
        constexpr uint32_t BUF = decltype(buf_c)::value;
        each<KK>([&](auto kk_c) __attribute__((always_inline)) {
            constexpr int kk = decltype(kk_c)::value;
            constexpr bool last = kk == KK - 1;
            constexpr int BAR = NM / 4, from = last ? BAR : 0, gaps = NM - from, nl = last ? NL : 0;
            each<NM>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value;
                if constexpr (last && i == BAR) {       // the next stage has landed, everyone has read this one
                    lds_reads_done();
                    wait_vmcnt<0>();
                    __syncthreads();
                    next_stage();
                }
                acc[i / CB][i % CB] = mfma32<DT>(wf[kk & 1][i % CB], xf[kk & 1][i / CB], acc[i / CB][i % CB]);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (i >= from) {
                    constexpr int j = i - from;         // this gap's share of the reads and loads
                    each<((j + 1) * NR + gaps - 1) / gaps - (j * NR + gaps - 1) / gaps>([&](auto e_c) __attribute__((always_inline)) {
                        constexpr int r = (j * NR + gaps - 1) / gaps + decltype(e_c)::value;
                        if constexpr (r < NR) {
                            if constexpr (last) read_frag(r, 0, BUF ^ 1u, 0);
                            else read_frag(r, (kk + 1) & 1, BUF, kk + 1);
                        }
                    });
                    each<((j + 1) * nl) / gaps - (j * nl) / gaps>([&](auto e_c) __attribute__((always_inline)) {
                        issue((j * nl) / gaps + decltype(e_c)::value, BUF);
                    });
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
        });
    };
    for (int s = 0; s < stages; s += 2) {
        stage(std::integral_constant<uint32_t, 0>{});
        if (s + 1 < stages) stage(std::integral_constant<uint32_t, 1>{});
    }
    lds_reads_done();
    wait_vmcnt<0>();
    __syncthreads();

    // ---- pieces of the reduction (small tiles): written in the registers' order, added by the last workgroup in the pieces' order ----
    if (TM == 128 && a.splits > 1) {
        constexpr uint32_t ITEMS = (uint32_t)PB * CB * 4 * NT;     // of four sums
        const auto part = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)tile * a.splits * (ITEMS * 4), 0, (uint32_t)a.splits * ITEMS * 16u, 0x00020000);
        each<PB * CB * 4>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value, q = i % 4 * 4;
            const f32x16_t &s = acc[i / 4 / CB][i / 4 % CB];
            const f32x4_t v = {s[q], s[q + 1], s[q + 2], s[q + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), part, ((uint32_t)split * ITEMS + (uint32_t)i * NT + threadIdx.x) * 16u, 0, kPiecesPastCaches);
        });
        if (!last_piece(a.arrived + tile, a.splits, flag)) return;
#pragma unroll
        for (int p = 0; p < PB; ++p)
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[p][b][i] = 0.f;
        for (int n = 0; n < a.splits; ++n)
            each<PB * CB * 4>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, q = i % 4 * 4;
                const f32x4_t v = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(part, ((uint32_t)n * ITEMS + (uint32_t)i * NT + threadIdx.x) * 16u, 0, kPiecesPastCaches));
                f32x16_t &s = acc[i / 4 / CB][i / 4 % CB];
                s[q] += v[0], s[q + 1] += v[1], s[q + 2] += v[2], s[q + 3] += v[3];
            });
    }

    // ---- epilogue: every wave turns its blocks of 32 rows x 64 columns through LDS of its own, so that a lane has eight columns next to each other ----
    constexpr int OP = CB * 32 + 4;     // floats from row to row
    static_assert((size_t)WM * WN * 32 * OP * 4 <= 2 * SB, "the waves' shares");
    float *const os = reinterpret_cast<float *>(smem_raw) + wave * (32 * OP);
    const int c8 = lane & 7, col = n0 + wave_n * (CB * 32) + c8 * 8;
#pragma unroll
    for (int p = 0; p < PB; ++p) {
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4_t v = {acc[p][b][q * 4], acc[p][b][q * 4 + 1], acc[p][b][q * 4 + 2], acc[p][b][q * 4 + 3]};
                *reinterpret_cast<f32x4_t *>(os + (lane & 31) * OP + b * 32 + q * 8 + (lane >> 5) * 4) = v;
            }
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + (lane >> 3), row = r0 + (wave_m * PB + p) * 32 + r;
            float v[8];
            load8_float(os + r * OP + c8 * 8, v);
            if (row < rows && col < a.n) finish_columns<TO, 8>(a, row, col, v);
        }
        wave_lds_order();
    }
}

// Rows laid out anew: padded_k elements each, zeros behind k.
__global__ __launch_bounds__(256) void k_linear_pad(LinearArgs a, int32_t padded_k, uint16_t *__restrict__ x, uint16_t *__restrict__ w)
{
    const int per_row = padded_k / 8;
    const int64_t x_items = x ? (int64_t)rows_there(a) * per_row : 0, items = x_items + (w ? (int64_t)a.n * per_row : 0);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const bool of_x = i < x_items;
        const int64_t at = of_x ? i : i - x_items, row = at / per_row;
        const int c = (int)(at - row * per_row) * 8;
        const uint16_t *const from = of_x ? a.x + row * a.x_row : a.w + row * a.w_row;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c + 8 <= a.k) {
            __builtin_memcpy(&v, from + c, 16);
        } else {
            uint16_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = c + j < a.k ? from[c + j] : 0;
            __builtin_memcpy(&v, e, 16);
        }
        *reinterpret_cast<uint4 *>((of_x ? x : w) + row * padded_k + c) = v;
    }
}

hipError_t launch_linear_pad(const LinearArgs &a, const LinearPlan &p, uint16_t *x, uint16_t *w, hipStream_t s)
{
    const int64_t items = ((x ? (int64_t)a.rows : 0) + (w ? a.n : 0)) * (p.padded_k / 8), blocks = (items + 255) / 256;
    k_linear_pad<<<dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s>>>(a, (int32_t)p.padded_k, x, w);
    return hipGetLastError();
}

template <int DT, typename TO, int WM, int WN, int PB> static hipError_t launch_tile_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = kTileLds<WM, WN, PB>;
    const hipError_t e = raise_dynamic_lds<&k_linear_tile<DT, TO, WM, WN, PB>>(lds);
    if (e != hipSuccess) return e;
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    k_linear_tile<DT, TO, WM, WN, PB><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_tile_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    return p.tile_m == 256 ? launch_tile_of<DT, TO, 2, 4, 4>(a, p, s) : launch_tile_of<DT, TO, 2, 2, 2>(a, p, s);
}

hipError_t launch_linear_tile(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_tile_as<FC_BF16, float>(a, p, s) : launch_tile_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_tile_as<FC_F16, float>(a, p, s) : launch_tile_as<FC_F16, f16_t>(a, p, s);
}

} // namespace fc
