// Matrix product of many rows: out = act(x w^T + bias) + residual.
//
// A workgroup has a tile of TM rows and TN columns (128 x 128, a wave 64 x 64), and goes over the reduction in stages of 64 (128 bytes of a row).  A stage's rows of x and of w go
// straight from memory into LDS, three stages of x and two of w deep, each row's 16-byte pieces exchanged by the row's number so that the reads of a fragment meet no bank
// twice.  A wave owns PB x CB blocks of 32 x 32 sums (32x32x16 matrix instructions).
// Everything that is not a product goes out between two of them: fragments a k-step ahead, across the stage's border too (its barrier stands inside
// the last k-step), a stage's loads after the barrier that frees their buffer.
//
// Bounds are explicit: a row or a piece that is not there has an offset out of every descriptor's range and comes back as zeros.  Bound by the L1 path: 64 bytes a clock for loads into LDS
// (4096 x 4096 x 4096 141 us, tiles of 256 100; 2048 x 4096 x 4096 71, so 83).
#include "fc_linear_tile.hpp"

namespace fc {

// three stages' rows of x, two stages' rows of w
template <int WM, int WN, int PB, int CB> constexpr size_t kTileLds = (size_t)(3 * WM * PB + 2 * WN * CB) * 32 * 128;

template <int DT, typename TO, int WM, int WN, int PB, int CB>
__global__ __launch_bounds__(WM * WN * 64, 2)
void k_linear_tile(LinearArgs a)
{
    constexpr int NT = WM * WN * 64, TM = WM * PB * 32, TN = WN * CB * 32;
    constexpr int RPL = NT / 8;                     // rows that the waves' loads cover side by side
    constexpr int XL = TM / RPL, WL = TN / RPL, KK = 4;
    constexpr uint32_t XB = TM * 128u, WB = TN * 128u, W0 = 3 * XB;     // a stage's rows of x, of w; where the latter begin
    static_assert(TM % RPL == 0 && TN % RPL == 0 && RPL % 16 == 0, "whole loads; the exchange is the same for all of a lane's rows");

    extern __shared__ __align__(16) unsigned char smem_raw[];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(smem_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave % WM, wave_n = wave / WM;

    const int rows = rows_there(a);
    const TileOf t = tile_of<TM>(a, rows);
    if (!t.there) return;
    const int split = t.split, r0 = t.tile_m * TM, n0 = t.tile_n * TN;

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
    // The next stages to be sent for.  From the stage on that the reduction ends in, pieces behind its end come from out of range (zeros): there is no stage
    // after it that would want them back.
    int nx_k = k0, nw_k = k0;
    uint32_t nx_s = 0, nw_s = 0;
    auto advance_x = [&]() __attribute__((always_inline)) {
        if (nx_k + kLinearK > k_end)
#pragma unroll
            for (int j = 0; j < XL; ++j) xo[j] = nx_k + piece * 8 < k_end ? xo[j] : kOutOfRange;
        nx_s = nx_k < k_end ? (uint32_t)nx_k * 2u : 0u;
        nx_k += kLinearK;
    };
    auto advance_w = [&]() __attribute__((always_inline)) {
        if (nw_k + kLinearK > k_end)
#pragma unroll
            for (int j = 0; j < WL; ++j) wo[j] = nw_k + piece * 8 < k_end ? wo[j] : kOutOfRange;
        nw_s = nw_k < k_end ? (uint32_t)nw_k * 2u : 0u;
        nw_k += kLinearK;
    };
    const uint32_t lds_wave = lds0 + (uint32_t)wave * 1024u;
    auto issue_x = [&](int j, uint32_t buf) __attribute__((always_inline)) {
        dma_load16_any(rsrc_x, xo[j], nx_s, lds_wave + buf * XB + (uint32_t)j * (RPL * 128u));
    };
    auto issue_w = [&](int j, uint32_t buf) __attribute__((always_inline)) {
        dma_load16_any(rsrc_w, wo[j], nw_s, lds_wave + W0 + buf * WB + (uint32_t)j * (RPL * 128u));
    };

    // where this lane's fragments are: row of the block, half of the k-step
    const uint32_t frow = (uint32_t)(lane & 31);
    const uint32_t fx = (uint32_t)(wave_m * (PB * 32)) * 128u + frow * 128u, fw = W0 + (uint32_t)(wave_n * (CB * 32)) * 128u + frow * 128u;
    const uint32_t ft = (uint32_t)((lane >> 5) ^ FC_SWZ(frow)) * 16u;       // (blocks begin at multiples of 32 rows: the exchange is the row's in the block)

    f32x16_t acc[PB][CB];
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[p][b][i] = 0.f;

    constexpr int NM = PB * CB, NR = PB + CB, NS = KK * NM;     // products and fragment reads of a k-step; products of a stage
    constexpr int BAR = NM / 4, BARRIER = (KK - 1) * NM + BAR;  // the barrier of a stage stands before this product of its last k-step, of the stage
    // From barrier to barrier the loads of the next stage's rows of w and then of the stage after next's rows of x go out at even distances: sent for in one
    // go they wait for each other, and the products behind them for the loads.
    constexpr int NL = XL + WL;
    auto issue_at = [&](auto q_c, uint32_t xbuf, uint32_t wbuf) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value, first = (q * NL + NS - 1) / NS, behind = ((q + 1) * NL + NS - 1) / NS;
        each<behind - first>([&](auto e_c) __attribute__((always_inline)) {
            constexpr int l = first + decltype(e_c)::value;
            if constexpr (l < WL) issue_w(l, wbuf);
            else issue_x(l - WL, xbuf);
        });
    };

    advance_x();
    advance_w();
#pragma unroll
    for (int j = 0; j < XL; ++j) issue_x(j, 0);
#pragma unroll
    for (int j = 0; j < WL; ++j) issue_w(j, 0);
    advance_x();
#pragma unroll
    for (int j = 0; j < XL; ++j) issue_x(j, 1);
    wait_vmcnt<XL>();
    __syncthreads();
    advance_x();
    advance_w();
    each<NS - BARRIER>([&](auto q_c) __attribute__((always_inline)) { issue_at(q_c, 2, 1); });

    Frag<DT> wf[2][CB], xf[2][PB];
    // fragment r of a k-step, in the order the products need them: w0, x0, w1, x1 ..
    auto read_frag = [&](int r, int set, uint32_t xbuf, uint32_t wbuf, int kk) __attribute__((always_inline)) {
        const uint32_t o = ((uint32_t)kk * 32u) ^ ft;
        if (r == 1 || r > CB) {
            const int p = r == 1 ? 0 : r - CB;
            xf[set][p].load(smem_raw, o + fx + xbuf * XB + (uint32_t)p * 4096u);
        } else {
            const int b = r == 0 ? 0 : r - 1;
            wf[set][b].load(smem_raw, o + fw + wbuf * WB + (uint32_t)b * 4096u);
        }
    };
#pragma unroll
    for (int r = 0; r < NR; ++r) read_frag(r, 0, 0, 0, 0);
    // stage N of six (three buffers of rows of x, two of w)
    auto stage = [&](auto n_c) __attribute__((always_inline)) {
        constexpr uint32_t N = decltype(n_c)::value, X = N % 3, W = N % 2;
        each<KK>([&](auto kk_c) __attribute__((always_inline)) {
            constexpr int kk = decltype(kk_c)::value;
            constexpr bool last = kk == KK - 1;
            constexpr int from = last ? BAR : 0, gaps = NM - from;
            each<NM>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, t = kk * NM + i;
                if constexpr (t == BARRIER) {       // the next stage has landed (its rows of x before the ones still on their way), everyone has read this one
                    lds_reads_done();
                    wait_vmcnt<XL>();
                    __syncthreads();
                    advance_x();
                    advance_w();
                }
                acc[i / CB][i % CB] = mfma32<DT>(wf[kk & 1][i % CB], xf[kk & 1][i / CB], acc[i / CB][i % CB]);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (i >= from) {
                    constexpr int j = i - from;         // this gap's share of the reads
                    each<((j + 1) * NR + gaps - 1) / gaps - (j * NR + gaps - 1) / gaps>([&](auto e_c) __attribute__((always_inline)) {
                        constexpr int r = (j * NR + gaps - 1) / gaps + decltype(e_c)::value;
                        if constexpr (r < NR) {
                            if constexpr (last) read_frag(r, 0, (X + 1) % 3, W ^ 1u, 0);
                            else read_frag(r, (kk + 1) & 1, X, W, kk + 1);
                        }
                    });
                }
                // (what goes out before the barrier belongs to the last one: stages one and two ahead of this)
                if constexpr (t >= BARRIER) issue_at(std::integral_constant<int, t - BARRIER>{}, X, W);
                else issue_at(std::integral_constant<int, t + NS - BARRIER>{}, (X + 2) % 3, W ^ 1u);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    for (int s = 0; s < stages; s += 6)
        each<6>([&](auto n_c) __attribute__((always_inline)) {
            if (s + decltype(n_c)::value < stages) stage(n_c);
        });
    lds_reads_done();
    wait_vmcnt<0>();
    __syncthreads();

    finish_tile<DT, TO, WM, WN, PB, CB, true, kTileLds<WM, WN, PB, CB>>(a, acc, smem_raw, t, rows, wave, wave_m, wave_n);
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
        const uint4 v = row_end(from, c, a.k);
        *reinterpret_cast<uint4 *>((of_x ? x : w) + row * padded_k + c) = v;
    }
}

hipError_t launch_linear_pad(const LinearArgs &a, const LinearPlan &p, uint16_t *x, uint16_t *w, hipStream_t s)
{
    const int64_t items = ((x ? (int64_t)a.rows : 0) + (w ? a.n : 0)) * (p.padded_k / 8), blocks = (items + 255) / 256;
    k_linear_pad<<<dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s>>>(a, (int32_t)p.padded_k, x, w);
    return hipGetLastError();
}

template <int DT, typename TO, int WM, int WN, int PB, int CB> static hipError_t launch_tile_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = kTileLds<WM, WN, PB, CB>;
    const hipError_t e = raise_dynamic_lds<&k_linear_tile<DT, TO, WM, WN, PB, CB>>(lds);
    if (e != hipSuccess) return e;
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    k_linear_tile<DT, TO, WM, WN, PB, CB><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_tile_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s) { return launch_tile_of<DT, TO, 2, 2, 2, 2>(a, p, s); }

hipError_t launch_linear_tile(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_tile_as<FC_BF16, float>(a, p, s) : launch_tile_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_tile_as<FC_F16, float>(a, p, s) : launch_tile_as<FC_F16, f16_t>(a, p, s);
}

} // namespace fc
