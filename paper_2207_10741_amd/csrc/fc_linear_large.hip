// Matrix product of many rows in tiles of 256 x 256.
//
// A workgroup of four waves has a tile, a wave 128 x 128 of it: 0.5 KB of LDS reads for the work of 32 x 32 x 16.  What bounds it is the power that the chip may draw, then the
// matrix pipes.  The products are 16x16x32 instructions: a loop of nothing but them holds 2.08 PFLOP/s on values of a normal distribution, one of 32x32x16
// instructions, which read and write twice as many sums for the same work, 1.82.
//
// The reduction goes in stages of 64, rows of x three stages deep in LDS and rows of w two.  Everything that is not a product goes out between two of them, one
// piece at a time: fragments a k-step ahead, across the stage's border too (its barrier stands inside the last k-step), a stage's loads at even distances from
// barrier to barrier.  8192 cubed with 32x32x16 instructions: loads in one go behind the barrier, eight waves, 862 us; spread 815; four waves 794.  With 16x16x32
// instructions 749, and with M0 set a product before its load, so that no gap of 16 clocks holds three instructions, 732; with the epilogue of
// today 715 - 720 (1.53 PFLOP/s; the library's product on the same values 688 - 695): 2315 clocks a stage of which the products take 2048.
#include "fc_linear_tile.hpp"

namespace fc {

__device__ __forceinline__ void aim(uint32_t lds_addr) { __asm__ volatile("s_mov_b32 m0, %0" : : "s"(lds_addr) : "memory"); }
__device__ __forceinline__ void load_aimed(const u32x4_t &rsrc, uint32_t byte_offset, uint32_t scalar_offset)
{
    __asm__ volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" : : "v"(byte_offset), "s"(rsrc), "s"(scalar_offset) : "memory");
}

constexpr int kLargeTile = 256, kLargeThreads = 256;
constexpr int kLoadShift = 1;       // where between two loads' products one stands (0 .. 6: all within 1 %)
constexpr size_t kLargeLds = (size_t)5 * kLargeTile * 128;     // three stages' rows of x, two stages' rows of w

template <int DT, typename TO>
__global__ __launch_bounds__(kLargeThreads, 1)
void k_linear_large(LinearArgs a)
{
    constexpr int NT = kLargeThreads, WM = 2, PB = 8, CB = 8, TM = kLargeTile, TN = kLargeTile;    // a wave: 8 x 8 blocks of 16 x 16
    constexpr int RPL = NT / 8;                     // rows that the waves' loads cover side by side
    constexpr int XL = TM / RPL, WL = TN / RPL, KK = 2;
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
    // A load in two pieces, a product between them, which is the wait state that M0 wants: where it goes (M0, which nothing else here writes), and the load.
    auto aim_x = [&](int j, uint32_t buf) __attribute__((always_inline)) { aim(lds_wave + buf * XB + (uint32_t)j * (RPL * 128u)); };
    auto aim_w = [&](int j, uint32_t buf) __attribute__((always_inline)) { aim(lds_wave + W0 + buf * WB + (uint32_t)j * (RPL * 128u)); };
    auto issue_x = [&](int j, uint32_t buf) __attribute__((always_inline)) {
        dma_load16_any(rsrc_x, xo[j], nx_s, lds_wave + buf * XB + (uint32_t)j * (RPL * 128u));
    };
    auto issue_w = [&](int j, uint32_t buf) __attribute__((always_inline)) {
        dma_load16_any(rsrc_w, wo[j], nw_s, lds_wave + W0 + buf * WB + (uint32_t)j * (RPL * 128u));
    };

    // where this lane's fragments are: row of the block, eighth of the stage (of the second k-step: four further)
    const uint32_t frow = (uint32_t)(lane & 15), ft = ((uint32_t)(lane >> 4) ^ FC_SWZ(frow)) * 16u;    // (blocks begin at multiples of 16 rows)
    const uint32_t fx = (uint32_t)(wave_m * (PB * 16)) * 128u + frow * 128u, fw = W0 + (uint32_t)(wave_n * (CB * 16)) * 128u + frow * 128u;

    f32x4_t acc[PB][CB];
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int b = 0; b < CB; ++b) acc[p][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    constexpr int NM = PB * CB, NR = PB + CB, NS = KK * NM;     // products and fragment reads of a k-step; products of a stage
    constexpr int BAR = 12, BARRIER = NM + BAR;                 // the barrier of a stage stands before this product of its last k-step, of the stage
    // From barrier to barrier the loads of the next stage's rows of w and then of the stage after next's rows of x go out at even distances, at products that no
    // read stands at.
    constexpr int NL = XL + WL, EVERY = NS / NL;
    auto issue_at = [&](auto q_c, uint32_t xbuf, uint32_t wbuf) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value, l = q / EVERY;
        if constexpr (q % EVERY == kLoadShift - 1) {
            if constexpr (l < WL) aim_w(l, wbuf);
            else aim_x(l - WL, xbuf);
        }
        if constexpr (q % EVERY == kLoadShift) {
            if constexpr (l < WL) load_aimed(rsrc_w, wo[l], nw_s);
            else load_aimed(rsrc_x, xo[l - WL], nx_s);
        }
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
    // (those before the first stage's barrier: no product stands between M0's write and a load, which have to be a wait state apart)
    static_assert((NS - BARRIER) % EVERY != kLoadShift, "a load and its place on the same side");
    each<NS - BARRIER>([&](auto q_c) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value, l = q / EVERY;
        if constexpr (q % EVERY == kLoadShift) {
            if constexpr (l < WL) issue_w(l, 1);
            else issue_x(l - WL, 2);
        }
    });

    uint4 wf[2][CB], xf[2][PB];
    // fragment r of a k-step, in the order the products need them: w0, x0, w1 .. w7, x1 ..
    auto read_frag = [&](int r, int set, uint32_t xbuf, uint32_t wbuf, int kk) __attribute__((always_inline)) {
        const uint32_t o = ((uint32_t)kk * 64u) ^ ft;
        if (r == 1 || r > CB) {
            const int p = r == 1 ? 0 : r - CB;
            xf[set][p] = *reinterpret_cast<const uint4 *>(smem_raw + o + fx + xbuf * XB + (uint32_t)p * 2048u);
        } else {
            const int b = r == 0 ? 0 : r - 1;
            wf[set][b] = *reinterpret_cast<const uint4 *>(smem_raw + o + fw + wbuf * WB + (uint32_t)b * 2048u);
        }
    };
#pragma unroll
    for (int r = 0; r < NR; ++r) read_frag(r, 0, 0, 0, 0);
    // stage N of six (three buffers of rows of x, two of w)
    auto stage = [&](auto n_c) __attribute__((always_inline)) {
        constexpr uint32_t N = decltype(n_c)::value, X = N % 3, W = N % 2;
        each<NS>([&](auto t_c) __attribute__((always_inline)) {
            constexpr int t = decltype(t_c)::value, kk = t / NM, i = t % NM;
            if constexpr (t == BARRIER) {       // the next stage has landed (its rows of x before the ones still on their way), everyone has read this one
                lds_reads_done();
                wait_vmcnt<XL>();
                __syncthreads();
                advance_x();
                advance_w();
            }
            acc[i / CB][i % CB] = mfma16_of<DT>(wf[kk][i % CB], xf[kk][i / CB], acc[i / CB][i % CB]);
            __builtin_amdgcn_sched_barrier(0);
            // the reads of the next k-step: one every fourth product, or from the barrier on every third
            if constexpr (kk == 0 && i % 4 == 0) read_frag(i / 4, 1, X, W, 1);
            if constexpr (kk == 1 && i >= BAR && (i - BAR) % 3 == 0 && (i - BAR) / 3 < NR) read_frag((i - BAR) / 3, 0, (X + 1) % 3, W ^ 1u, 0);
            // (what goes out before the barrier belongs to the last one: stages one and two ahead of this)
            if constexpr (t >= BARRIER) issue_at(std::integral_constant<int, t - BARRIER>{}, X, W);
            else issue_at(std::integral_constant<int, t + NS - BARRIER>{}, (X + 2) % 3, W ^ 1u);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    for (int s = 0; s < stages; s += 6)
        each<6>([&](auto n_c) __attribute__((always_inline)) {
            if (s + decltype(n_c)::value < stages) stage(n_c);
        });
    lds_reads_done();
    wait_vmcnt<0>();
    __syncthreads();

    finish_tile<DT, TO, WM, 2, PB, CB, false, kLargeLds>(a, acc, smem_raw, t, rows, wave, wave_m, wave_n);
}

template <int DT, typename TO> hipError_t launch_large_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    const hipError_t e = raise_dynamic_lds<&k_linear_large<DT, TO>>(kLargeLds);
    if (e != hipSuccess) return e;
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
    k_linear_large<DT, TO><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), dim3(kLargeThreads), kLargeLds, s>>>(a);
    return hipGetLastError();
}

// (compiled as several units, one instance each)
#if !defined(FC_LARGE_PART) || FC_LARGE_PART == 0
template hipError_t launch_large_as<FC_BF16, bf16_t>(const LinearArgs &, const LinearPlan &, hipStream_t);
#endif
#if !defined(FC_LARGE_PART) || FC_LARGE_PART == 1
template hipError_t launch_large_as<FC_BF16, float>(const LinearArgs &, const LinearPlan &, hipStream_t);
#endif
#if !defined(FC_LARGE_PART) || FC_LARGE_PART == 2
template hipError_t launch_large_as<FC_F16, f16_t>(const LinearArgs &, const LinearPlan &, hipStream_t);
#endif
#if !defined(FC_LARGE_PART) || FC_LARGE_PART == 3
template hipError_t launch_large_as<FC_F16, float>(const LinearArgs &, const LinearPlan &, hipStream_t);
#endif

} // namespace fc
