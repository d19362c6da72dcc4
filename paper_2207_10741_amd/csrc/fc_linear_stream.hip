// Matrix product of some dozens of rows: out = act(x w^T + bias) + residual.
//
// The weights' bytes bound it, as with fewer rows, but rows of x are many enough that reading both operands straight into fragments (16 rows of 64 bytes a load) is
// slower than memory: 18 bytes a clock and CU.  So both come in whole 128-byte lines through LDS, D stages of 64 deep, and a workgroup's eight waves share
// the tile.  One barrier a stage: behind it everyone has left the buffer that the loads sent for next go to, and the stage to be multiplied has landed.
// Workgroups divide the reduction where there are fewer tiles than CUs.  128 x 4096 x 4096 20 us (in registers straight from memory 40), 1024 x 4096 x 4096 43.
//
// k_linear_any: rows of any alignment, which cannot go to LDS by themselves.  They come into registers two stages ahead and are written to LDS from there; no operand
// is laid out anew first.
#include "fc_linear_tile.hpp"

namespace fc {

// The products of a stage that lies at `at`.
template <int DT, int PB, int CB>
__device__ __forceinline__ void multiply_stage(f32x16_t (&acc)[PB][CB], const unsigned char *at, uint32_t fx, uint32_t fw, uint32_t ft)
{
    constexpr int KK = 4;
    Frag<DT> xf[KK][PB], wf[KK][CB];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        const uint32_t o = ((uint32_t)kk * 32u) ^ ft;
#pragma unroll
        for (int b = 0; b < CB; ++b) wf[kk][b].load(at, o + fw + (uint32_t)b * 4096u);
#pragma unroll
        for (int p = 0; p < PB; ++p) xf[kk][p].load(at, o + fx + (uint32_t)p * 4096u);
    }
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int p = 0; p < PB; ++p)
#pragma unroll
            for (int b = 0; b < CB; ++b) acc[p][b] = mfma32<DT>(wf[kk][b], xf[kk][p], acc[p][b]);
}
template <int PB, int CB> __device__ __forceinline__ void clear_sums(f32x16_t (&acc)[PB][CB])
{
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[p][b][i] = 0.f;
}

template <int WM, int WN, int PB, int CB, int D> constexpr size_t kStreamLds = (size_t)D * (WM * PB + WN * CB) * 32 * 128;

template <int DT, typename TO, int WM, int WN, int PB, int CB, int D>
__global__ __launch_bounds__(WM * WN * 64, 2)
void k_linear_stream(LinearArgs a)
{
    constexpr int NT = WM * WN * 64, TM = WM * PB * 32, TN = WN * CB * 32;
    constexpr int RPL = NT / 8, XL = TM / RPL, WL = TN / RPL, NL = XL + WL;
    constexpr uint32_t XB = TM * 128u, SB = (TM + TN) * 128u;      // a stage: rows of x, then of w
    static_assert(TM % RPL == 0 && TN % RPL == 0 && RPL % 16 == 0, "whole loads; the exchange is the same for all of a lane's rows");

    extern __shared__ __align__(16) unsigned char smem_raw[];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(smem_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave % WM, wave_n = wave / WM;
    const int rows = rows_there(a);
    const TileOf t = tile_of<TM>(a, rows);
    if (!t.there) return;
    const int r0 = t.tile_m * TM, n0 = t.tile_n * TN;

    const int here = min(rows - r0, TM), cols = min(a.n - n0, TN);
    const u32x4_t rsrc_x = make_rsrc_words(a.x + (int64_t)r0 * a.x_row, (uint32_t)((int64_t)(here - 1) * a.x_row + a.k) * 2u);
    const u32x4_t rsrc_w = make_rsrc_words(a.w + (int64_t)n0 * a.w_row, (uint32_t)((int64_t)(cols - 1) * a.w_row + a.k) * 2u);
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
    const int k0 = t.split * a.per_split * kLinearK, stages = min(a.per_split, (a.k - k0 + kLinearK - 1) / kLinearK);
    const int k_end = min(a.k, k0 + stages * kLinearK);
    int ld_k = k0;
    uint32_t ld_buf = 0;
    const uint32_t lds_wave = lds0 + (uint32_t)wave * 1024u;
    // the next stage is sent for (behind the last one: zeros)
    auto send = [&]() __attribute__((always_inline)) {
        const bool ok = ld_k + piece * 8 < k_end;
        const uint32_t s = ld_k < k_end ? (uint32_t)ld_k * 2u : 0u, to = lds_wave + ld_buf * SB;
#pragma unroll
        for (int j = 0; j < WL; ++j) dma_load16_any(rsrc_w, ok ? wo[j] : kOutOfRange, s, to + XB + (uint32_t)j * (RPL * 128u));
#pragma unroll
        for (int j = 0; j < XL; ++j) dma_load16_any(rsrc_x, ok ? xo[j] : kOutOfRange, s, to + (uint32_t)j * (RPL * 128u));
        ld_k += kLinearK;
        ld_buf = ld_buf + 1 == D ? 0 : ld_buf + 1;
    };
    const uint32_t frow = (uint32_t)(lane & 31), ft = (uint32_t)((lane >> 5) ^ FC_SWZ(frow)) * 16u;
    const uint32_t fx = (uint32_t)(wave_m * (PB * 32)) * 128u + frow * 128u, fw = XB + (uint32_t)(wave_n * (CB * 32)) * 128u + frow * 128u;

    f32x16_t acc[PB][CB];
    clear_sums(acc);
#pragma unroll
    for (int d = 0; d < D - 1; ++d) send();
    uint32_t buf = 0;
    for (int s = 0; s < stages; ++s) {
        lds_reads_done();
        wait_vmcnt<(D - 2) * NL>();
        __syncthreads();
        send();
        multiply_stage<DT, PB, CB>(acc, smem_raw + buf * SB, fx, fw, ft);
        buf = buf + 1 == D ? 0 : buf + 1;
    }
    lds_reads_done();
    wait_vmcnt<0>();
    __syncthreads();
    finish_tile<DT, TO, WM, WN, PB, CB, true, kStreamLds<WM, WN, PB, CB, D>>(a, acc, smem_raw, t, rows, wave, wave_m, wave_n);
}

template <int DT, typename TO, int WM, int WN, int PB, int CB>
__global__ __launch_bounds__(WM * WN * 64, PB == 1 ? 4 : 2)
void k_linear_any(LinearArgs a)
{
    constexpr int NT = WM * WN * 64, TM = WM * PB * 32, TN = WN * CB * 32;
    constexpr int RPL = NT / 8, XL = TM / RPL, WL = TN / RPL, NL = XL + WL;
    constexpr uint32_t XB = TM * 128u, SB = (TM + TN) * 128u;      // a stage: rows of x, then of w; two of them
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave % WM, wave_n = wave / WM;
    const int rows = rows_there(a);
    const TileOf t = tile_of<TM>(a, rows);
    if (!t.there) return;
    const int r0 = t.tile_m * TM, n0 = t.tile_n * TN;
    const int k0 = t.split * a.per_split * kLinearK, stages = min(a.per_split, (a.k - k0 + kLinearK - 1) / kLinearK);
    const int k_end = min(a.k, k0 + stages * kLinearK);
    const int lrow = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ FC_SWZ(lrow)) * 8;
    // (rows and columns that are not there: the last one's again, whose sums nobody stores)
    const uint16_t *from[NL];
#pragma unroll
    for (int j = 0; j < NL; ++j)
        from[j] = j < XL ? a.x + (int64_t)min(r0 + j * RPL + lrow, rows - 1) * a.x_row : a.w + (int64_t)min(n0 + (j - XL) * RPL + lrow, a.n - 1) * a.w_row;
    unsigned char *const to = smem_raw + lrow * 128 + (lane & 7) * 16;
    uint4 r[2][NL];
    auto fetch = [&](int s, auto set) __attribute__((always_inline)) {
        const int c = k0 + s * kLinearK + piece;
        if (k0 + (s + 1) * kLinearK <= k_end) {
#pragma unroll
            for (int j = 0; j < NL; ++j) __builtin_memcpy(&r[decltype(set)::value][j], from[j] + c, 16);
        } else {
#pragma unroll
            for (int j = 0; j < NL; ++j) r[decltype(set)::value][j] = row_end(from[j], c, a.k);     // (only the last stage of the reduction)
        }
    };
    auto put = [&](int buf, auto set) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NL; ++j)
            *reinterpret_cast<uint4 *>(to + buf * SB + (j < XL ? (uint32_t)j * (RPL * 128u) : XB + (uint32_t)(j - XL) * (RPL * 128u))) = r[decltype(set)::value][j];
    };
    const uint32_t frow = (uint32_t)(lane & 31), ft = (uint32_t)((lane >> 5) ^ FC_SWZ(frow)) * 16u;
    const uint32_t fx = (uint32_t)(wave_m * (PB * 32)) * 128u + frow * 128u, fw = XB + (uint32_t)(wave_n * (CB * 32)) * 128u + frow * 128u;
    f32x16_t acc[PB][CB];
    clear_sums(acc);
    typedef std::integral_constant<int, 0> I0;
    typedef std::integral_constant<int, 1> I1;
    fetch(0, I0{});
    if (stages > 1) fetch(1, I1{});
    put(0, I0{});
    if (stages > 2) fetch(2, I0{});
    // stage s: the next one goes from its registers to LDS, the one behind that two further is sent for
    auto stage = [&](int s, auto cur, auto next) __attribute__((always_inline)) {
        lds_reads_done();       // (and writes)
        __syncthreads();
        if (s + 1 < stages) put(decltype(next)::value, next);
        if (s + 3 < stages) fetch(s + 3, next);
        multiply_stage<DT, PB, CB>(acc, smem_raw + decltype(cur)::value * SB, fx, fw, ft);
    };
    for (int s = 0; s < stages; s += 2) {
        stage(s, I0{}, I1{});
        if (s + 1 < stages) stage(s + 1, I1{}, I0{});
    }
    lds_reads_done();
    __syncthreads();
    finish_tile<DT, TO, WM, WN, PB, CB, true, 2 * SB>(a, acc, smem_raw, t, rows, wave, wave_m, wave_n);
}

template <int DT, typename TO, int WM, int WN, int PB, int CB, int D> static hipError_t launch_stream_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    constexpr size_t lds = kStreamLds<WM, WN, PB, CB, D>;
    const hipError_t e = raise_dynamic_lds<&k_linear_stream<DT, TO, WM, WN, PB, CB, D>>(lds);
    if (e != hipSuccess) return e;
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    k_linear_stream<DT, TO, WM, WN, PB, CB, D><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO, int WM, int WN, int PB, int CB> static hipError_t launch_any_of(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    constexpr size_t lds = (size_t)2 * (WM * PB + WN * CB) * 32 * 128;
    k_linear_any<DT, TO, WM, WN, PB, CB><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, typename TO> static hipError_t launch_stream_as(const LinearArgs &a, const LinearPlan &p, hipStream_t s)
{
    if (!p.wide) return p.tile_m == 64 ? launch_any_of<DT, TO, 2, 4, 1, 1>(a, p, s) : launch_any_of<DT, TO, 2, 4, 2, 1>(a, p, s);
    return p.tile_m == 64 ? launch_stream_of<DT, TO, 2, 4, 1, 1, 6>(a, p, s) : launch_stream_of<DT, TO, 2, 4, 2, 1, 4>(a, p, s);
}

hipError_t launch_linear_stream(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_stream_as<FC_BF16, float>(a, p, s) : launch_stream_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_stream_as<FC_F16, float>(a, p, s) : launch_stream_as<FC_F16, f16_t>(a, p, s);
}

} // namespace fc
