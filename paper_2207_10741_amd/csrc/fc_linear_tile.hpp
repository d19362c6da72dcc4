// Pieces shared by the kernels of the matrix product that work in tiles: which tile a workgroup has, joining pieces of the reduction, the epilogue.
#pragma once
#include "fc_layers_internal.hpp"

namespace fc {

// f(integral_constant 0) .. f(integral_constant N - 1)
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

// A workgroup's tile and piece of the reduction.  An XCD (workgroups number 0 .. 7 in turn) takes a run of the tiles, which go down eight tiles of rows before the
// next columns: what its workgroups read at a time is a block of both operands that its L2 holds.
struct TileOf {
    bool there;
    int tile, split, tile_m, tile_n;
};
template <int TM> __device__ __forceinline__ TileOf tile_of(const LinearArgs &a, int rows)
{
    const int m_tiles = (rows + TM - 1) / TM, total = m_tiles * a.n_tiles * a.splits;
    const int xcd = (int)blockIdx.x & 7, first = (int)(((int64_t)total * xcd) >> 3), behind = (int)(((int64_t)total * (xcd + 1)) >> 3);
    const int number = first + ((int)blockIdx.x >> 3);
    TileOf t;
    t.there = number < behind;
    t.split = number % a.splits;
    t.tile = number / a.splits;
    constexpr int GROUP = 8;
    const int group = t.tile / (GROUP * a.n_tiles), in_group = t.tile - group * GROUP * a.n_tiles;
    const int high = max(min(GROUP, m_tiles - group * GROUP), 1);
    t.tile_m = group * GROUP + in_group % high;
    t.tile_n = in_group / high;
    return t;
}

// From a workgroup's sums to the output.  acc: blocks of 32 columns x 32 rows in the order of the 32x32 matrix instructions (a lane: row lane % 32, columns
// 8 (i / 4) + 4 (lane / 32) + i % 4); everyone has left LDS, which holds LDS bytes.
template <int DT, typename TO, int WM, int WN, int PB, int CB, bool SPLIT, size_t LDS>
__device__ __forceinline__ void finish_tile(const LinearArgs &a, f32x16_t (&acc)[PB][CB], unsigned char *smem_raw, const TileOf &t, int rows, int wave, int wave_m, int wave_n)
{
    constexpr int NT = WM * WN * 64;
    const int lane = threadIdx.x & 63, tile = t.tile, split = t.split, r0 = t.tile_m * (WM * PB * 32), n0 = t.tile_n * (WN * CB * 32);
    // ---- pieces of the reduction: written in the registers' order, added by the last workgroup in the pieces' order ----
    if (SPLIT && a.splits > 1) {
        constexpr uint32_t ITEMS = (uint32_t)PB * CB * 4 * NT;     // of four sums
        const auto part = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)tile * a.splits * (ITEMS * 4), 0, (uint32_t)a.splits * ITEMS * 16u, 0x00020000);
        each<PB * CB * 4>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value, q = i % 4 * 4;
            const f32x16_t &s = acc[i / 4 / CB][i / 4 % CB];
            const f32x4_t v = {s[q], s[q + 1], s[q + 2], s[q + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), part, ((uint32_t)split * ITEMS + (uint32_t)i * NT + threadIdx.x) * 16u, 0, kPiecesPastCaches);
        });
        if (!last_piece(a.arrived + tile, a.splits, reinterpret_cast<int32_t *>(smem_raw))) return;
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PB; ++p)
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[p][b][i] = 0.f;
        // (enough of them on their way together: one piece after another is a round trip each)
        constexpr int AT_ONCE = PB * CB >= 4 ? 1 : PB * CB == 2 ? 2 : 4;
        for (int n = 0; n < a.splits; n += AT_ONCE) {
            f32x4_t v[AT_ONCE][PB * CB * 4];
            each<AT_ONCE>([&](auto u_c) __attribute__((always_inline)) {
                each<PB * CB * 4>([&](auto i_c) __attribute__((always_inline)) {
                    constexpr int i = decltype(i_c)::value, u = decltype(u_c)::value;
                    v[u][i] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(part, ((uint32_t)min(n + u, a.splits - 1) * ITEMS + (uint32_t)i * NT + threadIdx.x) * 16u, 0, kPiecesPastCaches));
                });
            });
            each<AT_ONCE>([&](auto u_c) __attribute__((always_inline)) {
                each<PB * CB * 4>([&](auto i_c) __attribute__((always_inline)) {
                    constexpr int i = decltype(i_c)::value, u = decltype(u_c)::value, q = i % 4 * 4;
                    f32x16_t &s = acc[i / 4 / CB][i / 4 % CB];
                    if (n + u < a.splits)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[q + j] += v[u][i][j];
                });
            });
        }
    }

    // ---- epilogue: a wave's blocks of 32 rows go through LDS of its own ----
    // (Sums of 256 registers are accumulators of the matrix instructions; left to itself the compiler copies all of them out at once and spills.  They stay
    // until they are asked for.)
    auto sums_of = [&](auto p_c, auto b_c) __attribute__((always_inline)) -> f32x16_t {
        f32x16_t &s = acc[decltype(p_c)::value][decltype(b_c)::value];
        if constexpr (CB == 4) __asm__ volatile("" : "+a"(s));
        return s;
    };
    const int col0 = n0 + wave_n * (CB * 32), half = lane >> 5;
    if (a.wide_out && a.act <= FC_ACT_RELU) {
        // In the registers' order (a lane: a row, fours of columns): residuals come in and results go out in 16-byte pieces of rows.
        constexpr int PPR = CB * 32 * (int)sizeof(TO) / 16, RPI = 64 / PPR, NI = 32 / RPI;    // pieces a row, rows a round, rounds
        constexpr uint32_t OP = CB * 32 * sizeof(TO) + 16;
        static_assert((size_t)WM * WN * 32 * OP <= LDS, "the waves' shares");
        unsigned char *const os = smem_raw + wave * (32 * OP), *const mine = os + (lane & 31) * OP + half * (4 * sizeof(TO));
        constexpr int EPP = 16 / (int)sizeof(TO);
        const int prow = lane / PPR, pcol = col0 + lane % PPR * EPP;
        unsigned char *const piece_at = os + prow * OP + lane % PPR * 16;
        f32x4_t bias[CB * 4];
        each<CB * 4>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            const int c = col0 + i * 8 + half * 4;
            bias[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (a.bias && c < a.n) bias[i] = *reinterpret_cast<const f32x4_t *>(a.bias + c);
        });
        each<PB>([&](auto p_c) __attribute__((always_inline)) {
            constexpr int p = decltype(p_c)::value;
            const int row0 = r0 + (wave_m * PB + p) * 32 + prow;
            if (a.residual) {
                const TO *from = static_cast<const TO *>(a.residual) + pcol;
                uint4 more[NI];
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    more[i] = make_uint4(0, 0, 0, 0);
                    if (row0 + i * RPI < rows && pcol < a.n) more[i] = *reinterpret_cast<const uint4 *>(from + (int64_t)(row0 + i * RPI) * a.residual_row);
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) *reinterpret_cast<uint4 *>(piece_at + i * RPI * OP) = more[i];
                wave_lds_order();
            }
            const bool relu_first = a.act == FC_ACT_RELU && !a.residual_first, relu_last = a.act == FC_ACT_RELU && a.residual_first;
            each<CB * 4>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, q = i % 4 * 4;
                const f32x16_t s = sums_of(p_c, std::integral_constant<int, i / 4>{});
                f32x4_t v = f32x4_t{s[q], s[q + 1], s[q + 2], s[q + 3]} + bias[i];
                TO *const at = reinterpret_cast<TO *>(mine) + i * 8;
                if (relu_first)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = relu_keep_nan(v[j]);
                if (a.residual) v += load4_float(at);
                if (relu_last)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = relu_keep_nan(v[j]);
                store4<DT, TO>(at, v[0], v[1], v[2], v[3]);
                if constexpr (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (the compiler would copy all sums out of the accumulators first)
            });
            wave_lds_order();
            uint4 done[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) done[i] = *reinterpret_cast<const uint4 *>(piece_at + i * RPI * OP);
            TO *to = static_cast<TO *>(a.out) + pcol;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (row0 + i * RPI < rows && pcol < a.n) *reinterpret_cast<uint4 *>(to + (int64_t)(row0 + i * RPI) * a.out_row) = done[i];
            wave_lds_order();
            __builtin_amdgcn_sched_barrier(0);
        });
        return;
    }
    // Activations with more arithmetic, and rows of any alignment: the sums go through LDS, and loops that are not unrolled finish them.
    constexpr int LPR = CB * 4, RPI = 64 / LPR;      // lanes a row, rows a round, of eight columns
    const int c8 = lane % LPR, col8 = col0 + c8 * 8;
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.wide_out && a.bias && col8 < a.n) load8_float(a.bias + col8, bias);
    constexpr int OP = CB * 32 + 4;     // floats from row to row
    static_assert((size_t)WM * WN * 32 * OP * 4 <= LDS, "the waves' shares");
    float *const os = reinterpret_cast<float *>(smem_raw) + wave * (32 * OP);
    // (A loop over p that is not unrolled would put the sums into memory.)
    each<PB>([&](auto p_c) __attribute__((always_inline)) {
        constexpr int p = decltype(p_c)::value;
        each<CB>([&](auto b_c) __attribute__((always_inline)) {
            const f32x16_t s = sums_of(p_c, b_c);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4_t *>(os + (lane & 31) * OP + decltype(b_c)::value * 32 + q * 8 + half * 4) = f32x4_t{s[q * 4], s[q * 4 + 1], s[q * 4 + 2], s[q * 4 + 3]};
        });
        wave_lds_order();
        const int row0 = r0 + (wave_m * PB + p) * 32, here = min(rows - row0, 32);
        if (a.wide_out) {
            // two rows' residuals are sent for together
            constexpr int AT_ONCE = 2;
#pragma unroll 1
            for (int i = 0; i < 32 / RPI; i += AT_ONCE) {
                float more[AT_ONCE][8];
                if (a.residual)
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int row = min(row0 + (i + u) * RPI + lane / LPR, rows - 1);
                        load8_float(static_cast<const TO *>(a.residual) + row * a.residual_row + (col8 < a.n ? col8 : 0), more[u]);
                    }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int r = (i + u) * RPI + lane / LPR, row = row0 + r;
                    float v[8];
                    load8_float(os + r * OP + c8 * 8, v);
                    finish_eight(a, bias, more[u], v);
                    if (row < rows && col8 < a.n) store8(static_cast<TO *>(a.out) + row * a.out_row + col8, v);
                }
            }
        } else {
            // a lane a column (of fewer than 64 columns: of several rows), eight rows' residuals sent for together
            constexpr int COLS = CB * 32 < 64 ? CB * 32 : 64, ROWS = 64 / COLS, AT_ONCE = 8;
#pragma unroll 1
            for (int c0 = 0; c0 < CB * 32; c0 += COLS) {
                const int c = c0 + lane % COLS, col = col0 + c;
                if (col >= a.n) continue;
                const float add = a.bias ? a.bias[col] : 0.f;
                const TO *const from = static_cast<const TO *>(a.residual) + col;
                TO *const to = static_cast<TO *>(a.out) + col;
#pragma unroll 1
                for (int r = lane / COLS; r < here; r += AT_ONCE * ROWS) {
                    float more[AT_ONCE], v[AT_ONCE];
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) more[u] = a.residual ? to_float(from[(int64_t)(row0 + min(r + u * ROWS, here - 1)) * a.residual_row]) : 0.f;
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) v[u] = os[min(r + u * ROWS, 31) * OP + c] + add;
                    if (a.residual_first)
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) v[u] += more[u];
                    activate_all(v, a.act);
                    if (!a.residual_first)
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) v[u] += more[u];
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u)
                        if (r + u * ROWS < here) from_float(v[u], to + (int64_t)(row0 + r + u * ROWS) * a.out_row);
                }
            }
        }
        wave_lds_order();
    });
}

} // namespace fc
