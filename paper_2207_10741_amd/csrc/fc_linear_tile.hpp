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

// From a workgroup's sums to the output.  acc: blocks in the order of the matrix instructions, 32 columns x 32 rows (a lane: row lane % 32, columns
// 8 (i / 4) + 4 (lane / 32) + i % 4) or 16 x 16 (row lane % 16, columns 4 (lane / 16) + i); everyone has left LDS, which holds LDS bytes.
template <int DT, typename TO, int WM, int WN, int PB, int CB, bool SPLIT, size_t LDS, typename V>
__device__ __forceinline__ void finish_tile(const LinearArgs &a, V (&acc)[PB][CB], unsigned char *smem_raw, const TileOf &t, int rows, int wave, int wave_m, int wave_n)
{
    constexpr int NT = WM * WN * 64, BS = sizeof(V) == 64 ? 32 : 16, CW = CB * BS;         // a block's side; a wave's columns
    constexpr int FOURS = BS == 32 ? 4 : 1, NF = CB * FOURS, CF = BS == 32 ? 8 : 16;        // a lane's fours of columns in a block and in a row of blocks; from one to the next
    const int lane = threadIdx.x & 63, tile = t.tile, split = t.split, r0 = t.tile_m * (WM * PB * BS), n0 = t.tile_n * (WN * CW);
    // ---- pieces of the reduction: written in the registers' order, added by the last workgroup in the pieces' order ----
    if (SPLIT && a.splits > 1) {
        constexpr uint32_t ITEMS = (uint32_t)PB * NF * NT;     // of four sums
        const auto part = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)tile * a.splits * (ITEMS * 4), 0, (uint32_t)a.splits * ITEMS * 16u, 0x00020000);
        each<PB * NF>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value, q = i % FOURS * 4;
            const V &s = acc[i / FOURS / CB][i / FOURS % CB];
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
                for (int i = 0; i < FOURS * 4; ++i) acc[p][b][i] = 0.f;
        // (enough of them on their way together: one piece after another is a round trip each)
        constexpr int AT_ONCE = PB * NF >= 16 ? 1 : PB * NF == 8 ? 2 : 4;
        for (int n = 0; n < a.splits; n += AT_ONCE) {
            f32x4_t v[AT_ONCE][PB * NF];
            each<AT_ONCE>([&](auto u_c) __attribute__((always_inline)) {
                each<PB * NF>([&](auto i_c) __attribute__((always_inline)) {
                    constexpr int i = decltype(i_c)::value, u = decltype(u_c)::value;
                    v[u][i] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(part, ((uint32_t)min(n + u, a.splits - 1) * ITEMS + (uint32_t)i * NT + threadIdx.x) * 16u, 0, kPiecesPastCaches));
                });
            });
            each<AT_ONCE>([&](auto u_c) __attribute__((always_inline)) {
                each<PB * NF>([&](auto i_c) __attribute__((always_inline)) {
                    constexpr int i = decltype(i_c)::value, u = decltype(u_c)::value, q = i % FOURS * 4;
                    V &s = acc[i / FOURS / CB][i / FOURS % CB];
                    if (n + u < a.splits)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[q + j] += v[u][i][j];
                });
            });
        }
    }

    // ---- epilogue: a wave's rows of blocks go through LDS of its own ----
    // (Sums of 256 registers are accumulators of the matrix instructions; left to itself the compiler copies all of them out at once and spills.  They stay
    // until they are asked for.)
    auto sums_of = [&](auto p_c, auto b_c) __attribute__((always_inline)) -> V {
        V &s = acc[decltype(p_c)::value][decltype(b_c)::value];
        if constexpr (PB * CB * sizeof(V) >= 1024) __asm__ volatile("" : "+a"(s));
        return s;
    };
    const int col0 = n0 + wave_n * CW, lrow = lane % BS, part4 = lane / BS * 4;
    // Residuals come in 16-byte pieces of rows, those of all blocks together where there are registers for them (block after block each waits for memory: 8192 x 64 x 8192
    // 82 us, so 78).
    constexpr int PPR = CW * (int)sizeof(TO) / 16, RPP = 64 / PPR, NI = BS / RPP;    // pieces a row, rows a round, rounds
    constexpr bool AHEAD = PB * NI <= 32;
    const int prow = lane / PPR, pcol = col0 + lane % PPR * (16 / (int)sizeof(TO));
    auto residual_piece = [&](int p, int i) __attribute__((always_inline)) {
        const int row = r0 + (wave_m * PB + p) * BS + prow + i * RPP;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows && pcol < a.n) v = *reinterpret_cast<const uint4 *>(static_cast<const TO *>(a.residual) + (int64_t)row * a.residual_row + pcol);
        return v;
    };
    uint4 ahead[AHEAD ? PB : 1][NI];
    if (AHEAD && a.wide_out && a.residual)
        each<AHEAD ? PB : 0>([&](auto p_c) __attribute__((always_inline)) {
            each<NI>([&](auto i_c) __attribute__((always_inline)) { ahead[decltype(p_c)::value][decltype(i_c)::value] = residual_piece(decltype(p_c)::value, decltype(i_c)::value); });
        });
    if (a.wide_out && a.act <= FC_ACT_RELU) {
        // In the registers' order (a lane: a row, fours of columns): residuals come in and results go out through LDS.
        constexpr uint32_t OP = CW * sizeof(TO) + 16;
        static_assert((size_t)WM * WN * BS * OP <= LDS, "the waves' shares");
        unsigned char *const os = smem_raw + wave * (BS * OP), *const mine = os + lrow * OP + part4 * sizeof(TO);
        unsigned char *const piece_at = os + prow * OP + lane % PPR * 16;
        f32x4_t bias[NF];
        each<NF>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            const int c = col0 + i * CF + part4;
            bias[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (a.bias && c < a.n) bias[i] = *reinterpret_cast<const f32x4_t *>(a.bias + c);
        });
        each<PB>([&](auto p_c) __attribute__((always_inline)) {
            constexpr int p = decltype(p_c)::value;
            const int row0 = r0 + (wave_m * PB + p) * BS + prow;
            if (a.residual) {
                uint4 more[NI];
                each<NI>([&](auto i_c) __attribute__((always_inline)) {
                    constexpr int i = decltype(i_c)::value;
                    if constexpr (AHEAD) more[i] = ahead[p][i];
                    else more[i] = residual_piece(p, i);
                });
#pragma unroll
                for (int i = 0; i < NI; ++i) *reinterpret_cast<uint4 *>(piece_at + i * RPP * OP) = more[i];
                wave_lds_order();
            }
            const bool relu_first = a.act == FC_ACT_RELU && !a.residual_first, relu_last = a.act == FC_ACT_RELU && a.residual_first;
            each<NF>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, q = i % FOURS * 4;
                const V s = sums_of(p_c, std::integral_constant<int, i / FOURS>{});
                f32x4_t v = f32x4_t{s[q], s[q + 1], s[q + 2], s[q + 3]} + bias[i];
                TO *const at = reinterpret_cast<TO *>(mine) + i * CF;
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
            for (int i = 0; i < NI; ++i) done[i] = *reinterpret_cast<const uint4 *>(piece_at + i * RPP * OP);
            TO *to = static_cast<TO *>(a.out) + pcol;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (row0 + i * RPP < rows && pcol < a.n) *reinterpret_cast<uint4 *>(to + (int64_t)(row0 + i * RPP) * a.out_row) = done[i];
            wave_lds_order();
            __builtin_amdgcn_sched_barrier(0);
        });
        return;
    }
    // Activations with more arithmetic, and rows of any alignment: the sums go through LDS, and loops that are not unrolled finish them.
    constexpr int LPR = CW / 8, RPI = 64 / LPR;      // lanes a row, rows a round, of eight columns
    const int c8 = lane % LPR, col8 = col0 + c8 * 8;
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.wide_out && a.bias && col8 < a.n) load8_float(a.bias + col8, bias);
    constexpr int OP = CW + 4;     // floats from row to row
    static_assert((size_t)WM * WN * BS * OP * 4 <= LDS, "the waves' shares");
    float *const os = reinterpret_cast<float *>(smem_raw) + wave * (BS * OP);
    // (A loop over p that is not unrolled would put the sums into memory.)
    each<PB>([&](auto p_c) __attribute__((always_inline)) {
        constexpr int p = decltype(p_c)::value;
        each<CB>([&](auto b_c) __attribute__((always_inline)) {
            const V s = sums_of(p_c, b_c);
#pragma unroll
            for (int q = 0; q < FOURS; ++q)
                *reinterpret_cast<f32x4_t *>(os + lrow * OP + decltype(b_c)::value * BS + q * CF + part4) = f32x4_t{s[q * 4], s[q * 4 + 1], s[q * 4 + 2], s[q * 4 + 3]};
        });
        wave_lds_order();
        const int row0 = r0 + (wave_m * PB + p) * BS, here = min(rows - row0, BS);
        if (a.wide_out) {
            // (a lane's eight columns are a piece of 16-bit values; by way of LDS, as the loop is not unrolled)
            constexpr int AT_ONCE = 2;
            constexpr bool PIECES = AHEAD && sizeof(TO) == 2 && (size_t)WM * WN * (BS * OP * 4 + NI * 1024) <= LDS;
            unsigned char *const pieces = smem_raw + WM * WN * BS * OP * 4 + wave * (NI * 1024) + lane * 16;
            if constexpr (PIECES) {
                if (a.residual) each<NI>([&](auto i_c) __attribute__((always_inline)) { *reinterpret_cast<uint4 *>(pieces + decltype(i_c)::value * 1024) = ahead[p][decltype(i_c)::value]; });
                wave_lds_order();
            }
#pragma unroll 1
            for (int i = 0; i < BS / RPI; i += AT_ONCE) {
                float more[AT_ONCE][8];
                if (!PIECES && a.residual)
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
                    if constexpr (PIECES)
                        if (a.residual) unpack8<TO>(*reinterpret_cast<const uint4 *>(pieces + (i + u) * 1024), more[u]);
                    finish_eight(a, bias, more[u], v);
                    if (row < rows && col8 < a.n) store8(static_cast<TO *>(a.out) + row * a.out_row + col8, v);
                }
            }
        } else {
            // a lane a column (of fewer than 64 columns: of several rows), many rows' residuals sent for together
            constexpr int COLS = CW < 64 ? CW : 64, ROWS = 64 / COLS, AT_ONCE = BS / ROWS < 16 ? BS / ROWS : 16;
#pragma unroll 1
            for (int c0 = 0; c0 < CW; c0 += COLS) {
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
                    for (int u = 0; u < AT_ONCE; ++u) v[u] = os[min(r + u * ROWS, BS - 1) * OP + c] + add;
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
