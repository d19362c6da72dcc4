// Declarations shared by the attention operators' translation units: the cache's layout, what a sequence's arrays say, conversions.
//
// Layout of the cache.  A unit is one block of one key/value head: unit = pool block * kv_heads + head.
//   codes    [unit][128 * dp] bytes: keys, then values; dp = head_dim rounded up to 64, 96, 128, 192 or 256, zeros behind
//   scales   [unit] of two floats: the keys' scale; the values', negative where a value of the block is NaN
//   sketches [unit][dp rounded up to a multiple of 64] signed bytes (behind dp anything: queries are zeros there), weights [unit] floats
// Keys and values lie in the order in which the matrix instructions want them, so that a load of 16 bytes a lane is 1 KB in one piece.  (The L1 gives
// 65 bytes a clock then, and 18 where sixteen lanes read from rows of 128 bytes, keys as [token][channel].)  A lane of the 16x16 instructions holds
// eight consecutive places of the reduction, lanes 16 apart the next eight (quarter = lane / 16):
//   scores S^T = K q^T: a lane's row is a token, and 16 channels of it are its share of two instructions: pieces
//     [token / 16][channel / 64][channel / 16 % 4][token % 16] of 16 channels.  Of 96 channels the last 32 are one instruction's: the pieces
//     [token / 32][1][channel / 8 % 4][token % 16] hold 8 channels of a token and the same of the token 16 further, between those tokens' first 64 channels
//     [token / 32][0 or 2][channel / 16][token % 16].
//   out^T = V^T P^T: P^T comes out of the first product with tokens 4 quarter + i of each 16 (i = 0 .. 3) in the lane that needs them as operand, so no
//     weight moves between lanes if V's rows are in that order too: token 32 h + 16 k + 4 quarter + i is at place 16 quarter + 8 h + 4 k + i:
//     pieces [channel / 16][place / 16][channel % 16] of 16 places, a lane's share for a whole block.
#pragma once
#include <atomic>
#include "fc_mfma_util.hpp"
#include "focused_attention.h"

namespace fc {

constexpr int kBlock = FC_KV_BLOCK;

struct KvGeom {
    int32_t blocks, kv_heads, d, dp;
    int32_t batch, tokens, max_new, max_len, width;
    uint8_t *codes;
    float2 *scales;
    int8_t *sketches;
    float *weights;
    const int32_t *table, *lengths, *starts;
};

// (96 for the head sizes 65 to 96, which a multiple of 64 would make 128 of: a quarter less to keep, read, convert and multiply; us at 128 -> at 96, pieces of up to 517
// tokens over 5003 with heads of 80 63.1 -> 57.5, lists of 9 blocks with heads of 96 39.5 -> 35.3)
static inline int32_t padded_dim(int32_t d) { return d > 64 && d <= 96 ? 96 : (d + 63) / 64 * 64; }
template <int DP> constexpr int kSketch = (DP + 63) / 64 * 64;

// Byte offsets of the cache's sections and its size.
struct KvLayout {
    size_t scales, sketches, weights, bytes;
};
static inline KvLayout kv_layout(int32_t blocks, int32_t kv_heads, int32_t head_dim)
{
    const size_t units = (size_t)blocks * (size_t)kv_heads, dp = (size_t)padded_dim(head_dim);
    KvLayout l;
    l.scales = units * 2 * kBlock * dp;
    l.sketches = l.scales + align_up(units * sizeof(float2), 256);
    l.weights = l.sketches + align_up(units * ((dp + 63) / 64 * 64), 256);
    l.bytes = l.weights + align_up(units * sizeof(float), 256);
    return l;
}

// Blocks that a sequence's new tokens can touch, at most.
static inline int32_t touched_blocks(const KvGeom &g)
{
    const int32_t n = g.max_new < g.tokens ? g.max_new : g.tokens;
    const int32_t touched = (int32_t)(((int64_t)n + kBlock - 2) / kBlock) + 1, held = (int32_t)(((int64_t)g.max_len + kBlock - 1) / kBlock);
    return touched < held ? touched : held;
}

// A sequence as its arrays describe it, cut to the call's bounds: rows row0 .. row0 + n - 1 are its new tokens, row0 has position pos0
// (negative: rows without a position come first).
struct Sequence {
    int32_t len, n, row0, pos0;
};
__device__ __forceinline__ Sequence sequence_of(const KvGeom &g, int b)
{
    Sequence s;
    s.len = min(max(g.lengths[b], 0), g.max_len);
    if (g.starts) {
        const int32_t from = min(max(g.starts[b], 0), g.tokens), to = min(max(g.starts[b + 1], from), g.tokens);
        s.row0 = from;
        s.n = min(to - from, g.max_new);
    } else {
        s.row0 = b * g.max_new;
        s.n = g.max_new;
    }
    s.pos0 = s.len - s.n;
    return s;
}

// The pool's number of a sequence's block, -1: not there.  (block < width: lengths are cut to the table on the host.)
__device__ __forceinline__ int32_t pool_block(const KvGeom &g, int b, int block)
{
    const int32_t p = g.table[(int64_t)b * g.width + block];
    return (uint32_t)p < (uint32_t)g.blocks ? p : -1;
}

__device__ __forceinline__ int64_t unit_of(const KvGeom &g, int32_t pool, int head) { return (int64_t)pool * g.kv_heads + head; }

// Where a token of its block is in a row of values.
__host__ __device__ __forceinline__ int value_place(int token)
{
    return (token >> 2 & 3) << 4 | (token >> 5) << 3 | (token >> 4 & 1) << 2 | (token & 3);
}

// Offsets in a unit's codes: of a key's channel, and of the piece of 16 bytes that holds a value (place & 15 is its place in the piece).
// Channels c .. c + 7, c a multiple of 8, are next to each other.
template <int DP> __host__ __device__ __forceinline__ uint32_t key_at(uint32_t token, uint32_t channel)
{
    if (DP == 96) {
        const uint32_t pair = (token >> 5) * 3, which = token >> 4 & 1;
        if (channel >= 64) return (((pair + 1) * 4 + (channel >> 3 & 3)) * 16 + (token & 15)) * 16 + which * 8 + (channel & 7);
        return (((pair + which * 2) * 4 + (channel >> 4)) * 16 + (token & 15)) * 16 + (channel & 15);
    }
    return ((((token >> 4) * (DP / 64) + (channel >> 6)) * 4 + (channel >> 4 & 3)) * 16 + (token & 15)) * 16 + (channel & 15);
}
// What half `half` (of 8 channels) of piece `piece` of the keys holds.
struct KeyHalf {
    uint32_t token, channel;
};
template <int DP> __host__ __device__ __forceinline__ KeyHalf key_half(uint32_t piece, uint32_t half)
{
    const uint32_t load = piece >> 6, group = piece >> 4 & 3, token = piece & 15;
    if (DP == 96) {
        const uint32_t nth = load % 3;
        return nth == 1 ? KeyHalf{load / 3 * 32 + half * 16 + token, 64 + group * 8} : KeyHalf{load / 3 * 32 + nth * 8 + token, group * 16 + half * 8};
    }
    return {load / (DP / 64) * 16 + token, load % (DP / 64) * 64 + group * 16 + half * 8};
}
template <int DP> __host__ __device__ __forceinline__ uint32_t value_piece(uint32_t channel, uint32_t place)
{
    return kBlock * DP + (((channel >> 4) * 4 + (place >> 4)) * 16 + (channel & 15)) * 16;
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4_t;

// Eight codes -> eight 16-bit floats, exact in both types (3 bits behind the point, 2^-9 .. 448).
template <int DT> __device__ __forceinline__ uint4 codes_to_16(uint32_t lo, uint32_t hi)
{
    uint4 r;
    if constexpr (DT == FC_BF16) {
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    } else {
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
    }
    return r;
}

template <int DT> __device__ __forceinline__ f32x4_t mfma16(const uint4 &a, const uint4 &b, const f32x4_t &c)
{
    if constexpr (DT == FC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

template <int DT> __device__ __forceinline__ float bits_to_float(uint16_t v)
{
    if constexpr (DT == FC_BF16) return to_float(bf16_t{v});
    else return to_float(f16_t{v});
}
template <int DT> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const f32x2_t v = {a, b};
    if constexpr (DT == FC_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}

// Eight elements c .. c + 7 of a row of d, zeros behind its end.  wide: 16 bytes lie together (d a multiple of 8, the row 16-byte aligned); without a
// branch, so that loads written one after another are under way together.
template <bool WIDE> __device__ __forceinline__ uint4 load8(const uint16_t *__restrict__ row, int c, int d)
{
    if constexpr (WIDE) {
        const uint4 x = *reinterpret_cast<const uint4 *>(row + (c < d ? c : 0));
        return c < d ? x : make_uint4(0, 0, 0, 0);
    }
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t lo = c + 2 * j < d ? row[c + 2 * j] : 0, hi = c + 2 * j + 1 < d ? row[c + 2 * j + 1] : 0;
        v[j] = lo | hi << 16;
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
// The same for code that makes one load at a time.
__device__ __forceinline__ uint4 load8(const uint16_t *__restrict__ row, int c, int d, bool wide) { return wide ? load8<true>(row, c, d) : load8<false>(row, c, d); }

__device__ __forceinline__ float pow2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // -126 <= e <= 127

// The least e with a <= limit * 2^e for a >= 0 that is not infinite; limit_bits: the fraction of the limit, limit_e its exponent.
// (a = 1.f 2^x: x - limit_e, one more where a's fraction is above the limit's.  Subnormals count as zero: far below every bound on e.)
__device__ __forceinline__ int least_exponent(float a, uint32_t limit_fraction, int limit_e)
{
    const uint32_t u = __float_as_uint(a);
    return (int)(u >> 23) - 127 - limit_e + ((u & 0x7fffffu) > limit_fraction ? 1 : 0);
}
// 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
__device__ __forceinline__ int scale_exponent(float amax) { return min(max(least_exponent(amax, 0x600000u, 8), -64), 120); }
__device__ __forceinline__ int unit_exponent(float amax) { return min(max(least_exponent(amax, 0x7e0000u, 6), -126), 120); }

// NaN among the values of a block that some rows see in part: a weight of zero does not silence it in a matrix product.  So the product runs on
// zeros in NaN's place, and a second one, of ones at the NaN and at what a row sees, finds the outputs that are NaN.
// The bytes of four codes that are NaN, as 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t codes)
{
    const uint32_t n = (((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
    return (n << 8) - n;
}
__device__ __forceinline__ uint4 without_nan(const uint4 &x)
{
    return make_uint4(x.x & ~nan_bytes(x.x), x.y & ~nan_bytes(x.y), x.z & ~nan_bytes(x.z), x.w & ~nan_bytes(x.w));
}
// Eight codes -> f16 ones where they are NaN.
__device__ __forceinline__ uint4 nan_marks(uint32_t lo, uint32_t hi)
{
    return codes_to_16<FC_F16>(nan_bytes(lo) & 0x38383838u, nan_bytes(hi) & 0x38383838u);
}
// Two f16 ones: are tokens `first` and the next at most `left`?
__device__ __forceinline__ uint32_t seen_pair(int first, int left) { return (first <= left ? 0x3c00u : 0u) | (first + 1 <= left ? 0x3c000000u : 0u); }

__device__ __forceinline__ uint4 flip_signs(uint4 x, uint32_t signs) { return make_uint4(x.x ^ signs, x.y ^ signs, x.z ^ signs, x.w ^ signs); }

template <int V> struct Const {
    static constexpr int value = V;
};

struct AttnArgs {
    KvGeom kv;
    const uint16_t *q;
    int64_t q_row, q_head;
    uint16_t *out;
    float *lse;
    const int32_t *selected;    // (list form)
    int32_t selected_width;
    int32_t shared, mask_words, entries;    // tokens a wave takes together; words of its LDS for masks and entries
    int32_t heads, group, causal;
    int32_t wide;               // q's rows are 16-byte pieces
    float scale_log2;           // |scale| * log2(e), finite; a negative scale changes the queries' signs
    uint32_t signs;             // of two 16-bit queries
    FastDiv div_group;
    int32_t tiles;              // row tiles of a sequence and key head
    int32_t splits, per_split;  // pieces of the long axis and a piece's blocks
    float *part_out;            // [unit of rows][split][rows][dp], not yet divided by the sum of the weights, in units of kFromSums
    float2 *part_ml;            // [unit of rows][split][rows]: the weights' reference (base 2) and their sum
    int32_t *arrived;           // [unit of rows]: pieces that are done; zero before and after every call
};

// What a block's products of codes with queries are multiplied by.  (Held to the largest finite number: a score of zero stays zero.)
__device__ __forceinline__ float score_factor(const AttnArgs &a, float keys_scale) { return fminf(a.scale_log2 * keys_scale, 0x1.fffffep127f); }

// Where row r of a tile is: its token among the sequence's new ones, its head among the group's.
struct RowPlace {
    int32_t token, head;
};
__device__ __forceinline__ RowPlace row_place(const AttnArgs &a, int row)
{
    const int32_t token = (int32_t)fast_div((uint32_t)row, a.div_group);
    return {token, row - token * a.group};
}

// Sums of weighted values that are not yet divided by the sum of the weights leave a wave in units of 2^56.  They may be 2^46 times the largest value (2^15 a token, 2^31
// tokens, and codes up to 2^9 of scales up to 2^120 come to 2^175), which 32 bits do not hold; in this unit they do, and the least code's part (2^-73) is still far
// above the least normal number.  A power of two: nothing is rounded.
constexpr int kSumsExponent = 56;
constexpr float kFromSums = 0x1p56f;

// Four channels c .. c + 3 of a finished row (head `row` of the output's tokens x heads), not yet divided by the sum of the weights.
template <int DT> __device__ __forceinline__ void finish_row(const AttnArgs &a, int64_t row, int c, f32x4_t sum, float most, float total)
{
    if (a.lse && c == 0) a.lse[row] = total == 0.f ? -__builtin_inff() : (most + __builtin_amdgcn_logf(total)) * 0.693147180559945f;
    const int d = a.kv.d;
    if (c >= d) return;
    const float inverse = total == 0.f ? 0.f : kFromSums / total;     // (nothing to attend to: the sum is zero)
    const uint32_t lo = pack2<DT>(sum[0] * inverse, sum[1] * inverse), hi = pack2<DT>(sum[2] * inverse, sum[3] * inverse);
    uint16_t *const to = a.out + row * d + c;
    if ((d & 3) == 0) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(lo, hi);
    } else {
        const uint16_t v[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < d) to[i] = v[i];
    }
}

// Raises a kernel's limit of dynamic LDS, once per device.
template <auto KERNEL> hipError_t raise_lds(size_t bytes)
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

// Weights are 2^(z - reference), rounded to f16 (11 bits, least step 2^-24) as operands of the matrix instructions; their sum, which the result is divided by, has them in 32 bits.
// Rounding is to nearest, so a row's error is a token's 2^-12 of its weight, and far less of many: below an output's own rounding to bf16, about that to f16.  The
// reference lies kLead below the largest score when it is brought up to date, and that is done when a score is more than kSlack above it: weights are then at
// most 2^15, which f16 holds, and the least that counts is 2^-31 of the largest (with the largest as reference, 2^-24: of 131 000 tokens that one dominates up to
// 2^-8 of the weight were lost, always towards zero).
constexpr float kLead = 7.f, kSlack = 15.f;

// Joining the pieces of a unit of rows.  A workgroup that has written its piece counts itself; the one that comes last reads all pieces (in
// their order, whoever is last) and finishes the rows.  What workgroups of other XCDs wrote is read past the caches (kDeviceScope both ways).
constexpr int kPastCaches = 16;
template <int DP> struct Pieces {
    __amdgpu_buffer_rsrc_t out, ml;
    __device__ __forceinline__ Pieces(const AttnArgs &a, int64_t unit, int rows_tile)
    {
        const uint32_t rows = (uint32_t)(a.splits * rows_tile);
        out = __builtin_amdgcn_make_buffer_rsrc(a.part_out + unit * rows * DP, 0, rows * DP * (uint32_t)sizeof(float), 0x00020000);
        ml = __builtin_amdgcn_make_buffer_rsrc(a.part_ml + unit * rows, 0, rows * (uint32_t)sizeof(float2), 0x00020000);
    }
    // item: split * rows_tile * DP / 4 + the place of four channels of a row, in whichever order the kernel has them together; row: split * rows_tile + row
    __device__ __forceinline__ void put(uint32_t item, f32x4_t v) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), out, item * 16u, 0, kPastCaches);
    }
    __device__ __forceinline__ void put_ml(uint32_t row, float m, float l) const
    {
        const u32x2_t v = {__float_as_uint(m), __float_as_uint(l)};
        __builtin_amdgcn_raw_buffer_store_b64(v, ml, row * 8u, 0, kPastCaches);
    }
    __device__ __forceinline__ f32x4_t get(uint32_t item) const
    {
        return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(out, item * 16u, 0, kPastCaches));
    }
    __device__ __forceinline__ float2 get_ml(uint32_t row) const
    {
        const u32x2_t v = __builtin_amdgcn_raw_buffer_load_b64(ml, row * 8u, 0, kPastCaches);
        return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
    }
};

// Every thread of the workgroup, after its stores of pieces: is this the unit's last workgroup?
__device__ __forceinline__ bool last_to_arrive(const AttnArgs &a, int64_t unit, int active, int32_t *lds_flag)
{
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wave's pieces have been acknowledged ...
    __syncthreads();                                        // ... and the others'
    if (threadIdx.x == 0) {
        const int32_t before = __hip_atomic_fetch_add(a.arrived + unit, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == active - 1) __hip_atomic_store(a.arrived + unit, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *lds_flag = before == active - 1;
    }
    __syncthreads();
    return *lds_flag;
}

// A row's running join: pieces with their references and sums added one by one.
struct Joined {
    f32x4_t o;
    float m, l;
    __device__ __forceinline__ void clear()
    {
        o = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m = -__builtin_inff();
        l = 0.f;
    }
    __device__ __forceinline__ void add(float2 ml, f32x4_t v)
    {
        const float most = fmaxf(m, ml.x), base = most == -__builtin_inff() ? 0.f : most;
        const float f0 = __builtin_amdgcn_exp2f(m - base), f1 = __builtin_amdgcn_exp2f(ml.x - base);
        l = l * f0 + ml.y * f1;
        o = o * f0 + v * f1;
        m = most;
    }
};

// The last workgroup's part: `items` places of four channels of a row; place(item) is the tile's row (kNoRow: none) and the first channel, out_row(row) the
// row's place in the output.  With fewer items than threads a thread takes every so-manyth piece of one, with more several items at once, so that eight
// loads are under way either way.
constexpr int kNoRow = -1;
struct ItemPlace {
    int row, c;
};
template <int DT, int DP, int THREADS, typename P, typename F>
__device__ __forceinline__ void join_pieces(const AttnArgs &a, const Pieces<DP> &pieces, int items, int rows_tile, int active, float *lds, P place, F out_row)
{
    const uint32_t next = (uint32_t)(rows_tile * (DP / 4));     // items from a piece to the next
    if (items > THREADS / 2) {
        constexpr int kItems = 4, kUnroll = 2;
        for (int first = threadIdx.x; first < items; first += kItems * THREADS) {
            Joined x[kItems];
            ItemPlace at[kItems];
            int item[kItems];
#pragma unroll
            for (int n = 0; n < kItems; ++n) {
                x[n].clear();
                item[n] = min(first + n * THREADS, items - 1);
                at[n] = place(item[n]);
            }
            for (int i = 0; i < active; i += kUnroll) {
                float2 ml[kItems][kUnroll];
                f32x4_t v[kItems][kUnroll];
#pragma unroll
                for (int n = 0; n < kItems; ++n)
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u) {
                        const int piece = min(i + u, active - 1);
                        ml[n][u] = pieces.get_ml((uint32_t)(piece * rows_tile + max(at[n].row, 0)));
                        v[n][u] = pieces.get(piece * next + item[n]);
                    }
#pragma unroll
                for (int n = 0; n < kItems; ++n)
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u)
                        if (i + u < active) x[n].add(ml[n][u], v[n][u]);
            }
#pragma unroll
            for (int n = 0; n < kItems; ++n)
                if (first + n * THREADS < items && at[n].row != kNoRow) finish_row<DT>(a, out_row(at[n].row), at[n].c, x[n].o, x[n].m, x[n].l);
        }
        return;
    }
    constexpr int kUnroll = 8;
    const int sets = THREADS / items, item = (int)threadIdx.x % items, set = (int)threadIdx.x / items;
    const ItemPlace at = place(item);
    Joined x;
    x.clear();
    if (set < sets)
        for (int i = set; i < active; i += sets * kUnroll) {
            float2 ml[kUnroll];
            f32x4_t v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int piece = min(i + u * sets, active - 1);
                ml[u] = pieces.get_ml((uint32_t)(piece * rows_tile + max(at.row, 0)));
                v[u] = pieces.get(piece * next + item);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (i + u * sets < active) x.add(ml[u], v[u]);
        }
    __syncthreads();
    float *const mine = lds + threadIdx.x * 8;
    mine[0] = x.m, mine[1] = x.l;
    *reinterpret_cast<f32x4_t *>(mine + 4) = x.o;
    __syncthreads();
    if (set) return;
    for (int i = 1; i < sets; ++i) {
        const float *const other = lds + (i * items + item) * 8;
        x.add(make_float2(other[0], other[1]), *reinterpret_cast<const f32x4_t *>(other + 4));
    }
    if (at.row != kNoRow) finish_row<DT>(a, out_row(at.row), at.c, x.o, x.m, x.l);
}

// max over the lanes 16 and 32 apart
__device__ __forceinline__ float max_over_32(float v)
{
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float max_over_16(float v)
{
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

// Eight codes -> eight f16 values in units of `scale` of them (exact for 2^-4 .. 2^4).
__device__ __forceinline__ uint4 codes_to_f16(uint32_t lo, uint32_t hi, float scale)
{
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true));
    return r;
}

// The exponent of the unit that a running sum of values is held in.  It stays while it is within 16 times the blocks' scales, either way, where every code times
// their ratio is exact in f16 (multiples of 2^-13 up to 7168); else it becomes the block's own scale's and the sum is brought to it.  That is sound while the scales
// so far are not further apart than 2^kUnitSpan: the sum is then below 2^(55 + 64 + 4) of any unit, and the least code at a weight of one above 2^-(9 + 64 + 4).  From
// there on (a block of zeros has the least scale there is, 2^-64) the unit is that of finished sums, and what blocks far from it add is multiplied by their ratio
// in 32 bits.
constexpr int kUnitSpan = 64, kNoUnit = -1024;
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23 & 0xffu) - 127; }      // (whatever its sign)
__device__ __forceinline__ float pow2_held(int e) { return pow2_of(min(max(e, -126), 127)); }       // (finite: a sum of zero stays zero)
struct RunningUnit {
    int e, least, most;     // of the blocks' scales, where they changed the unit
    __device__ __forceinline__ void clear()
    {
        e = kNoUnit;
        least = 1024;
        most = -1024;
    }
    static __device__ __forceinline__ bool far(int scale, int unit) { return scale - unit > 4 || unit - scale > 4; }
    // The unit with a block of this scale's exponent among what is summed.
    __device__ __forceinline__ int with(int scale)
    {
        if (__builtin_expect(!far(scale, e), 1)) return e;
        least = min(least, scale);
        most = max(most, scale);
        return most - least <= kUnitSpan ? scale : kSumsExponent;
    }
    // a sum's factor from this unit to that of finished sums
    __device__ __forceinline__ float to_sums() const { return pow2_held(e - kSumsExponent); }
};

hipError_t launch_kv_append(const KvGeom &g, int dtype, const uint16_t *k, const uint16_t *v, int64_t k_row, int64_t k_head, int64_t v_row,
                            int64_t v_head, bool wide_k, bool wide_v, hipStream_t s);
hipError_t launch_kv_read(const KvGeom &g, float *k, float *v, hipStream_t s);

// Few rows (see fc_attn_rows.hip); rows_tile: rows a workgroup holds, 16 or 32; waves: its waves, 4 or (16 rows of up to 128 channels) 8.
hipError_t launch_attend_rows(const AttnArgs &a, int dtype, int rows_tile, int waves, hipStream_t s);
// Rows of one token, over its list of blocks; a wave's (of a.shared tokens, over all of theirs), or (a.splits counts the pieces) a workgroup's.
constexpr int kSharedMaxBlocks = 2048;                                  // of a sequence: masks and entries fit a wave's share of LDS
constexpr int kSharedMaxWords = kSharedMaxBlocks / 2 + kSharedMaxBlocks;
hipError_t launch_attend_lists(const AttnArgs &a, int dtype, bool whole, hipStream_t s);

// Many rows (see fc_attn_tile.hip); rows_tile: rows a workgroup holds, 128 or (up to 128 channels) 256.
hipError_t launch_attend_tile(const AttnArgs &a, int dtype, int rows_tile, hipStream_t s);

// The selection (see fc_attn_select.hip).
constexpr int kSelectMaxBlocks = 32768;     // blocks of a sequence whose scores fit LDS
constexpr int kMostGroup = 32767;           // heads of a group whose rounded queries' sum fits three signed 8-bit digits: 255 * 32767 <= 127 * (65536 + 256 + 1)
// Scores of a token in LDS, and tokens a workgroup: as many as their scores have room in LDS; single tokens alone (1024 threads, else 256).
static inline int32_t select_stride(const KvGeom &g) { return (int32_t)align_up((size_t)(g.max_len + kBlock - 1) / kBlock, 16); }
static inline int32_t select_tokens(const KvGeom &g)
{
    const int32_t stride = select_stride(g);
    return g.max_new == 1 || stride > 8192 ? 1 : stride > 2048 ? 4 : 16;
}
// clear, n_clear: counters that the attention behind it wants zero.
hipError_t launch_select(const KvGeom &g, int dtype, const uint16_t *q, int64_t q_row, int64_t q_head, int heads, bool wide, int first, int last,
                         int top, int32_t *selected, int32_t *clear, int32_t n_clear, hipStream_t s);

} // namespace fc
