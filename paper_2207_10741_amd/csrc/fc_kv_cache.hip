// The key/value cache in 8 bits: appending tokens and reading them back.
//
// k_kv_append: a workgroup takes one block of one head that new tokens of a sequence fall into: it reads their rows, finds the largest magnitude,
// makes the scale, and writes codes.  Bound by memory: 4 bytes read and 2 written a channel of a token.
// k_kv_append_one: a sequence's single new token; a wave takes a head, so that a step of a batch is one round of waves without a barrier.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

constexpr int kThreads = 256;

struct AppendArgs {
    KvGeom kv;
    const uint16_t *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    int32_t wide_k, wide_v;
};

// Four codes under another scale; ratio = old scale / new scale, a power of two.
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float ratio)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(c, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8(c, 1) * ratio, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(c, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8(c, 3) * ratio, r, true);
}

__device__ __forceinline__ void rescale16(uint4 *p, float ratio)
{
    const uint4 x = *p;
    *p = make_uint4(rescale4(x.x, ratio), rescale4(x.y, ratio), rescale4(x.z, ratio), rescale4(x.w, ratio));
}

// Adds eight codes, NaN as zero.
__device__ __forceinline__ void add_codes(uint2 x, float (&sum)[8])
{
    const float f[8] = {__builtin_amdgcn_cvt_f32_fp8(x.x, 0), __builtin_amdgcn_cvt_f32_fp8(x.x, 1), __builtin_amdgcn_cvt_f32_fp8(x.x, 2),
                        __builtin_amdgcn_cvt_f32_fp8(x.x, 3), __builtin_amdgcn_cvt_f32_fp8(x.y, 0), __builtin_amdgcn_cvt_f32_fp8(x.y, 1),
                        __builtin_amdgcn_cvt_f32_fp8(x.y, 2), __builtin_amdgcn_cvt_f32_fp8(x.y, 3)};
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += f[j] == f[j] ? f[j] : 0.f;
}

// A channel's sum of codes in units of 2^-9, as a sketch holds it under 2^e.
__device__ __forceinline__ int8_t sketch_of(int sum, int e) { return (int8_t)(int)__builtin_rintf((float)sum * (pow2_of(-e) * (1.f / 512.f))); }

// A unit's codes in LDS: the pieces of every 256 bytes are exchanged by the number of the 256, or the accesses that step by 256 would meet in one bank.
__device__ __forceinline__ uint32_t in_image(uint32_t offset) { return offset ^ (offset >> 4 & 0xf0u); }

// A value in units of its scale; what is not finite becomes NaN.
__device__ __forceinline__ float code_of(float v, float inverse)
{
    v *= inverse;
    return __builtin_fabsf(v) <= 448.f ? v : __builtin_nanf("");
}

__device__ __forceinline__ float max_over_workgroup(float v, float *scratch)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3]));
    __syncthreads();
    return v;
}

// Magnitudes of 16-bit floats are in the order of their bits without the sign.
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u16x2_t largest_bits(const uint4 &x, u16x2_t most)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, w[j] & 0x7fff7fffu));
    return most;
}

// The same of the finite ones; the others become NaN.
template <uint32_t INFINITY_BITS> __device__ __forceinline__ u16x2_t finite_bits(uint4 &x, u16x2_t most)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t counts = 0;
#pragma unroll
        for (int half = 0; half < 32; half += 16) {
            const uint32_t bits = w[j] >> half & 0x7fffu;
            if (bits >= INFINITY_BITS) w[j] |= 0x7fffu << half;
            else counts |= bits << half;
        }
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, counts));
    }
    x = make_uint4(w[0], w[1], w[2], w[3]);
    return most;
}

// The larger half of each over the workgroup: the first in the lower half, the second in the upper one.
__device__ __forceinline__ uint32_t max_bits_over_workgroup(u16x2_t first, u16x2_t second, float *scratch)
{
    u16x2_t m = __builtin_elementwise_max(u16x2_t{first.x, second.x}, u16x2_t{first.y, second.y});
#pragma unroll
    for (int i = 32; i; i >>= 1) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, __shfl_xor(__builtin_bit_cast(int, m), i)));
    uint32_t *const waves = reinterpret_cast<uint32_t *>(scratch);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = __builtin_bit_cast(uint32_t, m);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, waves[i]));
    __syncthreads();
    return __builtin_bit_cast(uint32_t, m);
}

// Eight values in units of their scale: 448 at most, or NaN.
template <int DT> __device__ __forceinline__ void scaled8(const uint4 &x, float inverse, float (&out)[8])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        out[2 * j] = bits_to_float<DT>((uint16_t)w[j]) * inverse;
        out[2 * j + 1] = bits_to_float<DT>((uint16_t)(w[j] >> 16)) * inverse;
    }
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// A block is a workgroup's because its scale needs its largest magnitude first: the rows are read once into registers and converted from there.
// Magnitudes are compared two at a time as whole numbers, and codes come out of the conversions in the order that they are stored in: in 32-bit floats and byte by
// byte the vector unit was the bound (append and read of 15 000 tokens of six sequences, 8 heads of 128, the same inputs again and again: 59.8 us, now 50.0).  Heads are
// next to each other in the grid, as their rows are in memory (then 46.4).
// The kernel alone, on inputs that change: 31 us for 92 MB read and written, 2.9 TB/s (the same inputs: 22 us): memory, and the phases of a workgroup (read, magnitude,
// convert, write), which overlap with others' only.
// A thread holds channels 8 c .. 8 c + 7 of four consecutive tokens 4 r .. 4 r + 3 at a time: four tokens are one word of a row of values.
template <int DT, int DP> __global__ __launch_bounds__(kThreads) void k_kv_append(AppendArgs a)
{
    constexpr int kChunks = DP / 8, kRows = kThreads / kChunks * 4, kRounds = (kBlock + kRows - 1) / kRows;
    __shared__ float scratch[4];
    __shared__ __align__(16) uint8_t image[2 * kBlock * DP];        // the unit's codes: new tokens' (of a block that is begun, all)
    __shared__ int sums[DP];
    const KvGeom &g = a.kv;
    const int b = blockIdx.z, h = blockIdx.x % (uint32_t)g.kv_heads, nth = blockIdx.x / (uint32_t)g.kv_heads;
    const Sequence s = sequence_of(g, b);
    const int from = max(s.pos0, 0);                        // first new position
    const int block = from / kBlock + nth;
    const int at = block * kBlock;
    if (at >= s.len || from >= s.len) return;
    const int32_t pool = pool_block(g, b, block);
    if (pool < 0) return;
    const int old = min(max(from - at, 0), kBlock), end = min(s.len - at, kBlock);    // new tokens of the block: old .. end - 1
    const int64_t unit = unit_of(g, pool, h);
    uint8_t *const unit_codes = g.codes + unit * (2 * kBlock * DP);
    const int c = threadIdx.x % kChunks, r = threadIdx.x / kChunks;

    uint4 kx[kRounds][4], vx[kRounds][4];
    // (all loads under way together: rows that are not new ones repeat one that is, and count as zeros below)
    auto bring = [&](auto wide, const uint16_t *x, int64_t x_row, uint4 (&to)[kRounds][4]) {
        constexpr bool kWide = decltype(wide)::value;
#pragma unroll
        for (int round = 0; round < kRounds; ++round)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = min(max(round * kRows + 4 * r + j, old), end - 1);
                to[round][j] = load8<kWide>(x + (int64_t)(s.row0 + (at + t - s.pos0)) * x_row, 8 * c, g.d);
            }
    };
    const uint16_t *const krows = a.k + h * a.k_head, *const vrows = a.v + h * a.v_head;
    if (a.wide_k & a.wide_v) {
        bring(Const<true>(), krows, a.k_row, kx);
        bring(Const<true>(), vrows, a.v_row, vx);
    } else {
        bring(Const<false>(), krows, a.k_row, kx);
        bring(Const<false>(), vrows, a.v_row, vx);
    }
    u16x2_t most_k = {0, 0}, most_v = {0, 0};
#pragma unroll
    for (int round = 0; round < kRounds; ++round)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = round * kRows + 4 * r + j;
            if (4 * r >= kRows || t < old || t >= end) kx[round][j] = vx[round][j] = make_uint4(0, 0, 0, 0);
            most_k = largest_bits(kx[round][j], most_k);
            most_v = largest_bits(vx[round][j], most_v);
        }
    uint32_t bits = max_bits_over_workgroup(most_k, most_v, scratch);
    constexpr uint32_t kInfinity = DT == FC_BF16 ? 0x7f80u : 0x7c00u;
    bool strange = bits >> 16 >= kInfinity;
    if (strange || (bits & 0xffffu) >= kInfinity) {         // what is not finite becomes NaN, and the scale is the others'
        most_k = most_v = u16x2_t{0, 0};
#pragma unroll
        for (int round = 0; round < kRounds; ++round)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                most_k = finite_bits<kInfinity>(kx[round][j], most_k);
                most_v = finite_bits<kInfinity>(vx[round][j], most_v);
            }
        bits = max_bits_over_workgroup(most_k, most_v, scratch);
    }
    const float ka = bits_to_float<DT>((uint16_t)bits), va = bits_to_float<DT>((uint16_t)(bits >> 16));
    float ks = pow2_of(scale_exponent(ka)), vs = pow2_of(scale_exponent(va));
    if (old) {
        const float2 was = g.scales[unit];
        const float was_v = __builtin_fabsf(was.y);
        strange |= was.y < 0.f;
        ks = fmaxf(ks, was.x);
        vs = fmaxf(vs, was_v);
        // (of tokens that are not there nothing is read)
        if (ks != was.x)
            for (int i = threadIdx.x; i < kBlock * (DP / 16); i += kThreads) rescale16(reinterpret_cast<uint4 *>(unit_codes) + i, was.x / ks);
        if (vs != was_v)
            for (int i = threadIdx.x; i < kBlock * (DP / 16); i += kThreads) rescale16(reinterpret_cast<uint4 *>(unit_codes + kBlock * DP) + i, was_v / vs);
        __syncthreads();        // (the scales have been read, and pieces are rewritten by other threads below)
    }
    if (threadIdx.x == 0) g.scales[unit] = make_float2(ks, strange ? -vs : vs);

    const float ki = 1.f / ks, vi = 1.f / vs;
    uint2 codes[kRounds][4];
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = round * kRows + 4 * r + j;
            float k[8];
            scaled8<DT>(kx[round][j], ki, k);
            codes[round][j] = make_uint2(codes4(k[0], k[1], k[2], k[3]), codes4(k[4], k[5], k[6], k[7]));
            if (4 * r < kRows && t < kBlock) *reinterpret_cast<uint2 *>(image + in_image(key_at<DP>(t, 8 * c))) = codes[round][j];
        }
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) scaled8<DT>(vx[round][j], vi, v[j]);
        uint32_t column[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) column[i] = codes4(v[0][i], v[1][i], v[2][i], v[3][i]);
        const int t0 = round * kRows + 4 * r;
        if (4 * r < kRows && t0 < kBlock)
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint32_t *>(image + in_image(value_piece<DP>(8 * c + i, value_place(t0))) + (value_place(t0) & 15)) = column[i];
    }
    __syncthreads();
    // A block that is begun is written whole, so that no place of it holds a NaN that its scale does not tell of; else the old tokens keep their bytes.
    for (int i = threadIdx.x; i < 2 * kBlock * (DP / 16); i += kThreads) {
        uint4 *const p = reinterpret_cast<uint4 *>(unit_codes) + i;
        const uint4 fresh = *reinterpret_cast<const uint4 *>(image + in_image(16 * i));
        if (old == 0) {
            *p = fresh;
        } else if (i < kBlock * (DP / 16)) {
            const int t0 = (int)key_half<DP>(i, 0).token, t1 = (int)key_half<DP>(i, 1).token;
            const bool first = t0 >= old && t0 < end, second = t1 >= old && t1 < end;
            if (first && second) *p = fresh;
            else if (first) reinterpret_cast<uint2 *>(p)[0] = make_uint2(fresh.x, fresh.y);
            else if (second) reinterpret_cast<uint2 *>(p)[1] = make_uint2(fresh.z, fresh.w);
        } else {
            uint32_t take[4];                               // four words of four tokens
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int t0 = 16 * w + 4 * (i >> 4 & 3);
                take[w] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) take[w] |= t0 + j >= old && t0 + j < end ? 0xffu << (8 * j) : 0u;
            }
            if (take[0] | take[1] | take[2] | take[3]) {
                const uint4 had = *p;
                *p = make_uint4((had.x & ~take[0]) | (fresh.x & take[0]), (had.y & ~take[1]) | (fresh.y & take[1]),
                                (had.z & ~take[2]) | (fresh.z & take[2]), (had.w & ~take[3]) | (fresh.w & take[3]));
            }
        }
    }

    if (end < kBlock) return;
    // The block is full: its sketch.  Codes are multiples of 2^-9 below 2^9, so their sums over 64 tokens are whole numbers below 2^24 in those units.
    // A block that was begun by this call has its codes in registers.
    for (int i = threadIdx.x; i < DP; i += kThreads) sums[i] = 0;
    __syncthreads();
    if (old == 0) {
        if (4 * r < kRows) {
            float sum[8] = {};
#pragma unroll
            for (int round = 0; round < kRounds; ++round)
#pragma unroll
                for (int j = 0; j < 4; ++j) add_codes(codes[round][j], sum);    // (rows past the block are zero)
#pragma unroll
            for (int j = 0; j < 8; ++j) atomicAdd(&sums[8 * c + j], (int)(sum[j] * 512.f));
        }
    } else {
        for (int i = threadIdx.x; i < kBlock * kChunks; i += kThreads) {
            const int channel = i % kChunks * 8;
            float sum[8] = {};
            add_codes(*reinterpret_cast<const uint2 *>(unit_codes + key_at<DP>(i / kChunks, channel)), sum);
#pragma unroll
            for (int j = 0; j < 8; ++j) atomicAdd(&sums[channel + j], (int)(sum[j] * 512.f));
        }
    }
    __syncthreads();
    float most = 0.f;
    for (int i = threadIdx.x; i < DP; i += kThreads) most = fmaxf(most, __builtin_fabsf((float)sums[i]));
    most = max_over_workgroup(most, scratch);
    const int e = unit_exponent(most * (1.f / 512.f));
    for (int i = threadIdx.x; i < DP; i += kThreads) g.sketches[unit * kSketch<DP> + i] = sketch_of(sums[i], e);
    if (threadIdx.x == 0) g.weights[unit] = ks * pow2_of(e) * (1.f / kBlock);
}

// A wave a head: no barrier, and the largest magnitude is a reduction over lanes.  Bound by latency: one sequence, 8 heads of 128: 3.4 us, two round trips (scale, codes).
// 256 sequences whose tokens fall anywhere: 15.7 us, which is the time of the slowest waves, the few that write a block's 64th token (its keys are read back a byte a
// lane) or whose token raises a scale (the block is rounded again).  All tokens in the middle of their blocks: 8.4 us, first of a block 8.8, 64th 25, all raising 24.  (A
// token's 128 values are bytes of pieces of their own in eight runs of 256 bytes: 16 lines, some 8 MB read and written by 2048 waves, 2 us of memory's time.)
// A wave's lane holds channels kEach * lane on (of 96 channels, 48 lanes do).
template <int DT, int DP> __global__ __launch_bounds__(kThreads) void k_kv_append_one(AppendArgs a)
{
    constexpr int kEach = (DP + 63) / 64;
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63;
    const uint32_t at = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    if (b >= g.batch) return;
    const Sequence s = sequence_of(g, b);
    if (s.n != 1 || s.len <= 0) return;
    const int token = s.len - 1, old = token % kBlock;
    const uint16_t *const krow = a.k + s.row0 * a.k_row + h * a.k_head, *const vrow = a.v + s.row0 * a.v_row + h * a.v_head;
    float kv[kEach], vv[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int c = lane * kEach + i;
        kv[i] = c < g.d ? bits_to_float<DT>(krow[c]) : 0.f;
        vv[i] = c < g.d ? bits_to_float<DT>(vrow[c]) : 0.f;
    }
    const int32_t pool = pool_block(g, b, token / kBlock);
    if (pool < 0) return;
    const int64_t unit = unit_of(g, pool, h);
    uint8_t *const unit_codes = g.codes + unit * (2 * kBlock * DP);
    const float2 was = old ? g.scales[unit] : make_float2(0.f, 0.f);
    float ka = 0.f, va = 0.f;
    bool strange = was.y < 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float x = __builtin_fabsf(kv[i]), y = __builtin_fabsf(vv[i]);
        ka = x < __builtin_inff() ? fmaxf(ka, x) : ka;
        va = y < __builtin_inff() ? fmaxf(va, y) : va;
        strange |= !(y < __builtin_inff());
    }
    strange = __any(strange);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        ka = fmaxf(ka, __shfl_xor(ka, m));
        va = fmaxf(va, __shfl_xor(va, m));
    }
    const float was_v = __builtin_fabsf(was.y);
    const float ks = fmaxf(pow2_of(scale_exponent(ka)), was.x), vs = fmaxf(pow2_of(scale_exponent(va)), was_v);
    uint4 *const keys = reinterpret_cast<uint4 *>(unit_codes), *const values = reinterpret_cast<uint4 *>(unit_codes + kBlock * DP);
    if (old == 0) {         // (a block that is begun: see k_kv_append; of keys that are not there nothing is read)
        for (int i = lane; i < kBlock * (DP / 16); i += 64) values[i] = make_uint4(0, 0, 0, 0);
    } else {
        if (ks != was.x)
            for (int i = lane; i < kBlock * (DP / 16); i += 64) rescale16(keys + i, was.x / ks);
        if (vs != was_v)
            for (int i = lane; i < kBlock * (DP / 16); i += 64) rescale16(values + i, was_v / vs);
    }
    if (old == 0 || ks != was.x || vs != was_v) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");      // other lanes' stores to the bytes below
    const float ki = 1.f / ks, vi = 1.f / vs;
    const int place = value_place(old);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int c = lane * kEach + i;
        if (DP % 64 && c >= DP) break;
        const int two = __builtin_amdgcn_cvt_pk_fp8_f32(code_of(kv[i], ki), code_of(vv[i], vi), 0, false);
        unit_codes[key_at<DP>(old, c)] = (uint8_t)two;
        unit_codes[value_piece<DP>(c, place) + (place & 15)] = (uint8_t)(two >> 8);
    }
    if (lane == 0) g.scales[unit] = make_float2(ks, strange ? -vs : vs);
    if (old < kBlock - 1) return;

    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");      // (the token's own codes, and rounded ones)
    int sum[kEach] = {};
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        float x = 0.f;
        if (DP % 64 == 0 || lane * kEach + i < DP)
#pragma unroll 8
        for (int t = 0; t < kBlock; ++t) {
            const float f = __builtin_amdgcn_cvt_f32_fp8(unit_codes[key_at<DP>(t, lane * kEach + i)], 0);
            x += f == f ? f : 0.f;
        }
        sum[i] = (int)(x * 512.f);
        most = fmaxf(most, __builtin_fabsf((float)sum[i]));
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    const int e = unit_exponent(most * (1.f / 512.f));
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (DP % 64 == 0 || lane * kEach + i < DP) g.sketches[unit * kSketch<DP> + lane * kEach + i] = sketch_of(sum[i], e);
    if (lane == 0) g.weights[unit] = ks * pow2_of(e) * (1.f / kBlock);
}

struct ReadArgs {
    KvGeom kv;
    float *k, *v;
};

// A block goes through LDS, where its codes are taken out of the matrix instructions' order into rows: four channels of a token a store of 16 bytes.  Bound by memory: 15 000
// tokens, 8 heads of 128: 27.6 us for 154 MB, 5.6 TB/s (what was just written is read from the chip's cache).
template <int DP> __global__ __launch_bounds__(kThreads) void k_kv_read(ReadArgs a)
{
    __shared__ __align__(16) uint8_t image[2 * kBlock * DP];
    const KvGeom &g = a.kv;
    const int b = blockIdx.z, h = blockIdx.x % (uint32_t)g.kv_heads, nth = blockIdx.x / (uint32_t)g.kv_heads;
    const Sequence s = sequence_of(g, b);
    // block -1: the rows without a position
    const int from = max(s.pos0, 0), first = s.pos0 < 0 ? -1 : 0;
    const int block = nth + first < 0 ? -1 : from / kBlock + nth + first;
    if (block < 0) {
        const int none = min(-s.pos0, s.n);
        for (int64_t i = threadIdx.x; i < (int64_t)none * g.d; i += kThreads) {
            const int64_t to = ((s.row0 + i / g.d) * g.kv_heads + h) * g.d + i % g.d;
            if (a.k) a.k[to] = 0.f;
            if (a.v) a.v[to] = 0.f;
        }
        return;
    }
    const int at = block * kBlock;
    if (at >= s.len || from >= s.len) return;
    const int begin = max(from - at, 0), end = min(s.len - at, kBlock);
    const int32_t pool = pool_block(g, b, block);
    const bool there = pool >= 0;
    const int64_t unit = unit_of(g, max(pool, 0), h);
    const uint4 *const codes = reinterpret_cast<const uint4 *>(g.codes + unit * (2 * kBlock * DP));
    for (int i = threadIdx.x; i < 2 * kBlock * (DP / 16); i += kThreads) *reinterpret_cast<uint4 *>(image + in_image(16 * i)) = there ? codes[i] : make_uint4(0, 0, 0, 0);
    __syncthreads();
    const float2 scale = there ? g.scales[unit] : make_float2(0.f, 0.f);
    const float vs = __builtin_fabsf(scale.y);
    const int64_t row0 = s.row0 + (int64_t)(at - s.pos0);
    const bool quads = (g.d & 3) == 0;      // (then rows are 16-byte pieces)
    auto put = [&](float *to, int t, int c, const float (&x)[4]) {
        float *const row = to + ((row0 + t) * g.kv_heads + h) * g.d + c;
        if (quads) {
            if (c < g.d) *reinterpret_cast<float4 *>(row) = make_float4(x[0], x[1], x[2], x[3]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < g.d) row[i] = x[i];
    };
    if (a.k)
        for (int i = threadIdx.x; i < kBlock * (DP / 4); i += kThreads) {
            const int t = i / (DP / 4), c = i % (DP / 4) * 4;
            if (t < begin || t >= end) continue;
            const uint32_t x = *reinterpret_cast<const uint32_t *>(image + in_image(key_at<DP>(t, c)));
            const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(x, 0) * scale.x, __builtin_amdgcn_cvt_f32_fp8(x, 1) * scale.x,
                                __builtin_amdgcn_cvt_f32_fp8(x, 2) * scale.x, __builtin_amdgcn_cvt_f32_fp8(x, 3) * scale.x};
            put(a.k, t, c, v);
        }
    if (!a.v) return;
    for (int i = threadIdx.x; i < 16 * (DP / 4); i += kThreads) {
        const int c = i % (DP / 4) * 4, t = i / (DP / 4) * 4;       // four tokens of four channels
        if (t + 3 < begin || t >= end) continue;
        float v[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = *reinterpret_cast<const uint32_t *>(image + in_image(value_piece<DP>(c + j, value_place(t))) + (value_place(t) & 15));
            v[0][j] = __builtin_amdgcn_cvt_f32_fp8(x, 0) * vs, v[1][j] = __builtin_amdgcn_cvt_f32_fp8(x, 1) * vs;
            v[2][j] = __builtin_amdgcn_cvt_f32_fp8(x, 2) * vs, v[3][j] = __builtin_amdgcn_cvt_f32_fp8(x, 3) * vs;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (t + j >= begin && t + j < end) put(a.v, t + j, c, v[j]);
    }
}

template <int DT, int DP> hipError_t run_append(const AppendArgs &a, hipStream_t s)
{
    if (a.kv.max_new == 1) {
        const int64_t waves = (int64_t)a.kv.batch * a.kv.kv_heads;
        k_kv_append_one<DT, DP><<<dim3((uint32_t)((waves + kThreads / 64 - 1) / (kThreads / 64))), kThreads, 0, s>>>(a);
        return hipGetLastError();
    }
    k_kv_append<DT, DP><<<dim3(touched_blocks(a.kv) * a.kv.kv_heads, 1, a.kv.batch), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <int DP> hipError_t run_read(const ReadArgs &a, hipStream_t s)
{
    k_kv_read<DP><<<dim3((touched_blocks(a.kv) + 1) * a.kv.kv_heads, 1, a.kv.batch), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

} // namespace

hipError_t launch_kv_append(const KvGeom &g, int dtype, const uint16_t *k, const uint16_t *v, int64_t k_row, int64_t k_head, int64_t v_row,
                            int64_t v_head, bool wide_k, bool wide_v, hipStream_t s)
{
    const AppendArgs a = {g, k, v, k_row, k_head, v_row, v_head, wide_k, wide_v};
    const bool b = dtype == FC_BF16;
    switch (g.dp) {
    case 64: return b ? run_append<FC_BF16, 64>(a, s) : run_append<FC_F16, 64>(a, s);
    case 96: return b ? run_append<FC_BF16, 96>(a, s) : run_append<FC_F16, 96>(a, s);
    case 128: return b ? run_append<FC_BF16, 128>(a, s) : run_append<FC_F16, 128>(a, s);
    case 192: return b ? run_append<FC_BF16, 192>(a, s) : run_append<FC_F16, 192>(a, s);
    default: return b ? run_append<FC_BF16, 256>(a, s) : run_append<FC_F16, 256>(a, s);
    }
}

hipError_t launch_kv_read(const KvGeom &g, float *k, float *v, hipStream_t s)
{
    const ReadArgs a = {g, k, v};
    switch (g.dp) {
    case 64: return run_read<64>(a, s);
    case 96: return run_read<96>(a, s);
    case 128: return run_read<128>(a, s);
    case 192: return run_read<192>(a, s);
    default: return run_read<256>(a, s);
    }
}

} // namespace fc
