// Group norm of channels-last rows, with the rows that a mask keeps, and an activation.
//
// Memory bounds it: x in and out once, or x in twice where an image does not stay on the chip between its statistics and its output.
//   k_norm_once    a workgroup holds all rows of a slice of an image's channels (whole groups) in registers: one launch, x is read once
//   k_norm_stats, k_norm_apply   images too large for that: workgroups of chunks of rows write what they found; a second launch reads the rows again, and each of
//                  its workgroups joins what all chunks of its image found first (a last workgroup that joins it for all has every workgroup wait for its
//                  place in a counter: 8 images of 256 chunks 55 us, 64 chunks 20)
//
// A thread has a piece of a row (16 bytes, or one element where rows are not made of those) and goes down the rows with it.  Its sums are about the value
// that it meets first: x - pivot is of the size of the spread, whatever the mean is, so that 32 bits lose nothing to it; joining (count, mean, squared
// distances) triples is exact algebra: n = n1 + n2, mean = m1 + (m2 - m1) n2 / n, s = s1 + s2 + (m2 - m1)^2 n1 n2 / n.
#include "fc_layers_internal.hpp"

namespace fc {

constexpr int kNormThreads = 1024;      // of the kernels with chunks

struct Triple {
    float n, mean, s;
    __device__ __forceinline__ void join(float n2, float mean2, float s2)
    {
        const float both = n + n2, part = both > 0.f ? n2 * __builtin_amdgcn_rcpf(both) : 0.f, d = mean2 - mean;
        s += s2 + d * d * (n * part);
        mean += n2 > 0.f ? d * part : 0.f;
        n = both;
    }
};
// over `lanes` (a power of two) neighbouring lanes, in a fixed order
__device__ __forceinline__ Triple join_lanes(Triple t, int lanes)
{
    for (int m = 1; m < lanes; m <<= 1) {
        const float n = __shfl_xor(t.n, m), mean = __shfl_xor(t.mean, m), s = __shfl_xor(t.s, m);
        // (both lanes of a pair join the same two in the same order)
        Triple lo = (threadIdx.x & m) ? Triple{n, mean, s} : t;
        const Triple hi = (threadIdx.x & m) ? t : Triple{n, mean, s};
        if (lo.n == 0.f) lo = hi;
        else if (hi.n > 0.f) lo.join(hi.n, hi.mean, hi.s);
        t = lo;
    }
    return t;
}
// Lanes that take a group together: as many as there are threads for it.
__device__ __forceinline__ int lanes_of(int groups)
{
    int lanes = 64;
    while (lanes > 1 && lanes * groups > (int)blockDim.x) lanes >>= 1;
    return lanes;
}

// A piece of a row: VE values, and the way back.
template <typename T, bool WIDE> struct Piece {
    static constexpr int VE = WIDE ? 16 / (int)sizeof(T) : 1;
    typedef typename std::conditional<WIDE, uint4, T>::type raw_t;
    static __device__ __forceinline__ void values(const raw_t &r, float (&v)[VE])
    {
        if constexpr (!WIDE) v[0] = to_float(r);
        else if constexpr (sizeof(T) == 4) {
            const float4 f = __builtin_bit_cast(float4, r);
            v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
        } else unpack8<T>(r, v);
    }
    static __device__ __forceinline__ raw_t rounded(const float (&v)[VE])
    {
        if constexpr (!WIDE) {
            T t;
            from_float(v[0], &t);
            return t;
        } else if constexpr (sizeof(T) == 4) {
            return __builtin_bit_cast(uint4, make_float4(v[0], v[1], v[2], v[3]));
        } else return pack8<T>(v);
    }
    static __device__ __forceinline__ raw_t select(bool which, const raw_t &a, const raw_t &b)
    {
        if constexpr (WIDE) return make_uint4(which ? a.x : b.x, which ? a.y : b.y, which ? a.z : b.z, which ? a.w : b.w);
        else return which ? a : b;
    }
    // (past the caches: x is still in them for the next call's or launch's reads; 268 MB of bf16, statistics 73 -> 52 us, outputs 100 -> 104; a mask that keeps half of 67 MB 15.6 -> 14.1 and 26.9 -> 25.4)
    static __device__ __forceinline__ void store(raw_t *p, const raw_t &v)
    {
        if constexpr (WIDE) __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t *>(p));
        else *p = v;
    }
    static __device__ __forceinline__ raw_t zero()
    {
        if constexpr (WIDE) return make_uint4(0, 0, 0, 0);
        else return T{};
    }
};

// An image's rows, cut to the call's bounds.
struct ImageRows {
    int32_t first, n;
};
__device__ __forceinline__ ImageRows image_rows(const NormArgs &a, int image)
{
    if (!a.starts) return {image * a.max_rows, a.max_rows};
    const int32_t from = min(max(a.starts[image], 0), a.rows), to = min(max(a.starts[image + 1], from), a.rows);
    return {from, min(to - from, a.max_rows)};
}

// How a workgroup's threads lie over a slice: piece `p` (of PR; more than there are threads: several each), row `phase` of every `phases`.
struct Spread {
    int pr, phases, p, phase;
    bool active;
};
template <typename P> __device__ __forceinline__ Spread spread_of(const NormArgs &a)
{
    Spread s;
    const int threads = (int)blockDim.x;
    s.pr = a.slice / P::VE;
    s.phases = s.pr < threads ? threads / s.pr : 1;
    s.phase = s.pr < threads ? (int)threadIdx.x / s.pr : 0;
    s.p = (int)threadIdx.x - s.phase * s.pr;
    s.active = s.phase < s.phases;
    return s;
}
// What threads found, in LDS: counts [phases], then (mean, squared distances) [phases][entries of a row].  An entry is a piece where pieces lie within a
// group, else a channel.
template <typename P> struct Found {
    float *counts;
    float2 *entries;
    int row, per_entry, per_group;      // entries of a row; values of an entry; entries of a group
    bool whole;
    __device__ __forceinline__ Found(const NormArgs &a, const Spread &s, unsigned char *lds)
    {
        whole = a.per_group % P::VE == 0;
        per_entry = whole ? P::VE : 1;
        row = a.slice / per_entry;
        per_group = a.per_group / per_entry;
        entries = reinterpret_cast<float2 *>(lds);
        counts = reinterpret_cast<float *>(entries + s.phases * row);
    }
    // rows: how many this thread saw; s1, s2: the sums about the pivots
    __device__ __forceinline__ void put(const Spread &sp, int p, float rows, const float (&pivot)[P::VE], const float (&s1)[P::VE], const float (&s2)[P::VE]) const
    {
        const float inverse = rows > 0.f ? 1.f / rows : 0.f;
        float mean[P::VE], s[P::VE];
#pragma unroll
        for (int i = 0; i < P::VE; ++i) {
            mean[i] = pivot[i] + s1[i] * inverse;
            s[i] = s2[i] - s1[i] * s1[i] * inverse;
            s[i] = s[i] < 0.f ? 0.f : s[i];
        }
        if (whole) {        // (equal counts)
            float m = 0.f, all = 0.f, off = 0.f;
#pragma unroll
            for (int i = 0; i < P::VE; ++i) m += mean[i] - mean[0];
            m = mean[0] + m * (1.f / P::VE);
#pragma unroll
            for (int i = 0; i < P::VE; ++i) {
                all += s[i];
                off = fmaf(mean[i] - m, mean[i] - m, off);
            }
            entries[sp.phase * row + p] = make_float2(m, fmaf(rows, off, all));
        } else {
#pragma unroll
            for (int i = 0; i < P::VE; ++i) entries[sp.phase * row + p * P::VE + i] = make_float2(mean[i], s[i]);
        }
        if (p == 0) counts[sp.phase] = rows;
    }
    // group g of the slice, by `lanes` lanes
    __device__ __forceinline__ Triple group(const Spread &sp, int g, int lanes) const
    {
        const int items = per_group * sp.phases;
        Triple t = {0.f, 0.f, 0.f};
        for (int i = (int)threadIdx.x & (lanes - 1); i < items; i += lanes) {
            const int phase = i / per_group, e = i - phase * per_group;
            const float n = counts[phase] * (float)per_entry;
            const float2 f = entries[phase * row + g * per_group + e];
            if (n > 0.f) {
                if (t.n == 0.f) t = {n, f.x, f.y};
                else t.join(n, f.x, f.y);
            }
        }
        return join_lanes(t, lanes);
    }
};
__device__ __forceinline__ float2 stats_of(const NormArgs &a, const Triple &t)
{
    return make_float2(t.mean, t.n > 0.f ? 1.f / sqrtf(t.s / t.n + a.eps) : 0.f);
}

// A thread's channels: (x - mean) * factor + bias.  weight and bias can be on their way before the statistics are known.
template <typename P> struct Affine {
    float mean[P::VE], factor[P::VE], bias[P::VE];
    __device__ __forceinline__ void load(const NormArgs &a, int c)  // c: of the row
    {
#pragma unroll
        for (int i = 0; i < P::VE; ++i) {
            factor[i] = a.weight ? a.weight[c + i] : 1.f;
            bias[i] = a.bias ? a.bias[c + i] : 0.f;
        }
    }
    __device__ __forceinline__ void set(const NormArgs &a, int c, const float2 *stats)     // c: of the slice
    {
#pragma unroll
        for (int i = 0; i < P::VE; ++i) {
            const float2 s = stats[(c + i) / a.per_group];
            mean[i] = s.x;
            factor[i] *= s.y;
        }
    }
    __device__ __forceinline__ typename P::raw_t operator()(const NormArgs &a, const typename P::raw_t &r) const
    {
        float v[P::VE];
        P::values(r, v);
#pragma unroll
        for (int i = 0; i < P::VE; ++i) v[i] = (v[i] - mean[i]) * factor[i] + bias[i];
        activate_all(v, a.act);
        return P::rounded(v);
    }
};

// A thread's sums about the first piece that it sees.  A piece that does not count is taken to be the pivot: it adds nothing.
template <typename P> struct Sums {
    typename P::raw_t first;
    float pivot[P::VE], s1[P::VE], s2[P::VE], rows;
    __device__ __forceinline__ Sums()
    {
        rows = 0.f;
        first = P::zero();
#pragma unroll
        for (int i = 0; i < P::VE; ++i) pivot[i] = s1[i] = s2[i] = 0.f;
    }
    template <int N> __device__ __forceinline__ void add(const typename P::raw_t (&r)[N], const bool (&seen)[N])
    {
        if (rows == 0.f) {
#pragma unroll
            for (int i = N - 1; i >= 0; --i) first = P::select(seen[i], r[i], first);
            P::values(first, pivot);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float v[P::VE];
            P::values(P::select(seen[n], r[n], first), v);
#pragma unroll
            for (int i = 0; i < P::VE; ++i) {
                const float d = v[i] - pivot[i];
                s1[i] += d;
                s2[i] = fmaf(d, d, s2[i]);
            }
            rows += seen[n] ? 1.f : 0.f;
        }
    }
};

template <typename T, bool WIDE, int NP>
__global__ __launch_bounds__(1024)
void k_norm_once(NormArgs a)
{
    typedef Piece<T, WIDE> P;
    typedef typename P::raw_t raw_t;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float2 group_stats[512];
    const int slice = (int)blockIdx.x % a.slices, image = (int)blockIdx.x / a.slices;
    const ImageRows rows = image_rows(a, image);
    if (rows.n <= 0) return;
    const Spread sp = spread_of<P>(a);
    const Found<P> found(a, sp, smem_raw);
    const int c = slice * a.slice + sp.p * P::VE;
    const T *const x = static_cast<const T *>(a.x) + (int64_t)rows.first * a.x_row + c;
    T *const out = static_cast<T *>(a.out) + (int64_t)rows.first * a.out_row + c;
    const uint8_t *const mask = a.mask ? a.mask + rows.first : nullptr;
    raw_t r[NP];
    bool seen[NP];
    const int last = rows.n - 1;
    if (mask) {
        uint32_t m[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) m[i] = mask[min(sp.phase + i * sp.phases, last)];
        loaded_together(m);
#pragma unroll
        for (int i = 0; i < NP; ++i) seen[i] = m[i] != 0;
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) seen[i] = true;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int row = sp.phase + i * sp.phases;
        seen[i] = seen[i] && row <= last && sp.active;
        r[i] = P::zero();
        if (seen[i]) r[i] = *reinterpret_cast<const raw_t *>(x + (int64_t)row * a.x_row);
    }
    Affine<P> affine;
    if (NP <= 4 && sp.active) affine.load(a, c);        // (with more pieces there are no registers for them yet)
    Sums<P> sums;
    sums.add(r, seen);
    if (sp.active) found.put(sp, sp.p, sums.rows, sums.pivot, sums.s1, sums.s2);
    __syncthreads();
    const int groups = a.slice / a.per_group, lanes = lanes_of(groups);
    for (int g = (int)threadIdx.x / lanes; g < groups; g += (int)blockDim.x / lanes) {
        const float2 s = stats_of(a, found.group(sp, g, lanes));
        if ((threadIdx.x & (lanes - 1)) == 0) group_stats[g] = s;
    }
    __syncthreads();
    if (!sp.active) return;
    if (NP > 4) affine.load(a, c);
    affine.set(a, sp.p * P::VE, group_stats);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int row = sp.phase + i * sp.phases;
        raw_t *const to = reinterpret_cast<raw_t *>(out + (int64_t)row * a.out_row);
        if (seen[i]) *to = affine(a, r[i]);
        else if (row <= last && !a.keep_out) *to = P::zero();
    }
}

constexpr int kNormUnroll = 4;           // (eight: statistics of 268 MB 67 us instead of 53)

// N rows (from `row` on, every phases-th, below `to`) of a thread's piece; which of them count.  Those that do not are not read: the chunk's first row is in
// their place, without a branch between the loads.
template <typename P, typename T, int N>
__device__ __forceinline__ void load_rows(const NormArgs &a, const T *x, const uint8_t *mask, int row, int phases, int from, int to, typename P::raw_t (&r)[N], bool (&seen)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) seen[i] = row + i * phases < to;
    if (mask) {
        uint32_t m[N];
#pragma unroll
        for (int i = 0; i < N; ++i) m[i] = mask[seen[i] ? row + i * phases : from];
        loaded_together(m);
#pragma unroll
        for (int i = 0; i < N; ++i) seen[i] = seen[i] && m[i] != 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = *reinterpret_cast<const typename P::raw_t *>(x + (int64_t)(seen[i] ? row + i * phases : from) * a.x_row);
}

// [image][slice][group of the slice][chunk]: count, mean, squared distances
__device__ __forceinline__ float4 *part_of(const NormArgs &a, int64_t unit, int groups, int g) { return a.part + (unit * groups + g) * a.chunks; }

template <typename T, bool WIDE>
__global__ __launch_bounds__(kNormThreads)
void k_norm_stats(NormArgs a)
{
    typedef Piece<T, WIDE> P;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const int chunk = (int)blockIdx.x % a.chunks, unit = (int)blockIdx.x / a.chunks, slice = unit % a.slices, image = unit / a.slices;
    const ImageRows rows = image_rows(a, image);
    const Spread sp = spread_of<P>(a);
    const Found<P> found(a, sp, smem_raw);
    const int from = chunk * a.chunk_rows, to = min(from + a.chunk_rows, rows.n);
    const uint8_t *const mask = a.mask ? a.mask + rows.first : nullptr;
    if (sp.active)
        for (int p = sp.p; p < sp.pr; p += kNormThreads) {
            const T *const x = static_cast<const T *>(a.x) + (int64_t)rows.first * a.x_row + slice * a.slice + p * P::VE;
            Sums<P> sums;
            typename P::raw_t r[kNormUnroll];
            bool seen[kNormUnroll];
            if (from < to) load_rows<P>(a, x, mask, from + sp.phase, sp.phases, from, to, r, seen);
            for (int row = from + sp.phase; row < to; row += kNormUnroll * sp.phases) {
                // (the next rows are sent for before these are added)
                typename P::raw_t now[kNormUnroll];
                bool counts[kNormUnroll];
#pragma unroll
                for (int i = 0; i < kNormUnroll; ++i) now[i] = r[i], counts[i] = seen[i];
                const int next = row + kNormUnroll * sp.phases;
                if (next < to) load_rows<P>(a, x, mask, next, sp.phases, from, to, r, seen);
                sums.add(now, counts);
            }
            found.put(sp, p, sums.rows, sums.pivot, sums.s1, sums.s2);
            if (sp.pr < kNormThreads) break;
        }
    __syncthreads();
    const int groups = a.slice / a.per_group, lanes = lanes_of(groups);
    for (int g = (int)threadIdx.x / lanes; g < groups; g += kNormThreads / lanes) {
        const Triple t = found.group(sp, g, lanes);
        if ((threadIdx.x & (lanes - 1)) == 0) part_of(a, unit, groups, g)[chunk] = make_float4(t.n, t.mean, t.s, 0.f);
    }
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(kNormThreads)
void k_norm_apply(NormArgs a)
{
    typedef Piece<T, WIDE> P;
    typedef typename P::raw_t raw_t;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float2 *const stats = reinterpret_cast<float2 *>(smem_raw);     // [groups of the slice]
    const int chunk = (int)blockIdx.x % a.chunks, unit = (int)blockIdx.x / a.chunks, slice = unit % a.slices, image = unit / a.slices;
    const ImageRows rows = image_rows(a, image);
    const Spread sp = spread_of<P>(a);
    const int from = chunk * a.chunk_rows, to = min(from + a.chunk_rows, rows.n);
    if (from >= to) return;
    const uint8_t *const mask = a.mask ? a.mask + rows.first : nullptr;
    const int c0 = slice * a.slice;
    const T *const x = static_cast<const T *>(a.x) + (int64_t)rows.first * a.x_row + c0;
    T *const out = static_cast<T *>(a.out) + (int64_t)rows.first * a.out_row + c0;
    // (the first rows, the weights and what the chunks found are on their way together)
    raw_t r[kNormUnroll];
    bool seen[kNormUnroll];
    if (sp.active) load_rows<P>(a, x + sp.p * P::VE, mask, from + sp.phase, sp.phases, from, to, r, seen);
    Affine<P> affine;
    if (sp.active) affine.load(a, c0 + sp.p * P::VE);

    const int groups = a.slice / a.per_group, lanes = lanes_of(groups), lane = threadIdx.x & (lanes - 1);
    for (int g = (int)threadIdx.x / lanes; g < groups; g += kNormThreads / lanes) {
        const float4 *const part = part_of(a, unit, groups, g);
        Triple t = {0.f, 0.f, 0.f};
        constexpr int AT_ONCE = 4;      // (chunks whose loads are under way together)
        for (int i = lane; i < a.chunks; i += AT_ONCE * lanes) {
            float4 f[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) f[u] = part[min(i + u * lanes, a.chunks - 1)];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (i + u * lanes < a.chunks && f[u].x > 0.f) {
                    if (t.n == 0.f) t = {f[u].x, f[u].y, f[u].z};
                    else t.join(f[u].x, f[u].y, f[u].z);
                }
        }
        t = join_lanes(t, lanes);
        if (lane == 0) stats[g] = stats_of(a, t);
    }
    __syncthreads();
    if (!sp.active) return;
    for (int p = sp.p; p < sp.pr; p += kNormThreads) {
        if (p != sp.p) {
            affine.load(a, c0 + p * P::VE);
            load_rows<P>(a, x + p * P::VE, mask, from + sp.phase, sp.phases, from, to, r, seen);
        }
        affine.set(a, p * P::VE, stats);
        for (int row = from + sp.phase; row < to; row += kNormUnroll * sp.phases) {
            // (the next rows are sent for before these are finished)
            raw_t now[kNormUnroll];
            bool counts[kNormUnroll];
#pragma unroll
            for (int i = 0; i < kNormUnroll; ++i) now[i] = r[i], counts[i] = seen[i];
            const int next = row + kNormUnroll * sp.phases;
            if (next < to) load_rows<P>(a, x + p * P::VE, mask, next, sp.phases, from, to, r, seen);
#pragma unroll
            for (int i = 0; i < kNormUnroll; ++i) {
                raw_t *const at = reinterpret_cast<raw_t *>(out + (int64_t)(row + i * sp.phases) * a.out_row + p * P::VE);
                const raw_t v = P::select(counts[i], affine(a, now[i]), P::zero());
                if (counts[i] || (row + i * sp.phases < to && !a.keep_out)) P::store(at, v);
            }
        }
        if (sp.pr < kNormThreads) break;
    }
}

template <typename T, bool WIDE> static hipError_t launch_norm_as(const NormArgs &a, const NormPlan &p, hipStream_t s)
{
    if (p.once) {
        const dim3 grid((uint32_t)(a.images * a.slices)), block((uint32_t)p.threads);
        if (p.per_thread <= 4) k_norm_once<T, WIDE, 4><<<grid, block, p.lds, s>>>(a);
        else k_norm_once<T, WIDE, 12><<<grid, block, p.lds, s>>>(a);
        return hipGetLastError();
    }
    if (p.lds > 65536) {
        const hipError_t e = raise_dynamic_lds<&k_norm_stats<T, WIDE>>(163840);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((uint32_t)((int64_t)a.chunks * a.slices * a.images));
    k_norm_stats<T, WIDE><<<grid, dim3(kNormThreads), p.lds, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_norm_apply<T, WIDE><<<grid, dim3(kNormThreads), (size_t)(a.slice / a.per_group) * sizeof(float2), s>>>(a);
    return hipGetLastError();
}

hipError_t launch_group_norm(const NormArgs &a, const NormPlan &p, int dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return p.wide ? launch_norm_as<bf16_t, true>(a, p, s) : launch_norm_as<bf16_t, false>(a, p, s);
    if (dtype == FC_F16) return p.wide ? launch_norm_as<f16_t, true>(a, p, s) : launch_norm_as<f16_t, false>(a, p, s);
    return p.wide ? launch_norm_as<float, true>(a, p, s) : launch_norm_as<float, false>(a, p, s);
}

} // namespace fc
