// Pages of the key/value cache: giving blocks to sequences and back, forking, compacting, copying.
//
// Tables are small and blocks are large: what bounds the calls is launches where only tables change, and memory where blocks are copied.  A call that gives out
// blocks is two launches.  The first goes over the sequences: blocks that are let go leave the counts of users by atomics (sums of whole numbers: the order
// does not matter), and every sequence says how many blocks it wants.  Its last workgroup then has the counts as they are after all of that, adds up what is
// wanted in order and lists the lowest free blocks.  The second launch writes the tables and copies blocks, every sequence for itself.  (Tables written by the
// last workgroup of the first launch: 38 us for 256 sequences, its waves' round trips one after another.)
//
// What workgroups of other XCDs wrote in the same launch is read past the caches.
#include "fc_attn_internal.hpp"
#include "focused_pages.h"
#include <initializer_list>

using namespace fc;

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kMostWorkgroups = 512;
constexpr int kScan = 16 * kThreads;        // users looked at in a step
constexpr int kMostBlocks = 1 << 29;        // users within a buffer of 2^31 bytes

// One section of a cache: bytes of a block, where the section begins.
struct Section {
    uint8_t *base;
    int64_t block;
};
struct CacheView {
    Section codes, scales, sketches, weights;
};

struct PagesArgs {
    int32_t blocks, blocks_to, batch, width;
    int32_t *users, *table, *lengths;
    const int32_t *parents;
    int32_t *missing;
    // workspace
    int32_t *arrived;           // one counter, of workgroups that are done; zero before and after every call
    int32_t *wanted;            // [batch]: blocks a sequence wants; its last one is to be a copy of own[b]
    int32_t *own;               // [batch]: -1, or the block that the sequence gets a copy of
    int32_t *offsets;           // [batch]
    int32_t *given;             // [blocks]: free blocks
    int32_t *found;             // one: how many of them are listed
    int32_t *rows, *new_lengths;    // fork: the new table
};

__device__ __forceinline__ int32_t load_shared(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_shared(int32_t *p, int32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void count_users(int32_t *p, int32_t by) { __hip_atomic_fetch_add(p, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ int32_t needed(int32_t length, int32_t width)
{
    const int64_t held = (int64_t)width * kBlock, n = length < 0 ? 0 : length < held ? length : held;
    return (int32_t)((n + kBlock - 1) / kBlock);
}
__device__ __forceinline__ bool unfinished(int32_t length, int32_t width) { return length > 0 && (int64_t)length < (int64_t)width * kBlock && length % kBlock != 0; }

// Sum over a workgroup of kThreads, and the sum of the threads before this one.
struct Scanned {
    int32_t before, all;
};
__device__ __forceinline__ Scanned scan(int32_t v, int32_t *lds)       // lds [kWaves]; two barriers
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t upto = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int32_t o = __shfl_up(upto, m);
        if (lane >= m) upto += o;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    int32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int32_t n = lds[w];
        before += w < wave ? n : 0;
        all += n;
    }
    return {before + upto - v, all};
}

// The lowest free blocks, as many as `total` if there are so many: their numbers into given, their users 1; how many there are is returned.
__device__ __forceinline__ int32_t find_free(const PagesArgs &a, int32_t total, int32_t *lds)
{
    int32_t found = 0;
    const auto users = __builtin_amdgcn_make_buffer_rsrc(a.users, 0, (uint32_t)a.blocks * 4u, 0x00020000);
    for (int32_t first = 0; first < a.blocks && found < total; first += kScan) {
        const int32_t at = first + (int32_t)threadIdx.x * 16;
        u32x4_t u[4];
        // (behind the last block: zeros, which do not count)
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_raw_buffer_load_b128(users, (uint32_t)(at + 4 * i) * 4u, 0, kPastCaches);
        uint32_t free = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) free |= (u[i / 4][i % 4] == 0 && at + i < a.blocks ? 1u : 0u) << i;
        const Scanned s = scan(__popc(free), lds);
        int32_t rank = found + s.before;
        for (uint32_t left = free; left && rank < total; left &= left - 1, ++rank) {
            const int32_t block = at + __ffs(left) - 1;
            a.given[rank] = block;
            a.users[block] = 1;
        }
        found += s.all;
    }
    return min(found, total);
}

// Is this the launch's last workgroup?  (Every thread; stores of others are visible to loads past the caches then.)
__device__ __forceinline__ bool last_workgroup(const PagesArgs &a, int32_t *flag)
{
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const int32_t before = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = before == (int32_t)gridDim.x - 1;
        if (*flag) store_shared(a.arrived, 0);
    }
    __syncthreads();
    return *flag;
}

// The last workgroup's part: offsets of what the sequences want, in order (all of it is returned), and the blocks they get.
__device__ __forceinline__ int32_t order_wanted(const PagesArgs &a, int32_t *lds)
{
    int32_t total = 0;
    for (int32_t first = 0; first < a.batch; first += kThreads) {
        const int32_t b = first + (int32_t)threadIdx.x;
        const Scanned s = scan(b < a.batch ? load_shared(a.wanted + b) : 0, lds);
        if (b < a.batch) a.offsets[b] = total + s.before;
        total += s.all;
    }
    return total;
}
__device__ __forceinline__ void dealt(const PagesArgs &a, int32_t total, int32_t found)
{
    if (threadIdx.x == 0) {
        *a.found = found;
        *a.missing = total - found;
    }
}

// Everything that this workgroup has written is there for all of it.
__device__ __forceinline__ void written()
{
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Too few blocks for all that is wanted: a block that nobody holds but sequences that are cut within it stays with the lowest of them, which wants no copy then.
// The blocks' users themselves say who that is: less those sequences none are left, and the lowest sequence leaves the least mark below zero.
__device__ __forceinline__ void keep_where_all_are_cut(const PagesArgs &a)
{
    constexpr int32_t MARKS = 65536;        // (sequences number below)
    for (int32_t b = threadIdx.x; b < a.batch; b += kThreads)
        if (a.own[b] >= 0) count_users(a.users + a.own[b], -1);
    written();
    for (int32_t b = threadIdx.x; b < a.batch; b += kThreads)
        if (a.own[b] >= 0 && load_shared(a.users + a.own[b]) <= 0) __hip_atomic_fetch_min(a.users + a.own[b], b - MARKS, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    written();
    // (a keeper's block is -2 - own until the counts are as they were)
    for (int32_t b = threadIdx.x; b < a.batch; b += kThreads)
        if (a.own[b] >= 0 && load_shared(a.users + a.own[b]) == b - MARKS) {
            a.own[b] = -2 - a.own[b];
            store_shared(a.wanted + b, load_shared(a.wanted + b) - 1);
        }
    written();
    for (int32_t b = threadIdx.x; b < a.batch; b += kThreads) {
        const int32_t own = a.own[b];
        if (own >= 0) count_users(a.users + own, 1);
        if (own < -1) {
            count_users(a.users + (-2 - own), 1 + MARKS - b);
            a.own[b] = -1;
        }
    }
    written();
}

__global__ __launch_bounds__(kThreads) void k_resize(PagesArgs a)
{
    __shared__ int32_t lds[kWaves], flag;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // a wave a sequence: what lies behind its need goes back, what is not there is wanted
    for (int32_t b = (int32_t)blockIdx.x * kWaves + wave; b < a.batch; b += (int32_t)gridDim.x * kWaves) {
        int32_t *const row = a.table + (int64_t)b * a.width;
        const int32_t need = needed(a.lengths[b], a.width);
        int32_t wants = 0;
        for (int32_t j0 = 0; j0 < a.width; j0 += 256) {
            int32_t e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = j0 + i * 64 + lane < a.width ? row[j0 + i * 64 + lane] : -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t j = j0 + i * 64 + lane;
                const bool there = (uint32_t)e[i] < (uint32_t)a.blocks;
                wants += __popcll(__ballot(j < need && !there));
                if (j >= need && j < a.width && e[i] != -1) {
                    if (there) count_users(a.users + e[i], -1);
                    row[j] = -1;
                }
            }
        }
        if (lane == 0) store_shared(a.wanted + b, wants);
    }
    if (!last_workgroup(a, &flag)) return;

    // an unfinished last block that others hold as well: a copy
    for (int32_t b = threadIdx.x; b < a.batch; b += kThreads) {
        int32_t source = -1;
        const int32_t length = a.lengths[b];
        if (unfinished(length, a.width)) {
            const int32_t e = a.table[(int64_t)b * a.width + needed(length, a.width) - 1];
            if ((uint32_t)e < (uint32_t)a.blocks && load_shared(a.users + e) > 1) source = e;
        }
        a.own[b] = source;
        if (source >= 0) store_shared(a.wanted + b, load_shared(a.wanted + b) + 1);
    }
    __syncthreads();
    int32_t total = order_wanted(a, lds);
    int32_t found = total ? find_free(a, total, lds) : 0;
    if (found < total) {
        written();
        keep_where_all_are_cut(a);
        total = order_wanted(a, lds);
        for (int32_t i = total + (int32_t)threadIdx.x; i < found; i += kThreads) a.users[a.given[i]] = 0;      // (more than are wanted now)
        found = min(found, total);
    }
    dealt(a, total, found);
}

__global__ __launch_bounds__(kThreads) void k_fork(PagesArgs a)
{
    __shared__ int32_t lds[kWaves], flag, lower;
    // a workgroup a slot
    for (int32_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        const int32_t p = a.parents[b];
        const bool lives = (uint32_t)p < (uint32_t)a.batch;
        if (p == b) {
            if (threadIdx.x == 0) {
                store_shared(a.wanted + b, 0);
                store_shared(a.own + b, -1);
            }
            continue;
        }
        const int32_t length = lives ? a.lengths[p] : 0, need = needed(length, a.width);
        const int32_t *const from = a.table + (int64_t)(lives ? p : 0) * a.width, *const old = a.table + (int64_t)b * a.width;
        int32_t *const row = a.rows + (int64_t)b * a.width;
        // does somebody else keep the unfinished block?
        bool copied = lives && unfinished(length, a.width);
        if (copied && a.parents[p] != p) {
            __syncthreads();
            if (threadIdx.x == 0) lower = 0;
            __syncthreads();
            bool any = false;
            for (int32_t i = threadIdx.x; i < b; i += kThreads) any = any || a.parents[i] == p;
            if (any) lower = 1;
            __syncthreads();
            copied = lower != 0;
        }
        const int32_t last = copied ? from[need - 1] : -1;
        copied = copied && (uint32_t)last < (uint32_t)a.blocks;
        for (int32_t j = threadIdx.x; j < a.width; j += kThreads) {
            const int32_t had = old[j];
            if ((uint32_t)had < (uint32_t)a.blocks) count_users(a.users + had, -1);
            int32_t e = j < need ? from[j] : -1;
            if ((uint32_t)e >= (uint32_t)a.blocks || (copied && j == need - 1)) e = -1;
            else count_users(a.users + e, 1);
            row[j] = e;
        }
        if (threadIdx.x == 0) {
            a.new_lengths[b] = length;
            store_shared(a.wanted + b, copied);
            store_shared(a.own + b, copied ? last : -1);
        }
    }
    if (!last_workgroup(a, &flag)) return;

    const int32_t total = order_wanted(a, lds);
    dealt(a, total, total ? find_free(a, total, lds) : 0);
}

// The block that a sequence's last wanted place gets, -1: none.
__device__ __forceinline__ int32_t last_given(const PagesArgs &a, int32_t b)
{
    const int32_t rank = a.offsets[b] + a.wanted[b] - 1;
    return rank < *a.found ? a.given[rank] : -1;
}

// ---- copying ----

// Sixteen-byte pieces of a block's codes that a workgroup of 256 threads copies at once.
constexpr int kCopyThreads = 256, kCopyPieces = 8, kCopyBytes = kCopyThreads * kCopyPieces * 16;

struct CopyArgs {
    CacheView from, to;
    int32_t blocks, blocks_to;
    const int32_t *sources, *targets;   // targets NULL: block i
    const int32_t *count;               // how many there are, or NULL: all
    int32_t most;
    int32_t segments;                   // of a block's codes
};

template <typename V> __device__ __forceinline__ void copy_small(const Section &from, const Section &to, int64_t s, int64_t t)
{
    const V *const x = reinterpret_cast<const V *>(from.base + s * from.block);
    V *const y = reinterpret_cast<V *>(to.base + t * to.block);
    const int32_t n = (int32_t)(from.block / (int64_t)sizeof(V));
    for (int32_t i = threadIdx.x; i < n; i += kCopyThreads) y[i] = x[i];
}

// A segment of block s of one cache to block t of the other.  MANY: its loads leave the caches to others.  (Whole caches move in 89 us so and in 112 without, 330 MB; a fork's
// few blocks are read again by whoever goes on with them: 256 sequences forked and their last tokens read 44 us so, 37 without.)
template <bool MANY> __device__ __forceinline__ void copy_segment(const CopyArgs &c, int32_t s, int32_t t, int32_t segment)
{
    const int64_t at = (int64_t)segment * kCopyBytes + threadIdx.x * 16, end = c.from.codes.block;
    const uint8_t *const x = c.from.codes.base + s * end;
    uint8_t *const y = c.to.codes.base + t * end;
    u32x4_t v[kCopyPieces];
#pragma unroll
    for (int j = 0; j < kCopyPieces; ++j) {
        const int64_t o = at + j * (kCopyThreads * 16);
        const u32x4_t *const p = reinterpret_cast<const u32x4_t *>(x + (o < end ? o : 0));
        if constexpr (MANY) v[j] = __builtin_nontemporal_load(p);
        else v[j] = *p;
    }
#pragma unroll
    for (int j = 0; j < kCopyPieces; ++j) {
        const int64_t o = at + j * (kCopyThreads * 16);
        if (o < end) *reinterpret_cast<u32x4_t *>(y + o) = v[j];
    }
    if (segment == 0) {
        copy_small<float2>(c.from.scales, c.to.scales, s, t);
        copy_small<float>(c.from.weights, c.to.weights, s, t);
        copy_small<uint4>(c.from.sketches, c.to.sketches, s, t);
    }
}

__device__ __forceinline__ void copy_blocks(const CopyArgs &c)
{
    const int32_t count = c.count ? min(max(*c.count, 0), c.most) : c.most;
    const int64_t items = (int64_t)count * c.segments;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int32_t n = (int32_t)(i / c.segments), segment = (int32_t)(i - (int64_t)n * c.segments);
        const int32_t s = c.sources[n], t = c.targets ? c.targets[n] : n;
        if ((uint32_t)s < (uint32_t)c.blocks && (uint32_t)t < (uint32_t)c.blocks_to) copy_segment<true>(c, s, t, segment);
    }
}

__global__ __launch_bounds__(kCopyThreads) void k_copy(CopyArgs c) { copy_blocks(c); }

// The copies that sequences get of blocks of their own: items of a sequence and a segment.
__device__ __forceinline__ void copy_own(const PagesArgs &a, const CopyArgs &c)
{
    const int64_t items = (int64_t)a.batch * c.segments;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int32_t b = (int32_t)(i / c.segments), segment = (int32_t)(i - (int64_t)b * c.segments);
        const int32_t source = a.own[b];
        if (source < 0) continue;
        const int32_t block = last_given(a, b);
        if (block >= 0) copy_segment<false>(c, source, block, segment);
    }
}

// What the sequences wanted goes into their tables.
__global__ __launch_bounds__(kCopyThreads) void k_resize_rows(PagesArgs a, CopyArgs c)
{
    const int lane = threadIdx.x & 63, waves = kCopyThreads / 64;
    for (int32_t b = (int32_t)blockIdx.x * waves + (int32_t)(threadIdx.x >> 6); b < a.batch; b += (int32_t)gridDim.x * waves) {
        if (a.wanted[b] == 0) continue;
        int32_t *const row = a.table + (int64_t)b * a.width;
        const int32_t need = needed(a.lengths[b], a.width), source = a.own[b], found = *a.found;
        int32_t rank = a.offsets[b];
        for (int32_t j0 = 0; j0 < need; j0 += 256) {
            int32_t e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = j0 + i * 64 + lane < need ? row[j0 + i * 64 + lane] : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t j = j0 + i * 64 + lane;
                const bool copy = source >= 0 && j == need - 1, wants = j < need && ((uint32_t)e[i] >= (uint32_t)a.blocks || copy);
                const uint64_t all = __ballot(wants);
                const int32_t mine = rank + __popcll(all & ((1ull << lane) - 1));
                if (wants) row[j] = mine < found ? a.given[mine] : -1;
                if (copy) count_users(a.users + source, -1);
                rank += __popcll(all);
            }
        }
    }
    copy_own(a, c);
}

__global__ __launch_bounds__(kCopyThreads) void k_fork_rows(PagesArgs a, CopyArgs c)
{
    for (int32_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (a.parents[b] == b) continue;
        const int32_t length = a.new_lengths[b];
        const int32_t last = a.own[b] >= 0 ? needed(length, a.width) - 1 : -1, block = a.own[b] >= 0 ? last_given(a, b) : -1;
        for (int32_t j = threadIdx.x; j < a.width; j += kCopyThreads)
            a.table[(int64_t)b * a.width + j] = j == last ? block : a.rows[(int64_t)b * a.width + j];
        if (threadIdx.x == 0) a.lengths[b] = length;
    }
    copy_own(a, c);
}

// ---- compacting ----

constexpr int kNumbered = 4 * kThreads;      // blocks that a workgroup numbers

struct CompactArgs {
    int32_t blocks, blocks_to, batch, width;
    const int32_t *users, *table;
    int32_t *users_to, *table_to, *missing;
    int32_t *numbers;       // [blocks]: a block's new number, -1: none
    int32_t *sources;       // [blocks_to]
    int32_t *count;         // blocks that are moved
};

// A workgroup's blocks are numbered behind all used blocks before them, which it counts itself.
__global__ __launch_bounds__(kThreads) void k_number(CompactArgs a)
{
    __shared__ int32_t lds[kWaves];
    const int64_t first = (int64_t)blockIdx.x * kNumbered;
    int32_t before = 0;
    for (int64_t i = (int64_t)threadIdx.x * 4; i < first; i += kNumbered) {
        const int4 u = *reinterpret_cast<const int4 *>(a.users + i);
        before += (u.x > 0) + (u.y > 0) + (u.z > 0) + (u.w > 0);
    }
    before = scan(before, lds).all;
    const int64_t at = first + (int64_t)threadIdx.x * 4;
    int32_t u[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = at + i < a.blocks ? a.users[at + i] : 0;
        mine += u[i] > 0;
    }
    const Scanned s = scan(mine, lds);
    int32_t number = before + s.before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (at + i >= a.blocks) break;
        const bool moves = u[i] > 0 && number < a.blocks_to;
        a.numbers[at + i] = moves ? number : -1;
        if (moves) {
            a.sources[number] = (int32_t)(at + i);
            a.users_to[number] = u[i];
        }
        number += u[i] > 0;
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) {
        const int32_t all = before + s.all;
        *a.count = min(all, a.blocks_to);
        *a.missing = max(all - a.blocks_to, 0);
    }
}

__global__ __launch_bounds__(kCopyThreads) void k_compact(CompactArgs a, CopyArgs c)
{
    const int64_t thread = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x, threads = (int64_t)gridDim.x * kCopyThreads;
    for (int64_t i = thread; i < (int64_t)a.batch * a.width; i += threads) {
        const int32_t e = a.table[i];
        a.table_to[i] = (uint32_t)e < (uint32_t)a.blocks ? a.numbers[e] : -1;
    }
    for (int64_t i = *a.count + thread; i < a.blocks_to; i += threads) a.users_to[i] = 0;
    copy_blocks(c);
}

// ---- the host side ----

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

CacheView view_of(const void *cache, int32_t blocks, const fc_pages_desc *d)
{
    const KvLayout l = kv_layout(blocks, d->kv_heads, d->head_dim);
    uint8_t *const base = static_cast<uint8_t *>(const_cast<void *>(cache));
    const int64_t heads = d->kv_heads, dp = padded_dim(d->head_dim);
    return {{base, heads * 2 * kBlock * dp}, {base + l.scales, heads * 8}, {base + l.sketches, heads * ((dp + 63) / 64 * 64)}, {base + l.weights, heads * 4}};
}

int32_t check_pages(const fc_pages_desc *d)
{
    if (!d) return FC_ERR_NULL;
    if (d->blocks <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->head_dim > FC_KV_MAX_HEAD_DIM) return FC_ERR_SHAPE;
    if (d->flags & ~(uint32_t)FC_WORKSPACE_READY) return FC_ERR_DTYPE;
    if ((int64_t)d->blocks * d->kv_heads >= INT32_MAX || d->blocks > kMostBlocks) return FC_ERR_RANGE;
    return FC_OK;
}
int32_t check_table(const fc_pages_desc *d)
{
    const int32_t rc = check_pages(d);
    if (rc != FC_OK) return rc;
    if (d->batch <= 0 || d->table_width <= 0) return FC_ERR_SHAPE;
    if (d->batch > 65535 || (int64_t)d->batch * d->table_width >= INT32_MAX) return FC_ERR_RANGE;
    return FC_OK;
}
int32_t check_to(const fc_pages_desc *d)
{
    if (d->blocks_to <= 0) return FC_ERR_SHAPE;
    if ((int64_t)d->blocks_to * d->kv_heads >= INT32_MAX || d->blocks_to > kMostBlocks) return FC_ERR_RANGE;
    return FC_OK;
}

// Workspace: offsets of its parts.
struct Parts {
    size_t wanted, own, offsets, given, rows, lengths, bytes;
};
Parts parts_of(const fc_pages_desc *d, bool fork)
{
    Parts p;
    const size_t batch = align_up((size_t)d->batch * 4, 256);
    p.wanted = 256;
    p.own = p.wanted + batch;
    p.offsets = p.own + batch;
    p.given = p.offsets + batch;
    p.rows = p.given + align_up((size_t)d->blocks * 4, 256);
    p.lengths = p.rows + (fork ? align_up((size_t)d->batch * d->table_width * 4, 256) : 0);
    p.bytes = p.lengths + (fork ? batch : 0);
    return p;
}

PagesArgs args_of(const fc_pages_desc *d, int32_t *users, int32_t *table, int32_t *lengths, const int32_t *parents, int32_t *missing, void *workspace, const Parts &p)
{
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    auto at = [&](size_t o) { return reinterpret_cast<int32_t *>(ws + o); };
    PagesArgs a;
    a.blocks = d->blocks; a.blocks_to = d->blocks; a.batch = d->batch; a.width = d->table_width;
    a.users = users; a.table = table; a.lengths = lengths; a.parents = parents; a.missing = missing;
    a.arrived = at(0); a.wanted = at(p.wanted); a.own = at(p.own); a.offsets = at(p.offsets); a.given = at(p.given); a.found = at(64);
    a.rows = at(p.rows); a.new_lengths = at(p.lengths);
    return a;
}

CopyArgs copies(const fc_pages_desc *d, const void *from, const void *to, int32_t blocks_to)
{
    CopyArgs c;
    c.from = view_of(from, d->blocks, d);
    c.to = view_of(to, blocks_to, d);
    c.blocks = d->blocks; c.blocks_to = blocks_to;
    c.sources = c.targets = nullptr;
    c.count = nullptr;
    c.most = 0;
    c.segments = (int32_t)((c.from.codes.block + kCopyBytes - 1) / kCopyBytes);
    return c;
}
CopyArgs copies_within(const fc_pages_desc *d, const void *cache)
{
    CopyArgs c = copies(d, cache, cache, d->blocks);
    c.most = d->batch;
    return c;
}
uint32_t workgroups_for(const CopyArgs &c, int64_t more)
{
    int64_t n = (int64_t)c.most * c.segments;
    if (n < more) n = more;
    return (uint32_t)(n < 1 ? 1 : n < 4096 ? n : 4096);
}

// Pointers of a call: none may be missing, all aligned.
int32_t check_pointers(std::initializer_list<const void *> pointers)
{
    for (const void *p : pointers)
        if (!p) return FC_ERR_NULL;
    for (const void *p : pointers)
        if (!aligned(p)) return FC_ERR_ALIGN;
    return FC_OK;
}
int32_t check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (!workspace || bytes < need) return FC_ERR_WORKSPACE;
    return aligned(workspace) ? FC_OK : FC_ERR_ALIGN;
}

size_t compact_bytes(const fc_pages_desc *d) { return 256 + align_up((size_t)d->blocks * 4, 256) + align_up((size_t)d->blocks_to * 4, 256); }

} // namespace

extern "C" {

int32_t fc_kv_resize_workspace_bytes(const fc_pages_desc *d, size_t *bytes)
{
    const int32_t rc = check_table(d);
    if (rc != FC_OK) return rc;
    if (!bytes) return FC_ERR_NULL;
    *bytes = parts_of(d, false).bytes;
    return FC_OK;
}

int32_t fc_kv_fork_workspace_bytes(const fc_pages_desc *d, size_t *bytes)
{
    const int32_t rc = check_table(d);
    if (rc != FC_OK) return rc;
    if (!bytes) return FC_ERR_NULL;
    *bytes = parts_of(d, true).bytes;
    return FC_OK;
}

int32_t fc_kv_compact_workspace_bytes(const fc_pages_desc *d, size_t *bytes)
{
    int32_t rc = check_table(d);
    if (rc == FC_OK) rc = check_to(d);
    if (rc != FC_OK) return rc;
    if (!bytes) return FC_ERR_NULL;
    *bytes = compact_bytes(d);
    return FC_OK;
}

int32_t fc_kv_resize(const fc_pages_desc *d, void *cache, int32_t *users, int32_t *table, const int32_t *lengths, int32_t *missing,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_table(d);
    if (rc == FC_OK) rc = check_pointers({cache, users, table, lengths, missing});
    if (rc != FC_OK) return rc;
    const Parts p = parts_of(d, false);
    rc = check_workspace(workspace, workspace_bytes, p.bytes);
    if (rc != FC_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const PagesArgs a = args_of(d, users, table, const_cast<int32_t *>(lengths), nullptr, missing, workspace, p);
    if (!(d->flags & FC_WORKSPACE_READY) && launch_zero_i32(a.arrived, 1, s) != hipSuccess) return FC_ERR_HIP;
    const int32_t workgroups = (d->batch + kWaves - 1) / kWaves;
    k_resize<<<dim3((uint32_t)(workgroups < kMostWorkgroups ? workgroups : kMostWorkgroups)), dim3(kThreads), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return FC_ERR_HIP;
    const CopyArgs c = copies_within(d, cache);
    k_resize_rows<<<dim3(workgroups_for(c, 1)), dim3(kCopyThreads), 0, s>>>(a, c);
    return hipGetLastError() == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_kv_fork(const fc_pages_desc *d, void *cache, int32_t *users, int32_t *table, int32_t *lengths, const int32_t *parents,
                   int32_t *missing, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_table(d);
    if (rc == FC_OK) rc = check_pointers({cache, users, table, lengths, parents, missing});
    if (rc != FC_OK) return rc;
    const Parts p = parts_of(d, true);
    rc = check_workspace(workspace, workspace_bytes, p.bytes);
    if (rc != FC_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const PagesArgs a = args_of(d, users, table, lengths, parents, missing, workspace, p);
    if (!(d->flags & FC_WORKSPACE_READY) && launch_zero_i32(a.arrived, 1, s) != hipSuccess) return FC_ERR_HIP;
    k_fork<<<dim3((uint32_t)(d->batch < kMostWorkgroups ? d->batch : kMostWorkgroups)), dim3(kThreads), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return FC_ERR_HIP;
    const CopyArgs c = copies_within(d, cache);
    k_fork_rows<<<dim3(workgroups_for(c, d->batch)), dim3(kCopyThreads), 0, s>>>(a, c);
    return hipGetLastError() == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_kv_compact(const fc_pages_desc *d, const void *cache, const int32_t *users, const int32_t *table, void *cache_to, int32_t *users_to,
                      int32_t *table_to, int32_t *missing, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_table(d);
    if (rc == FC_OK) rc = check_to(d);
    if (rc == FC_OK) rc = check_pointers({cache, users, table, cache_to, users_to, table_to, missing});
    if (rc != FC_OK) return rc;
    // (a block would be read after it was written)
    if (cache == cache_to || users == users_to || table == table_to) return FC_ERR_SHAPE;
    rc = check_workspace(workspace, workspace_bytes, compact_bytes(d));
    if (rc != FC_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    CompactArgs a;
    a.blocks = d->blocks; a.blocks_to = d->blocks_to; a.batch = d->batch; a.width = d->table_width;
    a.users = users; a.table = table; a.users_to = users_to; a.table_to = table_to; a.missing = missing;
    a.count = reinterpret_cast<int32_t *>(ws);
    a.numbers = reinterpret_cast<int32_t *>(ws + 256);
    a.sources = reinterpret_cast<int32_t *>(ws + 256 + align_up((size_t)d->blocks * 4, 256));
    k_number<<<dim3((uint32_t)((d->blocks + kNumbered - 1) / kNumbered)), dim3(kThreads), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return FC_ERR_HIP;
    CopyArgs c = copies(d, cache, cache_to, d->blocks_to);
    c.sources = a.sources;
    c.count = a.count;
    c.most = d->blocks < d->blocks_to ? d->blocks : d->blocks_to;
    k_compact<<<dim3(workgroups_for(c, ((int64_t)d->batch * d->table_width + d->blocks_to) / 2048)), dim3(kCopyThreads), 0, s>>>(a, c);
    return hipGetLastError() == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_kv_copy(const fc_pages_desc *d, const void *cache, const int32_t *sources, void *cache_to, const int32_t *targets, void *stream)
{
    int32_t rc = check_pages(d);
    if (rc == FC_OK) rc = check_to(d);
    if (rc != FC_OK) return rc;
    if (d->pairs < 0 || (cache && cache == cache_to && d->blocks_to != d->blocks)) return FC_ERR_SHAPE;
    if (d->pairs == 0) return FC_OK;
    rc = check_pointers({cache, sources, cache_to, targets});
    if (rc != FC_OK) return rc;
    CopyArgs c = copies(d, cache, cache_to, d->blocks_to);
    c.sources = sources; c.targets = targets;
    c.most = d->pairs;
    k_copy<<<dim3(workgroups_for(c, 1)), dim3(kCopyThreads), 0, static_cast<hipStream_t>(stream)>>>(c);
    return hipGetLastError() == hipSuccess ? FC_OK : FC_ERR_HIP;
}

} // extern "C"
