// C ABI of the attention operators: argument checks on the host, then launches.
#include "fc_attn_internal.hpp"
#include <float.h>
#include <math.h>

using namespace fc;

namespace {

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Fields that describe the cache.
int32_t check_cache(const fc_attention_desc *d)
{
    if (!d) return FC_ERR_NULL;
    if (d->blocks <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->head_dim > FC_KV_MAX_HEAD_DIM) return FC_ERR_SHAPE;
    if ((int64_t)d->blocks * d->kv_heads >= INT32_MAX) return FC_ERR_RANGE;
    return FC_OK;
}

// Those and the sequences.
int32_t make_kv_geom(const fc_attention_desc *d, const void *cache, const int32_t *table, const int32_t *lengths, const int32_t *starts, KvGeom *g)
{
    const int32_t rc = check_cache(d);
    if (rc != FC_OK) return rc;
    if (d->batch <= 0 || d->tokens < 0 || d->max_new <= 0 || d->max_len <= 0 || d->table_width <= 0) return FC_ERR_SHAPE;
    if (d->flags & ~(uint32_t)(FC_CAUSAL | FC_WORKSPACE_READY) || d->reserved) return FC_ERR_DTYPE;
    // (one dimension of a grid)
    if (d->batch > 65535 || d->kv_heads > 65535) return FC_ERR_RANGE;
    if (!starts && d->tokens && (int64_t)d->batch * d->max_new != d->tokens) return FC_ERR_SHAPE;
    const KvLayout l = kv_layout(d->blocks, d->kv_heads, d->head_dim);
    uint8_t *const base = static_cast<uint8_t *>(const_cast<void *>(cache));
    g->blocks = d->blocks; g->kv_heads = d->kv_heads; g->d = d->head_dim; g->dp = padded_dim(d->head_dim);
    g->batch = d->batch; g->tokens = d->tokens; g->max_new = d->max_new; g->width = d->table_width;
    const int64_t held = (int64_t)d->table_width * kBlock;
    g->max_len = held < d->max_len ? (int32_t)held : d->max_len;
    g->codes = base;
    g->scales = reinterpret_cast<float2 *>(base + l.scales);
    g->sketches = reinterpret_cast<int8_t *>(base + l.sketches);
    g->weights = reinterpret_cast<float *>(base + l.weights);
    g->table = table; g->lengths = lengths; g->starts = starts;
    return FC_OK;
}

// One dimension of a grid is counted in threads.
bool grid_fits(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }

// A workgroup of 256 threads a touched block and head.
bool blocks_fit(const KvGeom &g) { return grid_fits(((int64_t)touched_blocks(g) + 1) * g.kv_heads, 256); }

int32_t check_pointers(const void *cache, const int32_t *table, const int32_t *lengths, const int32_t *starts)
{
    if (!cache || !table || !lengths) return FC_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(table, 16) || !aligned(lengths, 16) || (starts && !aligned(starts, 16))) return FC_ERR_ALIGN;
    return FC_OK;
}

// Are rows of `d` channels with these strides whole 16-byte pieces?
bool wide_rows(const void *p, int64_t row, int64_t head, int32_t d) { return aligned(p, 16) && row % 8 == 0 && head % 8 == 0 && d % 8 == 0; }

bool known_type(int32_t dtype) { return dtype == FC_BF16 || dtype == FC_F16; }

// How a call's rows and blocks are cut.
struct Plan {
    int32_t rows_tile, tiles, splits, per_split, waves;
    int64_t units;              // of rows: sequences x key heads x tiles
    bool whole;                 // a wave takes a token's whole list
    int32_t shared, mask_words, entries;        // ... or those of several tokens
    size_t counters, workspace; // bytes; none where nothing is split
};

// Pieces of the long axis where memory is the bound: eight waves a CU, as many as are there at once, and no piece of less than a block a wave.  More pieces
// balance nothing and take longer to join; up to two blocks a wave are one piece (us, in pieces -> in one: one sequence of 300 / 500 / 1000 tokens
// 8.0 / 8.1 / 8.4 -> 7.3 / 7.5 / 9.6).
void cut_to_fill(int64_t units, int32_t blocks, int waves, int32_t *splits, int32_t *per_split)
{
    const int64_t workgroups = 2048 / waves, most = blocks <= 2 * waves ? 1 : (blocks + waves - 1) / waves;
    int64_t n = (workgroups + units - 1) / units;
    n = n < 1 ? 1 : n > most ? most : n;
    *per_split = (int32_t)((blocks + n - 1) / n + waves - 1) / waves * waves;
    *splits = (blocks + *per_split - 1) / *per_split;
}

// ... and where the matrix cores are: one piece where the rows are a workgroup for every CU (us, in one piece -> in two: 4096 tokens of 32 heads of 128 over 8
// 144 -> 216, 3000 87 -> 131, 1024 28 -> 29), else as many as take the least time.  In tenths of a block's time of a workgroup that has its CU for itself: two on
// a CU take 1.4 times as long each, and the launch no less than its longest piece or its share of all of them; four blocks' time goes to beginning and ending
// a piece, three to joining one.  `units` is what the call's rows come to and `mean` the blocks that a row sees on average.  (512 tokens after 16000 329 -> 154
// in four pieces, 128 after 4000, a key head a head, 87 -> 39.)
void cut_for_rounds(int64_t units, int32_t blocks, int32_t mean, int32_t *splits, int32_t *per_split)
{
    int64_t best = 0;
    *splits = 1, *per_split = blocks;
    for (int64_t n = 1; n <= (units < 256 ? 64 : 1) && n <= blocks; ++n) {
        const int64_t per = (blocks + n - 1) / n, pieces = (blocks + per - 1) / per, workgroups = units * ((mean + per - 1) / per);
        const int64_t share = (units * mean + 4 * workgroups) / 512;
        const int64_t cost = (workgroups <= 256 ? 10 : 14) * (share > per + 4 ? share : per + 4) + (pieces > 1 ? 32 * pieces : 0);
        if (n == 1 || cost < best) {
            best = cost;
            *splits = (int32_t)pieces;
            *per_split = (int32_t)per;
        }
    }
}

// Lists: from this many on there are enough to fill the chip with a wave each (us of the whole call, split -> whole, 9 / 16 / 32 blocks of 8 key heads of 128 with 4 queries
// each, over 313: 512 units 30.0 / 36.6 / 48.8 -> 30.4 / 38.0 / 52.7, 768 35.5 / 43.1 / 56.6 -> 30.8 / 38.2 / 52.8, 1024 38.6 / 46.5 / 59.8 -> 31.0 / 38.3 / 53.0, 2800
// 59.7 / 73.0 / 107 -> 45.5 / 61.5 / 97; 9 blocks of 2 key heads of 96 with 5: 512 26.1 -> 28.8, 768 28.0 -> 29.2, 1024 31.6 -> 29.4, 2800 45.6 -> 38.9).
constexpr int64_t kWholeLists = 1024;
// Neighbouring tokens' lists together: from this many waves on (us, apart -> together, lists of 16 blocks of 8 key heads of 128, keys that select independently:
// 4 heads a key head, 512 / 1024 / 2048 / 4096 tokens (1024 waves on) 79 / 132 / 245 / 475 -> 81 / 114 / 203 / 389; one head a key head, 4096 tokens 469 -> 333;
// tokens that select alike gain as much more as they share).
constexpr int64_t kSharedLists = 2048;

int32_t make_plan(const fc_attention_desc *d, const KvGeom &g, bool list, Plan *p)
{
    if (d->heads <= 0 || d->heads % d->kv_heads) return FC_ERR_SHAPE;
    if (!known_type(d->dtype)) return FC_ERR_DTYPE;
    if (!isfinite(d->scale) || d->q_row < 0 || d->q_head < 0) return FC_ERR_SHAPE;
    const int32_t group = d->heads / d->kv_heads;
    if ((int64_t)d->tokens * d->heads >= INT32_MAX || (int64_t)d->max_new * group >= INT32_MAX / 2) return FC_ERR_RANGE;
    const int64_t rows = (int64_t)d->max_new * group;
    int32_t blocks = (g.max_len + kBlock - 1) / kBlock;
    p->shared = 1, p->mask_words = p->entries = 0;
    if (list) {
        if (d->first < 0 || d->last < 1 || d->top < 0 || d->first > FC_MAX_SELECTED || d->last > FC_MAX_SELECTED || d->top > FC_MAX_SELECTED ||
            d->first + d->last + d->top > FC_MAX_SELECTED)
            return FC_ERR_SHAPE;
        if (blocks > kSelectMaxBlocks || group > kMostGroup) return FC_ERR_RANGE;
        const int32_t width = d->first + d->last + d->top, all = blocks;
        blocks = blocks < width ? blocks : width;
        p->rows_tile = 16;
        p->tiles = d->max_new * ((group + 15) / 16);
        const int32_t together = group <= 8 ? 16 / group : 1;
        const int32_t tiles = (d->max_new + together - 1) / together;
        if (together > 1 && all <= kSharedMaxBlocks && (int64_t)d->batch * d->kv_heads * tiles >= kSharedLists) {
            p->shared = together;
            p->tiles = tiles;
            p->mask_words = (all + 1) / 2;
            p->entries = (int64_t)together * width < all ? together * width : all;
        }
    } else {
        // 256 rows share a block's conversion where there are enough of them for two rounds of a workgroup a CU (us, 128 -> 256 rows, 32 heads of 128 over 8:
        // 8192 tokens 565 -> 544, 4096 158 -> 148, two times 2048 after 16000 996 -> 932; 2048 56 -> 83; of 96: 8192 481 -> 459, 4096 137 -> 125, of 80, two times 3000 over
        // 9000, 634 -> 601; of 64, where a block is as soon converted: 8192 357 -> 365, 4096 107 -> 101, not taken)
        const int64_t large = (rows + 255) / 256 * d->batch * d->kv_heads;
        p->rows_tile = rows <= 16 ? 16 : rows <= 32 && g.dp <= 128 ? 32 : large >= 512 && (g.dp == 96 || g.dp == 128) ? 256 : 128;
        p->tiles = (int32_t)((rows + p->rows_tile - 1) / p->rows_tile);
    }
    const int64_t units = p->units = (int64_t)d->batch * d->kv_heads * p->tiles;
    p->whole = list && (p->shared > 1 || units >= kWholeLists);
    if (p->whole) {
        p->per_split = blocks;
        p->splits = 1;
    } else if (p->rows_tile >= 128) {
        const int64_t filled = ((int64_t)d->tokens * group / p->rows_tile + (d->batch + 1) / 2) * d->kv_heads;
        const int32_t mean = d->flags & FC_CAUSAL ? blocks - d->max_new / (2 * kBlock) : blocks;
        cut_for_rounds(filled < units ? filled : units, blocks, mean < 1 ? 1 : mean, &p->splits, &p->per_split);
    } else {
        p->waves = 4;
        cut_to_fill(units, blocks, p->waves, &p->splits, &p->per_split);
        // Few sequences over long axes: half as many pieces of eight waves (us at 4 -> 8 waves, tokens of sequences with 8 key heads of 128: one of 2000 /
        // 4000 / 8000 / 16000 / 32000 8.9 / 9.8 / 12.6 / 19.8 / 25.4 -> 10.0 / 10.6 / 11.4 / 13.4 / 19.5, two of 16000 22.7 -> 19.2, four of 8000
        // 18.9 -> 18.9, 64 of 2000 44.2 -> 47.2)
        if (!list && p->rows_tile == 16 && g.dp <= 128 && p->splits > 16) {
            p->waves = 8;
            cut_to_fill(units, blocks, p->waves, &p->splits, &p->per_split);
        }
    }
    if (units * p->splits >= INT32_MAX || (int64_t)p->splits * p->rows_tile * g.dp * 4 >= INT32_MAX) return FC_ERR_RANGE;
    if (list) {
        const int32_t tokens = select_tokens(g);
        if (!grid_fits((int64_t)d->batch * d->kv_heads * ((d->max_new + tokens - 1) / tokens), tokens == 1 ? 1024 : 256)) return FC_ERR_RANGE;
        if (!grid_fits(p->whole ? (units + 31) / 32 * 8 : units * p->splits, 256)) return FC_ERR_RANGE;
    } else if (!grid_fits(units * p->splits, p->rows_tile <= 32 ? 64 * p->waves : 2 * p->rows_tile)) {
        return FC_ERR_RANGE;
    }
    p->counters = p->splits == 1 ? 0 : align_up((size_t)units * sizeof(int32_t), 256);
    p->workspace = p->counters + (p->splits == 1 ? 0 : (size_t)units * p->splits * p->rows_tile * (g.dp * sizeof(float) + sizeof(float2)));
    return FC_OK;
}

int32_t workspace_bytes(const fc_attention_desc *d, bool list, size_t *bytes)
{
    KvGeom g;
    Plan p;
    if (!bytes) return FC_ERR_NULL;
    // (whether rows are counted by starts does not matter here)
    const int32_t dummy = 0;
    int32_t rc = make_kv_geom(d, nullptr, nullptr, nullptr, &dummy, &g);
    if (rc == FC_OK) rc = make_plan(d, g, list, &p);
    if (rc == FC_OK) *bytes = p.workspace;
    return rc;
}

int32_t attend(const fc_attention_desc *d, const void *cache, const void *q, const int32_t *table, const int32_t *lengths, const int32_t *starts,
               void *out, float *lse, int32_t *selected, bool list, void *workspace, size_t workspace_bytes, void *stream)
{
    KvGeom g;
    Plan p;
    int32_t rc = make_kv_geom(d, cache, table, lengths, starts, &g);
    if (rc == FC_OK) rc = make_plan(d, g, list, &p);
    if (rc != FC_OK) return rc;
    if (d->tokens == 0) return FC_OK;
    rc = check_pointers(cache, table, lengths, starts);
    if (rc != FC_OK) return rc;
    if (!q || !out || (list && !selected)) return FC_ERR_NULL;
    if (!aligned(q, 2) || !aligned(out, 16) || (lse && !aligned(lse, 16)) || (list && !aligned(selected, 16))) return FC_ERR_ALIGN;
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return FC_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return FC_ERR_ALIGN;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    AttnArgs a;
    a.kv = g;
    a.q = static_cast<const uint16_t *>(q);
    a.q_row = d->q_row; a.q_head = d->q_head;
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    a.heads = d->heads; a.group = d->heads / d->kv_heads;
    a.causal = list || (d->flags & FC_CAUSAL);
    a.wide = wide_rows(q, d->q_row, d->q_head, d->head_dim);
    a.scale_log2 = fminf(fabsf(d->scale) * 1.44269504088896f, FLT_MAX);
    a.signs = d->scale < 0.f ? 0x80008000u : 0u;
    a.div_group = make_fastdiv((uint32_t)a.group);
    a.selected = list ? selected : nullptr;
    a.selected_width = d->first + d->last + d->top;
    a.shared = p.shared; a.mask_words = p.mask_words; a.entries = p.entries;
    a.tiles = p.tiles; a.splits = p.splits; a.per_split = p.per_split;
    a.arrived = static_cast<int32_t *>(workspace);
    a.part_out = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.counters);
    a.part_ml = reinterpret_cast<float2 *>(a.part_out + (size_t)p.units * p.splits * p.rows_tile * g.dp);
    const int32_t counters = p.counters && !(d->flags & FC_WORKSPACE_READY) ? (int32_t)p.units : 0;     // to be cleared
    hipError_t e;
    if (list) {
        e = launch_select(g, d->dtype, a.q, d->q_row, d->q_head, d->heads, a.wide, d->first, d->last, d->top, selected, a.arrived, counters, s);
        if (e == hipSuccess) e = launch_attend_lists(a, d->dtype, p.whole, s);
    } else {
        e = counters ? launch_zero_i32(a.arrived, counters, s) : hipSuccess;
        if (e == hipSuccess) e = p.rows_tile <= 32 ? launch_attend_rows(a, d->dtype, p.rows_tile, p.waves, s) : launch_attend_tile(a, d->dtype, p.rows_tile, s);
    }
    return e == hipSuccess ? FC_OK : FC_ERR_HIP;
}

} // namespace

extern "C" {

int32_t fc_kv_cache_bytes(const fc_attention_desc *d, size_t *bytes)
{
    const int32_t rc = check_cache(d);
    if (rc != FC_OK) return rc;
    if (!bytes) return FC_ERR_NULL;
    *bytes = kv_layout(d->blocks, d->kv_heads, d->head_dim).bytes;
    return FC_OK;
}

int32_t fc_kv_append(const fc_attention_desc *d, void *cache, const void *k, const void *v, const int32_t *table, const int32_t *lengths,
                     const int32_t *starts, void *stream)
{
    KvGeom g;
    int32_t rc = make_kv_geom(d, cache, table, lengths, starts, &g);
    if (rc != FC_OK) return rc;
    if (!known_type(d->dtype)) return FC_ERR_DTYPE;
    if (!blocks_fit(g) || (g.max_new == 1 && !grid_fits(((int64_t)g.batch * g.kv_heads + 3) / 4, 256))) return FC_ERR_RANGE;
    if (d->k_row < 0 || d->k_head < 0 || d->v_row < 0 || d->v_head < 0) return FC_ERR_SHAPE;
    if (d->tokens == 0) return FC_OK;
    rc = check_pointers(cache, table, lengths, starts);
    if (rc != FC_OK) return rc;
    if (!k || !v) return FC_ERR_NULL;
    if (!aligned(k, 2) || !aligned(v, 2)) return FC_ERR_ALIGN;
    return launch_kv_append(g, d->dtype, static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), d->k_row, d->k_head, d->v_row, d->v_head,
                            wide_rows(k, d->k_row, d->k_head, d->head_dim), wide_rows(v, d->v_row, d->v_head, d->head_dim),
                            static_cast<hipStream_t>(stream)) == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_kv_read(const fc_attention_desc *d, const void *cache, const int32_t *table, const int32_t *lengths, const int32_t *starts, float *k,
                   float *v, void *stream)
{
    KvGeom g;
    int32_t rc = make_kv_geom(d, cache, table, lengths, starts, &g);
    if (rc != FC_OK) return rc;
    if (!blocks_fit(g)) return FC_ERR_RANGE;
    if (d->tokens == 0) return FC_OK;
    rc = check_pointers(cache, table, lengths, starts);
    if (rc != FC_OK) return rc;
    if (!k && !v) return FC_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16)) return FC_ERR_ALIGN;
    return launch_kv_read(g, k, v, static_cast<hipStream_t>(stream)) == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_cache_attention_workspace_bytes(const fc_attention_desc *d, size_t *bytes) { return workspace_bytes(d, false, bytes); }
int32_t fc_focused_attention_workspace_bytes(const fc_attention_desc *d, size_t *bytes) { return workspace_bytes(d, true, bytes); }

int32_t fc_cache_attention(const fc_attention_desc *d, const void *cache, const void *q, const int32_t *table, const int32_t *lengths,
                           const int32_t *starts, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend(d, cache, q, table, lengths, starts, out, lse, nullptr, false, workspace, workspace_bytes, stream);
}

int32_t fc_focused_attention(const fc_attention_desc *d, const void *cache, const void *q, const int32_t *table, const int32_t *lengths,
                             const int32_t *starts, void *out, float *lse, int32_t *selected, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend(d, cache, q, table, lengths, starts, out, lse, selected, true, workspace, workspace_bytes, stream);
}

} // extern "C"
