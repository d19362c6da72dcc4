// C ABI of the matrix product and of group norm: argument checks on the host, then launches.
#include "fc_layers_internal.hpp"
#include <math.h>

using namespace fc;

namespace {

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool stride_ok(int64_t stride, int64_t least) { return stride >= least && stride <= FC_LAYERS_MAX_STRIDE; }
int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }
int size_of(int32_t dtype) { return dtype == FC_F32 ? 4 : 2; }

// ---- the matrix product ----

int32_t check_linear(const fc_linear_desc *d, bool residual)
{
    if (!d) return FC_ERR_NULL;
    if (d->rows < 0 || d->n <= 0 || d->k <= 0) return FC_ERR_SHAPE;
    if (d->dtype != FC_BF16 && d->dtype != FC_F16) return FC_ERR_DTYPE;
    if (d->out_dtype != d->dtype && d->out_dtype != FC_F32) return FC_ERR_DTYPE;
    if (d->activation < FC_ACT_NONE || d->activation > FC_ACT_GELU) return FC_ERR_DTYPE;
    if (d->flags & ~(uint32_t)(FC_RESIDUAL_FIRST | FC_WORKSPACE_READY | FC_ANY_POINTERS | FC_COUNTED) || d->reserved) return FC_ERR_DTYPE;
    if (d->x_row < 0 || d->w_row < 0 || d->residual_row < 0 || d->out_row < d->n) return FC_ERR_SHAPE;
    if (d->k > FC_LAYERS_MAX_STRIDE || d->n > FC_LAYERS_MAX_STRIDE) return FC_ERR_RANGE;
    if (!stride_ok(d->x_row, 0) || !stride_ok(d->w_row, 0) || !stride_ok(d->out_row, 0) || (residual && !stride_ok(d->residual_row, 0))) return FC_ERR_RANGE;
    return FC_OK;
}

// What a cut of the product takes, in microseconds: beginning and ending a launch, its rounds of stages of 64, the weights' bytes where the kernel waits for
// them, and joining pieces.  From times of every form on 41 products (64 .. 4096 rows, 256 .. 8192 columns of x, 1024 .. 16384 of out), which it gives to within a fifth or
// so; what it is for is the order of the forms.  Measured there, rows x k x n (rings, which have become 0.2 to 0.5 us shorter since / shared stages / tiles of 128 / of 256):
//   64 x 4096 x 4096 14.7 / 15.0 in four pieces      128 x 1024 x 1024 6.0 / 10.8 / 11.3         256 x 4096 x 4096 30.6 / 23.1 in four / 25.1 in four
//   512 x 4096 x 4096 59.5 / 30.1 in two / 35.3      1024 x 4096 x 4096 121 / 43.6 / 52.4 / 80.8   2048 x 4096 x 4096 - / - / 71.2 / 82.5
//   4096 x 4096 x 4096 - / - / 141 / 100             2048 x 8192 x 1024 - / - / 51.6 in four, 87.4 in one / 146
// Rows of any alignment (through registers / laid out anew for tiles of 128 / of 256): 128 x 4097 x 4095 26 in eight / 37 in four / -, 512 x 4097 x 4095 44 in two / 54 / 111,
// 2048 x 4097 x 4095 127 / 87 / 117, 2048 x 4097 x 16383 493 / 329 / 292.
struct Cut {
    double us;
    int32_t form, tile_m, tile_n, splits;
    bool ring;
};
double rounds_of(int64_t units) { return (double)((units + 255) / 256); }
// tiles of 128 columns; rows of a tile over 128
double join_us(int64_t units, int32_t splits, double rows) { return splits > 1 ? 2.5 + 0.03 * (double)units * rows : 0.; }

Cut best_cut(int32_t rows, int32_t n, int32_t k, bool wide)
{
    const int32_t chunks = ceil_div(k, kLinearK);
    const double weights = 2e-6 * (double)n * (double)k / 6.;
    Cut best = {1e30, 0, 0, 0, 1, false};
    auto take = [&](const Cut &c) {
        if (c.us < best.us) best = c;
    };
    // rings: a wave's steps; of 64, 32 or 16 rows and 16, 32 or 64 columns
    const int32_t ring_m = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    static const double step_us[3][3] = {{0.2, 0.3, 0.}, {0.25, 0.33, 0.45}, {0.36, 0.5, 0.67}};
    for (int32_t i = 0; i < (!wide ? 0 : ring_m == 16 ? 2 : 3); ++i) {
        const int64_t units = (int64_t)ceil_div(rows, ring_m) * ceil_div(n, 16 << i);
        const double steps = ceil_div(chunks, ring_m == 64 || i == 2 ? 4 : 8);
        // (several tiles of rows: the weights come from the L2, and the steps wait for it as the chip fills)
        const double full = rows > ring_m ? 1. + 0.6 * (double)(units < 256 ? units : 256) / 256. : 1.;
        take({1.2 + rounds_of(units) * (2. + steps * step_us[ring_m / 32][i] * full) + weights, 0, ring_m, 16 << i, 1, true});
    }
    // rows of any alignment straight into fragments (us, so / through LDS: 1 x 1001 x 4095 5.8 / 9.1, 1 x 8191 x 1023 11.7 / 15.6, 32 x 1001 x 4095 9.8 / 10.4; 16 x 4097 x 4095
    // 28.4 / 17.4, 1 x 4097 x 16383 60 / 37)
    if (!wide && rows <= 32 && (double)n * (double)k * (1. + rows / 16.) <= 16777216.) {
        const int32_t units = ceil_div(n, 16), wanted = ceil_div(256, units), most = chunks < 16 ? 1 : chunks / 8;
        return {0., 0, ring_m, 16, wanted < most ? wanted : most, false};
    }
    // laying both operands out anew
    const double pad = wide ? 0. : 4. + 4e-6 / 8. * ((double)rows + (double)n) * (double)k;
    for (int32_t splits = 1; splits <= 16; splits *= 2) {
        if (splits > 1 && chunks / splits < 2) break;
        const int32_t stages = ceil_div(chunks, splits);
        // shared stages
        const int32_t m = rows <= 64 ? 64 : 128;
        const int64_t units = (int64_t)ceil_div(rows, m) * ceil_div(n, 128) * splits;
        const double stage_us = wide ? (m == 64 ? 0.31 : units < 256 ? 0.45 : 0.5) : m == 64 ? 0.8 : 1.05;
        take({(wide ? 1. : 3.) + rounds_of(units) * (2.5 + stages * stage_us) + (wide ? (m == 64 ? 0.85 : 0.7) * weights : 0.) + join_us(units, splits, wide || units > 256 ? m / 128. : m / 384.), 2, m, 128, splits, false});
        // tiles of 128: two on a CU
        if (rows > 64 && splits <= 8) {
            const int64_t u = (int64_t)ceil_div(rows, 128) * ceil_div(n, 128) * splits;
            take({3.5 + pad + stages * (u <= 256 ? 0.8 : 1.1 * (double)((u + 511) / 512)) + join_us(u, splits, 1.), 1, 128, 128, splits, false});
        }
    }
    const int64_t large = (int64_t)ceil_div(rows, 256) * ceil_div(n, 256);
    take({3.5 + pad + rounds_of(large) * (5. + chunks * (1.2 + 0.2 * (large < 256 ? large : 256) / 256.)), 3, 256, 256, 1, false});
    return best;
}

int32_t plan_linear(const fc_linear_desc *d, LinearPlan *p)
{
    const int32_t rows = d->rows < 1 ? 1 : d->rows, chunks = ceil_div(d->k, kLinearK);
    const bool pieces = d->k % 8 == 0 && !(d->flags & FC_ANY_POINTERS), x_pieces = pieces && d->x_row % 8 == 0, w_pieces = pieces && d->w_row % 8 == 0;
    p->padded_k = (int64_t)chunks * kLinearK;
    p->pad_x = p->pad_w = false;
    p->wide = x_pieces && w_pieces;
    p->per_wave = 0;
    // (half of the rows, as a mask that keeps about half leaves them: 1924 of 4811 rows of 1001 with 515 columns in two pieces, a plan for all of them in one.  It is a guess: the count is the device's)
    const Cut c = best_cut(d->flags & FC_COUNTED ? (rows + 1) / 2 : rows, d->n, d->k, p->wide);
    p->form = c.form;
    p->ring = c.ring;
    p->tile_m = c.tile_m;
    p->tile_n = c.tile_n;
    p->splits = c.splits;
    if (p->form == 1 || p->form == 3) {
        p->pad_x = !x_pieces;
        p->pad_w = !w_pieces;
    }
    p->m_tiles = ceil_div(rows, p->tile_m);
    p->n_tiles = ceil_div(d->n, p->tile_n);
    p->per_split = ceil_div(chunks, p->splits);
    p->splits = ceil_div(chunks, p->per_split);
    if (p->form == 0) p->per_wave = ceil_div(p->per_split, p->ring && (p->tile_m == 64 || p->tile_n == 64) ? 4 : 8);
    const int64_t tiles = (int64_t)p->m_tiles * p->n_tiles;
    if (tiles * p->splits >= INT32_MAX / 512) return FC_ERR_RANGE;      // (a dimension of a grid is counted in threads)
    p->counters = p->splits == 1 ? 0 : align_up((size_t)tiles * sizeof(int32_t), 256);
    p->at_x = p->counters;
    p->at_w = p->at_x + (p->pad_x ? (size_t)rows * p->padded_k * 2 : 0);
    p->at_part = align_up(p->at_w + (p->pad_w ? (size_t)d->n * p->padded_k * 2 : 0), 256);
    p->workspace = p->splits == 1 ? p->at_part : p->at_part + (size_t)tiles * p->splits * p->tile_m * p->tile_n * sizeof(float);
    return FC_OK;
}

hipError_t launch_linear_large(const LinearArgs &a, const LinearPlan &p, int dtype, int out_dtype, hipStream_t s)
{
    if (dtype == FC_BF16) return out_dtype == FC_F32 ? launch_large_as<FC_BF16, float>(a, p, s) : launch_large_as<FC_BF16, bf16_t>(a, p, s);
    return out_dtype == FC_F32 ? launch_large_as<FC_F16, float>(a, p, s) : launch_large_as<FC_F16, f16_t>(a, p, s);
}

// ---- group norm ----

int32_t check_norm(const fc_group_norm_desc *d)
{
    if (!d) return FC_ERR_NULL;
    if (d->images <= 0 || d->rows < 0 || d->max_rows < 0 || d->channels <= 0 || d->groups <= 0 || d->channels % d->groups) return FC_ERR_SHAPE;
    if (d->dtype != FC_F32 && d->dtype != FC_BF16 && d->dtype != FC_F16) return FC_ERR_DTYPE;
    if (d->activation < FC_ACT_NONE || d->activation > FC_ACT_GELU) return FC_ERR_DTYPE;
    if (d->flags & ~(uint32_t)(FC_SKIP_ZERO_FILL | FC_WORKSPACE_READY | FC_ANY_POINTERS) || d->reserved) return FC_ERR_DTYPE;
    if (!(d->eps >= 0.f) || !isfinite(d->eps) || d->x_row < 0 || d->out_row < d->channels) return FC_ERR_SHAPE;
    if (d->channels > FC_LAYERS_MAX_STRIDE || d->channels / d->groups > FC_GROUP_MAX_CHANNELS) return FC_ERR_RANGE;
    if (d->max_rows > FC_NORM_MAX_ROWS) return FC_ERR_RANGE;
    if (!stride_ok(d->x_row, 0) || !stride_ok(d->out_row, 0)) return FC_ERR_RANGE;
    return FC_OK;
}

constexpr int kOnceGroups = 512;        // of a slice, at most
constexpr int kNormGrid = 256;          // workgroups of the kernels with chunks

// (wide: in pieces of 16 bytes, which the rows have to be made of)
int32_t plan_norm_as(const fc_group_norm_desc *d, bool wide, NormPlan *p)
{
    const int32_t size = size_of(d->dtype), ve = 16 / size, per_group = d->channels / d->groups;
    p->wide = wide;
    const int32_t e = p->wide ? ve : 1;         // elements of a piece
    // the least slices: whole groups, whole pieces, and 32 bytes where the groups divide so that they are not long
    int32_t least = 1;
    while (least < d->groups && (d->groups % least || least * per_group % e)) ++least;
    for (int32_t of = least; of <= d->groups && of * per_group <= 4096; ++of)
        if (d->groups % of == 0 && of * per_group % e == 0 && of * per_group * size >= 32) {
            least = of;
            break;
        }
    auto entries = [&](int32_t channels) { return per_group % e == 0 ? channels / e : channels; };
    // an image's slice in the registers of a workgroup: up to 1024 threads with 12 pieces each
    p->slice = least * per_group;
    const int32_t pieces = p->slice / e;
    p->once = false;
    if (least <= kOnceGroups && pieces <= 1024) {
        const int32_t threads[] = {256, 512, 1024};
        for (int i = 0; i < 6 && !p->once; ++i) {
            p->threads = threads[i % 3];
            p->per_thread = i < 3 ? 4 : 12;
            if (pieces > p->threads) continue;
            const int32_t phases = p->threads / pieces;
            p->lds = (size_t)phases * (entries(p->slice) * 8 + 4);
            p->once = (int64_t)phases * p->per_thread >= d->max_rows && p->lds <= 60000;
        }
    }
    p->chunks = p->chunk_rows = 1;
    if (!p->once) {
        // whole rows; shorter slices where rows are longer than 4096 channels, or have more than 64 groups and are longer than 512 bytes
        int32_t of = d->groups;
        while (of > least && ((int64_t)of * per_group > 4096 || (of > 64 && (int64_t)of * per_group * size > 512) || d->groups % of || of * per_group % e)) --of;
        p->slice = of * per_group;
        const int32_t row_pieces = p->slice / e, phases = row_pieces < 1024 ? 1024 / row_pieces : 1;
        p->lds = (size_t)phases * (entries(p->slice) * 8 + 4);
        if (p->lds > 163840) return FC_ERR_RANGE;
        // a workgroup a CU (two: outputs of 8 images of 16384 x 256 with a mask 26 -> 35 us); a chunk is no less than a round of a workgroup's loads, and an image's chunks leave no more than 128 KB to join
        const int64_t units = (int64_t)d->images * (d->channels / p->slice), most = 8192 / of < 1 ? 1 : 8192 / of;
        int64_t wanted = (kNormGrid + units - 1) / units;
        if (wanted > most) wanted = most;
        const int64_t least_rows = (int64_t)phases * 4;
        int64_t rows = (d->max_rows + wanted - 1) / wanted;
        rows = (rows + least_rows - 1) / least_rows * least_rows;
        p->chunk_rows = (int32_t)(rows < 1 ? 1 : rows > INT32_MAX / 2 ? INT32_MAX / 2 : rows);
        p->chunks = ceil_div(d->max_rows, p->chunk_rows);
        if (p->chunks < 1) p->chunks = 1;
        p->threads = 1024;
    }
    p->slices = d->channels / p->slice;
    const int64_t units = (int64_t)d->images * p->slices;
    if (units * p->chunks >= (1ll << 32) / 1024) return FC_ERR_RANGE;       // (a dimension of a grid is counted in threads)
    p->workspace = p->once ? 0 : (size_t)d->images * p->chunks * d->groups * 16;
    return FC_OK;
}

int32_t plan_norm(const fc_group_norm_desc *d, NormPlan *p)
{
    const int32_t ve = 16 / size_of(d->dtype);
    const bool wide = !(d->flags & FC_ANY_POINTERS) && d->channels % ve == 0 && d->x_row % ve == 0 && d->out_row % ve == 0;
    const int32_t rc = plan_norm_as(d, wide, p);
    // (long groups that are not whole pieces: several of them that are together may have more entries than LDS holds; one of them by elements never has)
    return wide && rc == FC_ERR_RANGE ? plan_norm_as(d, false, p) : rc;
}

} // namespace

extern "C" {

int32_t fc_linear_workspace_bytes(const fc_linear_desc *d, size_t *bytes)
{
    if (!bytes) return FC_ERR_NULL;
    int32_t rc = check_linear(d, true);
    if (rc != FC_OK) return rc;
    LinearPlan p;
    rc = plan_linear(d, &p);
    if (rc == FC_OK) *bytes = d->rows == 0 ? 0 : p.workspace;
    return rc;
}

int32_t fc_linear_cut_of(const fc_linear_desc *d, fc_linear_cut *cut)
{
    if (!cut) return FC_ERR_NULL;
    int32_t rc = check_linear(d, true);
    if (rc != FC_OK) return rc;
    LinearPlan p;
    rc = plan_linear(d, &p);
    if (rc != FC_OK) return rc;
    cut->kernel = p.form == 0 ? (p.ring ? FC_LINEAR_RINGS : FC_LINEAR_ROWS) : p.form == 1 ? FC_LINEAR_TILES : p.form == 3 ? FC_LINEAR_LARGE
                  : p.wide ? FC_LINEAR_STAGES : FC_LINEAR_STAGES_ANY;
    cut->tile_rows = p.tile_m;
    cut->tile_columns = p.tile_n;
    cut->pieces = p.splits;
    cut->anew_x = p.pad_x;
    cut->anew_w = p.pad_w;
    return FC_OK;
}

int32_t fc_group_norm_workspace_bytes(const fc_group_norm_desc *d, size_t *bytes)
{
    if (!bytes) return FC_ERR_NULL;
    int32_t rc = check_norm(d);
    if (rc != FC_OK) return rc;
    NormPlan p;
    rc = plan_norm(d, &p);
    if (rc == FC_OK) *bytes = d->rows == 0 ? 0 : p.workspace;
    return rc;
}

int32_t fc_linear(const fc_linear_desc *d, const void *x, const void *w, const float *bias, const void *residual, const int32_t *count,
                  void *out, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_linear(d, residual != nullptr);
    if (rc != FC_OK) return rc;
    const int size = size_of(d->out_dtype);
    LinearPlan p;
    rc = plan_linear(d, &p);
    if (rc != FC_OK) return rc;
    if (d->rows == 0) return FC_OK;
    if (!x || !w || !out) return FC_ERR_NULL;
    const uintptr_t least = d->flags & FC_ANY_POINTERS ? 2 : 16;
    if (!aligned(x, least) || !aligned(w, least) || !aligned(out, size) || (residual && !aligned(residual, size)) || (bias && !aligned(bias, 16)) ||
        (count && !aligned(count, 16)))
        return FC_ERR_ALIGN;
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return FC_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return FC_ERR_ALIGN;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    LinearArgs a;
    a.x = static_cast<const uint16_t *>(x);
    a.w = static_cast<const uint16_t *>(w);
    a.bias = bias;
    a.residual = residual;
    a.out = out;
    a.count = count;
    a.rows = d->rows; a.n = d->n; a.k = d->k; a.act = d->activation;
    a.residual_first = (d->flags & FC_RESIDUAL_FIRST) != 0;
    a.wide_out = d->n % 8 == 0 && aligned(out, 16) && d->out_row * size % 16 == 0 && (!residual || (aligned(residual, 16) && d->residual_row * size % 16 == 0));
    a.x_row = d->x_row; a.w_row = d->w_row; a.residual_row = d->residual_row; a.out_row = d->out_row;
    a.m_tiles = p.m_tiles; a.n_tiles = p.n_tiles; a.splits = p.splits; a.per_split = p.per_split; a.per_wave = p.per_wave;
    a.part = reinterpret_cast<float *>(ws + p.at_part);
    a.arrived = reinterpret_cast<int32_t *>(ws);
    hipError_t e = hipSuccess;
    if (p.counters && !(d->flags & FC_WORKSPACE_READY)) e = launch_zero_i32(a.arrived, p.m_tiles * p.n_tiles, s);
    if (e == hipSuccess && (p.pad_x || p.pad_w)) {
        uint16_t *const px = p.pad_x ? reinterpret_cast<uint16_t *>(ws + p.at_x) : nullptr, *const pw = p.pad_w ? reinterpret_cast<uint16_t *>(ws + p.at_w) : nullptr;
        e = launch_linear_pad(a, p, px, pw, s);
        if (px) a.x = px, a.x_row = p.padded_k;
        if (pw) a.w = pw, a.w_row = p.padded_k;
        if (px && pw) a.k = (int32_t)p.padded_k;
    }
    if (e == hipSuccess)
        e = p.form == 0 ? launch_linear_rows(a, p, d->dtype, d->out_dtype, s) : p.form == 1 ? launch_linear_tile(a, p, d->dtype, d->out_dtype, s)
            : p.form == 2 ? launch_linear_stream(a, p, d->dtype, d->out_dtype, s) : launch_linear_large(a, p, d->dtype, d->out_dtype, s);
    return e == hipSuccess ? FC_OK : FC_ERR_HIP;
}

int32_t fc_group_norm(const fc_group_norm_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *mask,
                      const int32_t *starts, void *out, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_norm(d);
    if (rc != FC_OK) return rc;
    if (!starts && (int64_t)d->images * d->max_rows != d->rows) return FC_ERR_SHAPE;
    NormPlan p;
    rc = plan_norm(d, &p);
    if (rc != FC_OK) return rc;
    if (d->rows == 0 || d->max_rows == 0) return FC_OK;
    if (!x || !out) return FC_ERR_NULL;
    const uintptr_t least = d->flags & FC_ANY_POINTERS ? size_of(d->dtype) : 16;
    if (!aligned(x, least) || !aligned(out, least) || (weight && !aligned(weight, 16)) || (bias && !aligned(bias, 16)) || (mask && !aligned(mask, 16)) ||
        (starts && !aligned(starts, 16)))
        return FC_ERR_ALIGN;
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return FC_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return FC_ERR_ALIGN;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    NormArgs a;
    a.x = x; a.out = out; a.weight = weight; a.bias = bias; a.mask = mask; a.starts = starts;
    a.images = d->images; a.rows = d->rows; a.max_rows = d->max_rows; a.channels = d->channels; a.groups = d->groups;
    a.per_group = d->channels / d->groups;
    a.act = d->activation;
    a.keep_out = (d->flags & FC_SKIP_ZERO_FILL) != 0;
    a.eps = d->eps;
    a.x_row = d->x_row; a.out_row = d->out_row;
    a.slices = p.slices; a.slice = p.slice; a.chunks = p.chunks; a.chunk_rows = p.chunk_rows;
    a.part = static_cast<float4 *>(workspace);
    return launch_group_norm(a, p, d->dtype, s) == hipSuccess ? FC_OK : FC_ERR_HIP;
}

} // extern "C"
