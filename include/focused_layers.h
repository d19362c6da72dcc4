/*
 * focused_layers.h - C ABI of the layers around attention of the focused convolution library for AMD MI355X (gfx950): the matrix product
 * with what follows it, and group norm.
 *
 * fc_linear
 *   - y = sum_k x[r][k] w[n][k] + bias[n], products of the stored values accumulated in 32 bits (bias added in 32 bits);
 *     out[r][n] = act(y) + residual[r][n], or act(y + residual[r][n]) with FC_RESIDUAL_FIRST; one rounding to the output type.
 *   - x and w are FC_BF16 or FC_F16, both alike; out is of their type or FC_F32, residual is of out's type.
 *   - Rows of x, w, residual and out have a stride each (elements; columns next to each other), and any size goes.  residual and out are aligned to
 *     their element, x and w to 16 bytes, or with FC_ANY_POINTERS to their element.  Where x's or w's rows are not whole 16-byte pieces (k, stride
 *     or that flag) and there are many rows, the call first lays that operand out anew in the workspace.  x_row 0 is one row for all.  residual may be
 *     out; nothing else may overlap out.
 *   - count (device, may be NULL): the rows that there are, min(max(*count, 0), rows); out's rows behind them stay as they were.  It is what
 *     fc_active_index_compact writes, so that compacted rows need no host.
 *
 * fc_group_norm
 *   - x[rows][channels], channels last; channels / groups next to each other share their statistics over the rows of one image:
 *     y = (x - mean) / sqrt(variance + eps) * weight + bias, variance = mean of the squared distances from the mean; out = act(y), one rounding.
 *   - Images: rows / images rows each, or with starts (device, [images + 1]) rows starts[b] .. starts[b + 1], max_rows of them at most.  What starts
 *     says beyond rows or max_rows is cut off.  out's rows that belong to no image stay as they were.
 *   - mask ([rows] bytes, nonzero = relevant, may be NULL): the statistics are those of the relevant rows, what irrelevant rows hold has no influence,
 *     NaN included, and out is +0.0 there, or stays as it was with FC_SKIP_ZERO_FILL.  An image without a relevant row has no output but zeros.
 *   - x and out are FC_BF16, FC_F16 or FC_F32, both alike; weight and bias float32 [channels] or NULL (ones, zeros).  Rows of x and out have strides and are
 *     aligned to 16 bytes, or with FC_ANY_POINTERS to their element; out may be x.
 *   - Statistics in 32 bits, each thread's sums about a value of its own and joined with counts, so a mean far from zero costs no precision;
 *     the order of sums is fixed.
 *
 * Activations: y < 0 ? 0 : y; y / (1 + exp(-y)); y (1 + erf(y / sqrt(2))) / 2, in 32 bits, NaN where the formula says so (-infinity of the last two).
 *
 * Sizes beyond the limits below, and more work than a launch holds (2^31 threads; of fc_group_norm 2^32), give FC_ERR_RANGE.
 *
 * Conventions are those of focused_conv.h: device pointers, a stream, nothing allocated and no waiting, argument errors found before
 * anything is launched, launches only (calls can be captured after one eager call).  bias, weight, count, starts, mask and workspaces are
 * aligned to 16 bytes.  With FC_WORKSPACE_READY (4) in flags the caller vouches that the workspace's counters are zero, as a workspace that was zeroed
 * once has them, and from then on after every completed call of the same function with the same descriptor: it saves the launch that clears them.
 * Two calls that overlap in time need a workspace each.
 */
#ifndef FOCUSED_LAYERS_H
#define FOCUSED_LAYERS_H

#include "focused_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FC_ACT_NONE = 0, FC_ACT_RELU = 1, FC_ACT_SILU = 2, FC_ACT_GELU = 3 };

enum {
    FC_RESIDUAL_FIRST = 128u, /* fc_linear: the residual is added before the activation */
    FC_ANY_POINTERS = 256u,   /* x and w (fc_linear), x and out (fc_group_norm) are aligned to their element only; without it to 16 bytes */
    FC_COUNTED = 512u         /* fc_linear: the work is laid out for half of the rows, as a count leaves them that a mask makes.  Any count goes with it; the order of sums is
                                 that of a product of half the rows, so results are those without the flag but for the roundings of 32-bit sums */
};

enum { FC_LAYERS_MAX_STRIDE = 4194304 };    /* elements between rows, and sizes of rows */
enum { FC_GROUP_MAX_CHANNELS = 16384 };      /* channels of a group */
enum { FC_NORM_MAX_ROWS = 1073741824 };      /* rows of an image */

typedef struct {
    int32_t rows, n, k;                                   /* rows of x and out, columns of out, columns of x and w */
    int32_t dtype, out_dtype;                             /* of x and w; of out and residual */
    int32_t activation;                                   /* FC_ACT_... */
    uint32_t flags;                                       /* FC_RESIDUAL_FIRST, FC_ANY_POINTERS, FC_COUNTED, FC_WORKSPACE_READY */
    int32_t reserved;                                     /* zero */
    int64_t x_row, w_row, residual_row, out_row;          /* strides in elements; out_row >= n */
} fc_linear_desc;

typedef struct {
    int32_t images, rows, max_rows, channels, groups;     /* max_rows: of an image (without starts rows / images) */
    int32_t dtype;                                        /* of x and out */
    int32_t activation;                                   /* FC_ACT_... */
    uint32_t flags;                                       /* FC_SKIP_ZERO_FILL, FC_ANY_POINTERS, FC_WORKSPACE_READY */
    float eps;                                            /* >= 0, finite */
    int32_t reserved;                                     /* zero */
    int64_t x_row, out_row;                               /* strides in elements; out_row >= channels */
} fc_group_norm_desc;

/* Bytes of workspace (zero: none is needed). */
int32_t fc_linear_workspace_bytes(const fc_linear_desc *d, size_t *bytes);
int32_t fc_group_norm_workspace_bytes(const fc_group_norm_desc *d, size_t *bytes);

/* How a product is cut, for measurements and tests; what a caller has to know of it is the workspace's size alone.  A reduction in several pieces is shared by as many
 * workgroups, and joined in the pieces' order. */
enum { FC_LINEAR_RINGS = 0, FC_LINEAR_ROWS = 1, FC_LINEAR_STAGES = 2, FC_LINEAR_STAGES_ANY = 3, FC_LINEAR_TILES = 4, FC_LINEAR_LARGE = 5 };
typedef struct {
    int32_t kernel;                                       /* FC_LINEAR_... */
    int32_t tile_rows, tile_columns;                      /* of a workgroup */
    int32_t pieces;                                       /* of the reduction */
    int32_t anew_x, anew_w;                               /* 1: the operand is laid out anew in the workspace first */
} fc_linear_cut;
int32_t fc_linear_cut_of(const fc_linear_desc *d, fc_linear_cut *cut);

/* x [rows][k], w [n][k], bias [n] float32 or NULL, residual [rows][n] or NULL, count one int32 or NULL, out [rows][n]. */
int32_t fc_linear(const fc_linear_desc *d, const void *x, const void *w, const float *bias, const void *residual, const int32_t *count,
                  void *out, void *workspace, size_t workspace_bytes, void *stream);

/* x [rows][channels], weight and bias [channels] float32 or NULL, mask [rows] or NULL, starts [images + 1] or NULL, out [rows][channels]. */
int32_t fc_group_norm(const fc_group_norm_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *mask,
                      const int32_t *starts, void *out, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FOCUSED_LAYERS_H */
