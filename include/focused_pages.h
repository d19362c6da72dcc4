/*
 * focused_pages.h - C ABI of the pages of the key/value cache of focused_attention.h on AMD MI355X (gfx950): which sequence holds which
 * block of the pool, kept on the device.
 *
 *   users   [blocks] int32 (device): how many sequences hold a block, zero = free.  Zeroed once for a new cache, and from then on kept by these
 *           calls; several tables may share a cache and its users.
 *   table   [batch][table_width] int32, lengths [batch] int32: as for appending and attention.  An entry outside [0, blocks) is no block, and the calls
 *           write -1 for it.  Sequence b needs the first ceil(lengths[b] / 64) entries; lengths beyond the table count as the table's.
 *
 * A block that several sequences hold is full: they can all read it and none appends to it.  fc_kv_fork and fc_kv_resize see to that; whoever
 * writes tables by hand does.
 *
 * Free blocks are given out lowest number first, to the places that want one in the order of sequences and entries.  Where the pool has too few, the last
 * places stay -1 (their tokens are written nowhere, read as zeros and attended to by nobody), and missing (device, one int32) counts
 * them; it is written by every call.  Results do not depend on the order in which the device does its work.
 *
 *   fc_kv_resize   every sequence holds what its length needs: entries behind that are given back and become -1 (a length of zero frees the
 *                  sequence), entries before it that are no block get one (nothing is written into it).  Before fc_kv_append with lengths that
 *                  have grown; after lengths were cut.  A cut that ends within a block that others hold too gives the sequence a copy
 *                  of its own of that block, in its place of the order above.  Blocks given back count as free in the same call, but for those that are copied from.
 *                  Where there are too few blocks for all that, a block that nobody holds but sequences that are cut within it stays with the lowest of them, and the
 *                  others alone want copies: what is cached there is not lost for all.
 *   fc_kv_fork     slot b becomes what slot parents[b] was before the call: the beams of a search, the samples of a prompt, a reordered batch.
 *                  parents[b] = b: it stays as it is; outside [0, batch): it is freed, its length becomes zero.  A slot that does
 *                  not stay gives its blocks back first and holds the blocks that the parent's length needs: full ones with it, an unfinished last one
 *                  with it if the parent does not stay and b is the lowest of its slots, else as a copy in a block of its own.  table and lengths
 *                  are rewritten.  (Tables that agree with users are assumed; the lowest slot takes the unfinished block over as it is.)
 *   fc_kv_compact  the blocks that are in use (users > 0) go, in order, to blocks 0, 1, .. of another cache, and table_to, users_to say where they are: a
 *                  pool that has become too large or too small moves to another.  Blocks beyond the other pool are lost: their entries are -1,
 *                  missing counts the blocks.  Entries of table that no user is counted for become -1.  (One table: a cache that
 *                  several tables share is not compacted.)
 *   fc_kv_copy     block targets[i] of one cache becomes block sources[i] of another or the same (a pair with a number out of range: nothing).
 *                  No target is a source or a target of another pair.
 *
 * Unchanged sequences cost a look at their table row only.  Bounds as for attention: contents of tables, lengths, parents and users beyond the sizes of the
 * descriptor are cut off, so wrong contents give wrong results and never an access out of range.
 *
 * Conventions are those of focused_conv.h.  Tables, lengths, users, parents, missing, lists and workspaces are aligned to 16 bytes.  No pointer may be the same as another
 * of the same call but cache_to of fc_kv_copy.  With FC_WORKSPACE_READY (4) in flags the caller vouches that the workspace's counters are
 * zero, as a workspace that was zeroed once has them, and from then on after every completed call of the same function with the same descriptor.
 */
#ifndef FOCUSED_PAGES_H
#define FOCUSED_PAGES_H

#include "focused_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t blocks, kv_heads, head_dim;     /* the cache */
    int32_t blocks_to;                      /* blocks of the other cache (fc_kv_copy, fc_kv_compact) */
    int32_t batch, table_width;             /* sequences, entries of a table row */
    int32_t pairs;                          /* fc_kv_copy */
    uint32_t flags;                         /* FC_WORKSPACE_READY */
} fc_pages_desc;

int32_t fc_kv_resize_workspace_bytes(const fc_pages_desc *d, size_t *bytes);
int32_t fc_kv_fork_workspace_bytes(const fc_pages_desc *d, size_t *bytes);
int32_t fc_kv_compact_workspace_bytes(const fc_pages_desc *d, size_t *bytes);

int32_t fc_kv_resize(const fc_pages_desc *d, void *cache, int32_t *users, int32_t *table, const int32_t *lengths, int32_t *missing,
                     void *workspace, size_t workspace_bytes, void *stream);
int32_t fc_kv_fork(const fc_pages_desc *d, void *cache, int32_t *users, int32_t *table, int32_t *lengths, const int32_t *parents,
                   int32_t *missing, void *workspace, size_t workspace_bytes, void *stream);
int32_t fc_kv_compact(const fc_pages_desc *d, const void *cache, const int32_t *users, const int32_t *table, void *cache_to, int32_t *users_to,
                      int32_t *table_to, int32_t *missing, void *workspace, size_t workspace_bytes, void *stream);
int32_t fc_kv_copy(const fc_pages_desc *d, const void *cache, const int32_t *sources, void *cache_to, const int32_t *targets, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FOCUSED_PAGES_H */
