/*
 * relpos.h -- C ABI of a learned relative position bias by buckets of offsets for AMD MI355X (gfx950),
 * with its gradient.
 *
 * gswa.h's bias table has a row for every offset inside a window.  Here offsets share the learned rows: near ones
 * have a row each, far ones a row for a range of distances that widens with the distance.  A bucket is found from the
 * offset r = key position - query position:
 *   n(d)      = number of edges <= d                 (edges ascend, edges[0] >= 1, so n(0) = 0)
 *   bucket(r) = n(max(-r, 0))                        one side: keys behind the query share bucket 0
 *   bucket(r) = n(|r|) + (r > 0 ? n_edges + 1 : 0)   with RELPOS_BIDIRECTIONAL
 * so a side has n_edges + 1 buckets.  Two forms:
 *
 *   sequence (window == 0)   query i stands at position q_start + i, key j at j:
 *     out[h, i, j]  = table[bucket(j - i - q_start), h]           [heads, q_len, k_len], for all images of a batch
 *     dtable[b, h]  = sum over batch, i, j of that bucket of dout[batch, h, i, j]
 *     With RELPOS_CAUSAL keys behind the query get -infinity, and the gradients there take no part, whatever they hold.
 *     q_len = 1 is the step of a decoder: one query against k_len cached keys.
 *   window (window = M > 0)  the bias table of a GSWA layer with M x M windows from a table of buckets per axis,
 *     B = 2 (n_edges + 1) of them (RELPOS_BIDIRECTIONAL is required; the sequence fields are ignored):
 *     out[(dr + M-1)(2M-1) + dc + M-1, h] = table[bucket(-dr) B + bucket(-dc), h],  dr, dc = query - key, as gswa.h
 *     dtable[b, h] = sum of dout over the offsets of that pair of buckets; dout is gswa_backward's dbias_table (fp32)
 *
 * The conventions of gswa.h hold: `desc` is a HOST pointer, everything else a DEVICE pointer the caller owns; nothing is
 * allocated, freed or synchronised; all work is enqueued on `hip_stream`; a failed call has enqueued nothing.  Pointers
 * are 16-byte aligned, `ws` 256-byte aligned.
 */
#ifndef RELPOS_H
#define RELPOS_H

#include "gswa.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { RELPOS_MAX_EDGES = 127 };

enum {
    RELPOS_BIDIRECTIONAL = 1u << 0, /* keys behind the query have buckets of their own                     */
    RELPOS_CAUSAL = 1u << 1,        /* sequence form: keys behind the query get -infinity and no gradient  */
    RELPOS_ACCUM_WGRAD = 1u << 2    /* relpos_backward adds into dtable                                    */
};

typedef struct relpos_desc {
    int32_t heads;       /* 1 .. 65535                                                                     */
    int32_t dtype;       /* GSWA_F32 or GSWA_BF16: table, out, and the sequence form's dout                */
    uint32_t flags;
    int32_t window;      /* M > 0: window form, at most 64; 0: sequence form                               */
    int32_t batch;       /* sequence form: images that share the bias (dout has this many)                 */
    int32_t q_len, k_len;
    int32_t q_start;     /* position of the first query, >= 0                                              */
    int64_t row_stride;  /* elements from one row of out / dout to the next, >= k_len; 0 = k_len           */
    int32_t n_edges;     /* 0 .. RELPOS_MAX_EDGES                                                          */
    int32_t edges[RELPOS_MAX_EDGES];
} relpos_desc;

/*
 * Fills *n_edges and edges (room for RELPOS_MAX_EDGES) with the usual spacing: of a side's S buckets (S = buckets / 2 with
 * `bidirectional`, else buckets) the first E = S / 2 hold one distance each, the others even steps of the logarithm from
 * E to max_distance, the last one everything beyond: edge E + k is the least whole r with r >= E (max_distance / E)^(k / (S - E)).
 * Found in whole numbers: no border depends on how a logarithm rounds.  GSWA_EINVAL unless S is 2 .. 128, `buckets`
 * is even where `bidirectional`, and max_distance > E.
 */
int relpos_log_edges(int32_t buckets, int32_t max_distance, int32_t bidirectional, int32_t *n_edges, int32_t *edges);

/* Scratch of relpos_backward in bytes, a multiple of 256. relpos_forward needs none. */
int relpos_query_bytes(const relpos_desc *desc, size_t *bwd_ws_bytes);

/* table [buckets, heads] in desc->dtype, buckets as above (B * B in the window form).  out must not overlap table. */
int relpos_forward(const relpos_desc *desc, const void *table, void *out, void *hip_stream);

/* dtable [buckets, heads] fp32, overwritten (added into with RELPOS_ACCUM_WGRAD); summed in a fixed order: the same bits every
 * run.  dtable and ws must be disjoint from dout and from each other; ws may be NULL where the queried size is 0. */
int relpos_backward(const relpos_desc *desc, const void *dout, float *dtable, void *ws, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RELPOS_H */
