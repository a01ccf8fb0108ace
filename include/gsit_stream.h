/*
 * gsit_stream.h -- a stream's past in 8 bits, for programs that run the layers of gsit.h and gsit_ops.h one step after the other: keys and values of
 * every segment in blocks of 32 positions, held in 8 bits with a scale for each block and key head, pages for the blocks from one pool, their tables
 * and a step's slots worked out on the GPU, and Interlaced-Mask attention that reads the cache where it lies.
 *
 * The conventions of gsit.h and gsit_ops.h hold.  A step brings seg_len[s] rows of segment s for every stream b of the batch, of which the first
 * valid_len[b][s] are real (all of them where valid_len is NULL): new positions of the stream, behind those that the cache holds.  A step is
 *   gsit_cache_plan             lengths, pages for what the step adds, and the slot of each of its rows
 *   gsit_cache_append           the step's keys and values
 *   gsit_im_cached_attention_fwd   the step's queries against everything the cache holds then
 * or all three by gsit_cache_step.  Every call reads lengths, tables and counts on the device, so a step can be captured into a graph and replayed while streams grow, end and
 * begin.  A step can also be taken again -- after a guess that was wrong, say -- from the lengths before it (plan's `held`), as long as it brought
 * no segment more than 32 rows, or started from nothing: the blocks it filled are filled anew.
 */
#ifndef GSIT_STREAM_H_
#define GSIT_STREAM_H_

#include "gsit_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GSIT_CACHE_BLOCK 32
#define GSIT_DEVFLAG_FULL 4u   /* gsit_last_device_status: a segment of a step found no pages, or no room in its table, and was not taken */

typedef enum { GSIT_CACHE_INT8 = 0, GSIT_CACHE_E4M3 = 1 } gsit_cache_kind;

/* Positions 32 j .. 32 j + 31 of segment s of stream b are block j.  A full block is held as  x8 * scale,  scale = max(max|x| / most, 2^-80)  over the
 * block's positions and one key head's features, keys and values apart, most = 127 (INT8) or 448 (E4M3), and x8 the representable value that is nearest
 * to x / scale (ties to even).  A block and head in which NaN or Inf stands has a scale of NaN: all of it reads as NaN.  Rows of the block that is not full
 * yet are kept as they came, in buffer j % 2 of open_keys and open_values (a row of NaN or Inf there: as above, for attention); so what the
 * cache holds does not depend on the steps it came in.
 * Bytes of a page's head: features in groups of 16, for each group [lane][m][c][h][e], lane = 4 g + t: keys of position 16 m + 8 h + g, feature
 * 16 group + 8 c + 2 t + e; values the same with position and feature exchanged, the groups of features where m stood and position halves where
 * groups stood -- [feature group][lane][position half][c][h][e], feature 16 group + 8 h + g, position 16 half + 8 c + 2 t + e.  head_dim 8: keys [lane][m][h][e]
 * with position 16 m + 8 h + g and feature 2 t + e, values [lane][half][c][e] with feature g and position 16 half + 8 c + 2 t + e. */
typedef struct gsit_cache {
  int32_t kind;                    /* gsit_cache_kind */
  int32_t dtype;                   /* GSIT_F32 or GSIT_BF16: of open rows, and of the rows that calls take and give */
  int32_t batch, kv_heads, head_dim;   /* head_dim 8, 16, 32 or 64 */
  int32_t pages;                   /* of the pool, at most 2^26 - 1 */
  int32_t blocks;                  /* entries of a segment's row in tables: it can grow to 32 * blocks positions */
  void *keys, *values;             /* DEVICE int8 or e4m3 [pages][kv_heads][32 * head_dim], 16-byte aligned */
  float *key_scale, *value_scale;  /* DEVICE float [pages][kv_heads] */
  float* times;                    /* DEVICE float [pages][32], 16-byte aligned, or NULL: the moment of each position */
  void *open_keys, *open_values;   /* DEVICE dtype [batch][3][2][kv_heads][32][head_dim], 16-byte aligned */
  int32_t* tables;                 /* DEVICE int32 [batch][3][blocks]: page of each block, -1 where there is none */
  int32_t* lengths;                /* DEVICE int32 [batch][3]: positions held */
  int32_t* free_list;              /* DEVICE int32 [pages]: free pages, the first n_free of them */
  int32_t* n_free;                 /* DEVICE int32 [1] */
} gsit_cache;

/* Pages for a step.  Of the cache batch, pages, blocks, tables, lengths, free_list and n_free are read; of the shape batch, seg_len and valid_len.
 *   held      DEVICE int32 [batch][3]: positions before the step; NULL: lengths.  lengths becomes held + valid_len.
 *   ended     DEVICE int32 [batch] or NULL: streams other than 0 begin anew with this step, from nothing; their pages go back to the list first.
 *   slots     DEVICE int32 [batch][L], written: 32 * page + place in it of every real row of the step, -1 for the others
 * Blocks that already have a page keep it.  The others take theirs from the end of the list in the order of streams, segments and positions; pages
 * that go back are put so that they would be handed out in that order again.  A segment whose rows do not fit its table is not taken
 * (its slots are -1, its length stays), and where pages run out, neither is the first one that finds too few, nor any behind it that needs some:
 * GSIT_DEVFLAG_FULL. */
gsit_status gsit_cache_plan(const gsit_shape* shape, const gsit_cache* cache, const int32_t* held, const int32_t* ended, int32_t* slots,
                            gsit_stream stream);

/* A step's keys and values, where plan's slots say: those alone tell which rows are real (valid_len is not read), lengths are those that plan left.
 *   k, v      dtype [batch][L][kv_heads][head_dim], 16-byte aligned, row strides (elements) whole multiples of 16 bytes
 *   times     DEVICE float, finite: the moment of row i of stream b at times[b * times_batch_stride + i * times_row_stride]; read where the
 *             cache holds times */
gsit_status gsit_cache_append(const gsit_shape* shape, const gsit_cache* cache, const void* k, int64_t k_row_stride, const void* v,
                              int64_t v_row_stride, const int32_t* slots, const float* times, int64_t times_batch_stride,
                              int64_t times_row_stride, gsit_stream stream);

/* The first seg_len[s] positions of every segment as rows again, +0 behind the last one held: for calls that take rows (gsit_im_scored_attention_fwd
 * on a long prompt), or to look at.  k, v as above, written. */
gsit_status gsit_cache_read(const gsit_shape* shape, const gsit_cache* cache, void* k, int64_t k_row_stride, void* v, int64_t v_row_stride,
                            gsit_stream stream);

/* gsit_im_scored_attention_fwd for a step's rows, keys and values from the cache: real row i of segment s is position lengths[b][s] - valid_len[b][s] + i,
 * and sees the open segments as they are then, up to their last position held.
 * (Rows of a segment that plan did not take are not in the cache, but are answered like the others, as the last positions that are: their slots say so.)
 *   shape        d_model, heads, phase, custom_mask and scale as there; dtype of the cache
 *   rule         softcap, causal and slopes; kv_heads of the cache, or 0.  times, documents, prefix and tail are not taken (GSIT_ERR_UNSUPPORTED).
 *   times        the moments of the step's rows, as above: given where the cache holds times and the rule goes by them (causal, slopes); NULL where it holds
 *                none (the index inside the segment counts, in tables of up to 2^19 blocks a segment: GSIT_ERR_UNSUPPORTED beyond)
 *   q            [batch][L][heads][head_dim], as above;  out [batch][L][d] contiguous;  lse float [batch][heads][L] or NULL
 *   workspace    gsit_cached_attention_workspace() bytes, 16-byte aligned (NULL and 0 where that is 0); what stands in it does not matter */
gsit_status gsit_im_cached_attention_fwd(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache, const void* q,
                                         int64_t q_row_stride, const float* times, int64_t times_batch_stride, int64_t times_row_stride,
                                         void* out, float* lse, void* workspace, size_t workspace_bytes, gsit_stream stream);
size_t gsit_cached_attention_workspace(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache);   /* (size_t)-1: invalid */

/* A step: the three calls above with one shape (that of attention) and the arguments that each of them takes.  What any of them would refuse is refused
 * before the cache is touched, where one call after the other would leave its lengths counting rows that are not there. */
gsit_status gsit_cache_step(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache, const int32_t* held, const int32_t* ended,
                            int32_t* slots, const void* q, int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride,
                            const float* times, int64_t times_batch_stride, int64_t times_row_stride, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, gsit_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* GSIT_STREAM_H_ */
