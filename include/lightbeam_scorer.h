/*
 * lightbeam_scorer.h -- operators of a fusion scorer on MI355X (gfx950).
 *
 * With LB_FUSION_EXTERNAL the caller of lb_decode_batch answers each fusion
 * event with log-probabilities of word sequences, from a language model of its
 * own (lb_fusion_request, lb_fusion_scores).  Here are the operators that such
 * a scorer is made of, beside its plain matrix products:
 *
 *   lb_kv_append, lb_kv_read     keys and values of new tokens into a paged
 *                                cache held in 4 bits, rotated on the way
 *   lb_kv_attend                 attention over that cache: prompts, single
 *                                tokens, and both in one ragged batch
 *   lb_lora_add                  low-rank adapters of many requests beside a
 *                                shared projection
 *   lb_logits_adjust             penalties, biases and masks on logits, and
 *                                their log-probabilities; over the 41 classes
 *                                its output is lb_decode_batch's input
 *   lb_rope_table                angles for lb_kv_append
 *
 * Conventions are those of lightbeam.h: every function returns an lb_status and
 * never throws or aborts, lb_last_error() describes the last failure, device
 * memory is the caller's, and work is enqueued asynchronously on `stream` of
 * the calling thread's current device, to which all device memory of the call
 * belongs.  No function allocates device memory, copies to the host or
 * synchronises, so every call may be captured into a HIP graph; a workspace
 * belongs to one call at a time (two captured graphs that may run side by side
 * need one each) and holds nothing between calls.  Calls on different streams
 * may overlap if no memory that one of them writes is used by the other.  What a
 * call writes overlaps nothing else of the call, except where that is said.
 * Descriptors are read during the call only.
 */
#ifndef LIGHTBEAM_SCORER_H_
#define LIGHTBEAM_SCORER_H_

#include "lightbeam.h"

#ifdef __cplusplus
extern "C" {
#endif

/* types of activations, weights and outputs */
enum { LB_F32 = 0, LB_BF16 = 1, LB_F16 = 2 };

/* ---------------------------------------------------------------- the cache */

/* Keys and values in pages of page_tokens tokens.  Each block of 32 channels of
 * one head of one token holds 4-bit codes and a scale:
 *   value = code * 2^(scale - 127),  code in {0, 0.5, 1, 1.5, 2, 3, 4, 6} and
 *   their negatives (e2m1: bit 3 is the sign), scale in 3..252; scale 255 stands
 *   for NaN in the whole block.
 * The memory of head h of page p starts at
 *   pages + (p * kv_heads + h) * page_tokens * (head_dim + head_dim / 16)
 * and holds, with P = page_tokens and D = head_dim,
 *   key codes    [P][D/2]      byte c/2 of a token: channels c (low half), c + 1
 *   value codes  [P/4][D/2][4] byte of (token t, pair c/2): [t/4][c/2][t%4]
 *   key scales   [P][D/32]
 *   value scales [P/4][D/32][4]
 * (four tokens' values of a channel pair side by side are what one lane of a
 * matrix instruction takes of the values). */
typedef struct lb_kv_cache {
  void* pages;         /* device, 16-B aligned, n_pages pages                    */
  int64_t n_pages;
  int32_t page_tokens; /* 16, 32, 64, 128 or 256                                 */
  int32_t kv_heads;    /* 1..1024                                                */
  int32_t head_dim;    /* 64, 128 or 256                                         */
  int32_t reserved;
  uint32_t* flags;     /* device word that faults of the data are or-ed into
                          (LB_KV_*), or NULL                                     */
} lb_kv_cache;

enum {
  LB_KV_BAD_PAGE = 1u,   /* a page number outside 0..n_pages-1: its tokens were
                            not written, and count as masked when read          */
  LB_KV_BAD_LENGTH = 2u  /* starts or lengths that do not fit each other, the
                            tables or max_new: the tokens concerned were left out */
};

/* A ragged batch of sequences.  The new tokens of sequence s are the rows
 * starts[s] .. starts[s+1]-1 of the call's activations (none, one or many), and
 * are the last ones of its lengths[s] tokens: row starts[s] + i has position
 * lengths[s] - (starts[s+1] - starts[s]) + i.  Token t lies in slot t % P of
 * page pages[s * max_pages + t / P].  Rows at or past starts[n_seqs] are padding:
 * no call reads or writes them. */
typedef struct lb_kv_batch {
  const int32_t* starts;  /* device [n_seqs + 1], not decreasing, from 0 on     */
  const int32_t* lengths; /* device [n_seqs]: tokens with the new ones          */
  const int32_t* pages;   /* device [n_seqs][max_pages]                         */
  int32_t n_seqs;         /* at most 2^22                                       */
  int32_t n_rows;         /* rows of the activations: at least starts[n_seqs],
                             at most 2^24                                       */
  int32_t max_pages;
  int32_t max_new;        /* at least every sequence's number of new tokens     */
} lb_kv_batch;
/* (max_pages * page_tokens is at most 2^30.  A call's workgroups number less than
 * 2^24: lb_kv_attend and lb_kv_attend_workspace refuse batches that need more.  They
 * take every batch with kv_heads * (n_seqs + n_rows * (q_heads / kv_heads) / 16)
 * below that, whatever max_new is.) */

/* Rotation of keys and queries: with row p of the tables for position p, the
 * pair (x1, x2) of channels becomes (x1 cos - x2 sin, x2 cos + x1 sin); pair i
 * is (i, i + rot_dim/2) or (2i, 2i + 1); channels from rot_dim on stay. */
enum { LB_ROPE_HALF = 0, LB_ROPE_INTERLEAVED = 1 };
typedef struct lb_rope {
  const float* cos;  /* device [positions][rot_dim/2], 16-B aligned             */
  const float* sin;
  int32_t positions; /* tokens at positions past the table are left out and
                        flagged (LB_KV_BAD_LENGTH)                              */
  int32_t rot_dim;   /* a multiple of 16, at most head_dim                      */
  int32_t layout;    /* LB_ROPE_*                                               */
  int32_t reserved;
} lb_rope;

/* Fills host tables cos, sin [positions][rot_dim/2] for lb_rope, in 64 bits and
 * rounded once: angle(p, i) = p * f_i, f_i = base^(-2i/rot_dim) scaled for
 * contexts `factor` times longer than `trained` positions:
 *   LB_ROPE_PLAIN   f_i
 *   LB_ROPE_LINEAR  f_i / factor
 *   LB_ROPE_BLEND   f_i for wavelengths (2 pi / f_i) below trained/high, f_i /
 *                   factor above trained/low, between them both weighted by
 *                   w = (trained / wavelength - low) / (high - low):
 *                   w f_i + (1 - w) f_i / factor  (0 < low < high)             */
enum { LB_ROPE_PLAIN = 0, LB_ROPE_LINEAR = 1, LB_ROPE_BLEND = 2 };
lb_status lb_rope_table(int32_t positions, int32_t rot_dim, double base, int32_t scaling, double factor,
                        double trained, double low, double high, float* cos, float* sin);

/* Rotates the queries and keys of a batch's new tokens and appends the keys and
 * values to the cache.
 *   q      device [n_rows][q_heads][D], row stride q_stride elements; NULL with
 *          q_heads = 0: no queries
 *   k, v   device [n_rows][kv_heads][D], row strides k_stride, v_stride
 *   q_out  device, as q: the rotated queries; may be q itself with the same
 *          stride
 *   rope   NULL: no rotation (q_out gets q as it is)
 * A block's scale is the smallest power of two 2^e, e in -124..125, with
 * |x| <= 6 * 2^e for its 32 values, each code the nearest (ties to the even code,
 * at most 6); keys are rotated in 64 bits first, so the codes are those of the
 * exact rotation.  A block with an infinity or a NaN gets scale 255.  Rows' strides
 * are multiples of 16 B and pointers 16-B aligned.  The slots of a call's tokens
 * must be distinct: what two tokens that share one leave there is not defined. */
lb_status lb_kv_append(const lb_kv_cache* cache, const lb_kv_batch* batch, const lb_rope* rope, int32_t dtype,
                       int32_t q_heads, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, void* stream);

/* The values that the cache holds of a batch's new tokens, as
 * [n_rows][kv_heads][D] of `dtype` (k_out or v_out may be NULL): exact in
 * LB_F32 and LB_BF16, rounded to nearest in LB_F16. */
lb_status lb_kv_read(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t dtype, void* k_out,
                     int64_t k_stride, void* v_out, int64_t v_stride, void* stream);

/* Attention of a batch's new tokens over their sequences' cached tokens (their
 * own included: append first).  The query of a token at position p sees the
 * tokens t <= p, with window > 0 only those with t > p - window (pages of which no
 * query sees a token need not be there):
 *   out = sum_t softmax_t(scale * q . k_t) v_t,   lse = ln sum_t exp(scale * q . k_t)
 * Query head h reads KV head h / (q_heads / kv_heads).  A query that sees no
 * token, or has scores of -infinity alone, gets out = 0 and lse = -infinity.
 * What unseen tokens hold, NaN and infinities included, has no effect.  Scores,
 * sums and outputs are held in 32 bits and an output is rounded once; the
 * probabilities enter the products with the values to 2^-16 of themselves for
 * LB_BF16 and LB_F16, 2^-24 for LB_F32.  Scores past 2^30 in magnitude, whose
 * softmax is below their own rounding to 32 bits, have no defined result.
 *   q, out     device [n_rows][q_heads][D] of `dtype`, row strides q_stride and
 *              out_stride (multiples of 16 B)
 *   lse        device float32 [n_rows][q_heads], or NULL
 *   workspace  device, 16-B aligned, at least what lb_kv_attend_workspace says
 *              for this cache, batch and q_heads (NULL if that is 0)           */
lb_status lb_kv_attend_workspace(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t q_heads,
                                 int64_t* bytes);
lb_status lb_kv_attend(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t dtype, int32_t q_heads,
                       const void* q, int64_t q_stride, float scale, int32_t window, void* out,
                       int64_t out_stride, float* lse, void* workspace, int64_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------- adapters */

/* out[i] = y[i] + scale[a] * B[a] (A[a] x[i]),  a = adapter[i]; rows whose
 * adapter is outside 0..n_adapters-1 become y[i].  Rows of one adapter need not
 * lie together (where they do, its weights are read once for all of them).
 * Products are summed in 32 bits and the sum is rounded once; A x enters the
 * product with B as it is for LB_F32, and to 2^-16 (LB_BF16) or 2^-21 (LB_F16) of
 * its row's largest magnitude.
 *   x       device [rows][d_in], y, out device [rows][d_out], of `dtype`, with
 *           row strides; out may be y itself with the same stride, and may
 *           overlap x, where the workspace has 4 * rows * rank bytes at least
 *   a, b    device [n_adapters][rank][d_in] and [n_adapters][d_out][rank]
 *   adapter device int32 [rows];  scale: device float32 [n_adapters], NULL: 1
 *   workspace  device, 16-B aligned, at least what lb_lora_workspace says for
 *              these rows and sizes (NULL if that is 0)
 * rows at most 2^28, d_in and d_out 2^30.
 * rank, d_in, d_out are multiples of 8, rank at most 128 (adapters of lower rank
 * are padded with zeros); strides are multiples of 16 B, pointers 16-B aligned. */
lb_status lb_lora_workspace(int64_t rows, int32_t d_in, int32_t d_out, int32_t rank, int64_t* bytes);
lb_status lb_lora_add(int32_t dtype, int64_t rows, int32_t d_in, int32_t d_out, int32_t rank, int32_t n_adapters,
                      const void* x, int64_t x_stride, const void* y, int64_t y_stride, const void* a,
                      const void* b, const int32_t* adapter, const float* scale, void* out, int64_t out_stride,
                      void* workspace, int64_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------- logits */

/* What lb_logits_adjust does to the logit x of class w in row r, in this order:
 *   n = how often w occurs in the row's history; if n > 0:
 *     x = x > 0 ? x / repetition : x * repetition
 *     x = x - presence - frequency * n
 *   x = x + (bias of w, 0 if none)
 *   x = x / temperature
 *   x = -infinity if the row's mask has bit w % 32 of word w / 32 clear
 * Ids outside 0..classes-1 in a history or a bias list are no entries; of several
 * biases for one class the last counts. */
typedef struct lb_logit_rules {
  float temperature;         /* a normal number > 0; 1: none                    */
  float repetition;          /* a normal number > 0; 1: none                    */
  float presence, frequency; /* 0: none                                         */
  const int32_t* history;    /* device [rows][history_width] or NULL            */
  const int32_t* bias_ids;   /* device [rows or 1][bias_width] or NULL          */
  const float* bias_values;  /* device, as bias_ids                             */
  const uint32_t* mask;      /* device [mask_rows][(classes + 31) / 32] or NULL */
  const int32_t* mask_row;   /* device [rows]: the mask of each row, none where
                                outside 0..mask_rows-1; NULL: row r uses mask r,
                                or mask 0 with mask_rows = 1                     */
  int32_t history_width;
  int32_t bias_width;        /* history_width + bias_width <= LB_MAX_RULE_IDS    */
  int32_t bias_per_row;      /* 0: one list for all rows                        */
  int32_t mask_rows;
} lb_logit_rules;
enum { LB_MAX_RULE_IDS = 4096 };

/* Adjusted logits and their log-probabilities: with z the row after the rules
 * and lse = ln sum_w exp z_w,
 *   logprobs  device float32 [rows][classes], row stride logprobs_stride: z - lse
 *   score     device float32 [rows]: logprobs at target[r]; 0 for a negative
 *             target (padding), NaN for one >= classes
 *   lse       device float32 [rows]
 * (each may be NULL; target is read if score is not).  Masked classes get
 * -infinity whatever their logits hold, those whose z is -infinity whatever the
 * rest of the row holds (else a row with a NaN is NaN), a row with nothing left
 * -infinity throughout.  rules NULL: none.
 *   logits    device [rows][classes] of `dtype`, row stride logits_stride; rows at
 *             most 2^28, classes 2^30
 *   workspace  device, 16-B aligned, at least what lb_logits_workspace says for
 *              these rows and classes (NULL if that is 0)
 * A call made again gives the same bits.  logits is only read; logprobs may be
 * the logits themselves where these are LB_F32 with the same stride. */
lb_status lb_logits_workspace(int64_t rows, int32_t classes, int64_t* bytes);
lb_status lb_logits_adjust(int32_t dtype, int64_t rows, int32_t classes, const void* logits,
                           int64_t logits_stride, const lb_logit_rules* rules, const int32_t* target,
                           float* logprobs, int64_t logprobs_stride, float* score, float* lse, void* workspace,
                           int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LIGHTBEAM_SCORER_H_ */
