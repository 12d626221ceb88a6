/*
 * alpaserve_ops.h -- C-ABI of the operators of a served model's step, part of
 * libalpaserve_sim.so (AMD MI355X, gfx950).
 *
 * The placement searches of alpaserve_sim.h plan with what a model costs on a
 * device (Sec. 4.1, Table 1): the bytes that it holds there and the time of its
 * stages.  For a model that generates, the operators here set both:
 *   as_linear_i8       a linear layer with weights of 8 bits
 *   as_cache_append    a step's new keys and values into a cache of 4 bits
 *   as_attention_kv4   attention over that cache, with the attention weight
 *                      that every cached token got where asked for
 *   as_cache_evict     the cache cut to a budget by accumulated weight
 * They serve; none of them has a gradient.
 *
 * Conventions: those of alpaserve_sim.h (device pointers unless marked HOST,
 * caller-owned buffers, asynchronous on `stream`, AS_OK or an AS_E_* code with
 * as_last_error(), no exception crosses).  Nothing is allocated: a call that
 * needs scratch memory takes it from `workspace`, whose size the matching
 * *_workspace function gives (0: may be NULL); it must be aligned to 256 bytes,
 * holds nothing between calls, and may be shared by calls ordered on one
 * stream.  Invalid device data (a page outside the pool, a length beyond the
 * page table) give unspecified results but never an access outside the buffers
 * described here: tokens beyond the page table or on such a page do not exist.
 */
#ifndef ALPASERVE_OPS_H
#define ALPASERVE_OPS_H

#include <stdint.h>

#include "alpaserve_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AS_BF16 0
#define AS_F16 1
#define AS_F32 2

#define AS_I8_MAX_INPUTS 131072 /* K: sums of K products of 8 bits fit 32 */

/* ---------------------------------------------------------------- 8 bits --
 * Codes of rows x[r][0..K):  a_r = max_k |x_rk|, code = rint(127 x_rk / a_r)
 * (ties to even; 0 if a_r = 0), value = code * scale_r, scale_r = a_r / 127.  A
 * row that holds an infinity or NaN gets codes 0 and the scale NaN.
 * Storage ("tiles"): 16 rows x 64 columns each, [ceil(R/16)][Kp/64][4][16][16]
 * bytes with Kp = K rounded up to 128, byte [R/16][k/64][(k/16)%4][r%16][k%16];
 * columns K..Kp-1 hold 0, rows beyond R anything.
 */

/*
 * Bytes of the codes of n_rows rows of n_cols columns (0 for sizes out of range:
 * at most 2^24 - 1 rows and AS_I8_MAX_INPUTS columns).
 */
int64_t as_i8_bytes(int64_t n_rows, int64_t n_cols);

/*
 * Quantise rows (a linear layer's weights [outputs][inputs], once).
 *   x        [n_rows][n_cols] of `type` (AS_BF16, AS_F16, AS_F32), rows
 *            row_stride elements apart; with AS_F32 the product 127 x is
 *            rounded once before the division
 *   codes    [as_i8_bytes(n_rows, n_cols)], aligned to 16 bytes
 *   scale    [n_rows] fp32
 */
int as_quantize_i8(const void* x, int32_t type, int64_t n_rows, int64_t n_cols, int64_t row_stride,
                   void* codes, float* scale, void* stream);

/*
 * y[t][n] = (sum_k c_tk w_nk) * s_t * u_n + b_n with the activations quantised
 * per token (c, s as above, computed in the call), weights w, u as
 * as_quantize_i8 stores them.  The sum is exact; the three fp32 operations are
 * rounded in this order, then y to its type.
 *   x         [n_tokens][n_in] of x_type (AS_BF16 or AS_F16), rows x_stride apart
 *   w         codes of n_out rows of n_in columns, aligned to 16 bytes
 *   w_scale   [n_out] fp32
 *   bias      [n_out] fp32, or NULL
 *   y         [n_tokens][n_out] of y_type (any of the three), rows y_stride apart
 * At most 1,048,560 tokens, 2^24 - 1 outputs and AS_I8_MAX_INPUTS inputs.
 */
int64_t as_linear_i8_workspace(int64_t n_tokens, int64_t n_in, int64_t n_out);
int as_linear_i8(const void* x, int32_t x_type, int64_t n_tokens, int64_t n_in, int64_t x_stride,
                 const void* w, const float* w_scale, const float* bias, int64_t n_out, void* y,
                 int32_t y_type, int64_t y_stride, void* workspace, int64_t workspace_bytes,
                 void* stream);

/* ---------------------------------------------------------------- cache --
 * Keys and values of 4 bits in pages shared by all sequences of a batch.  Slot
 * s of sequence b lies on page page_table[b][s / page] at place s % page, for
 * every key/value head.  A group of `group` channels of one token has
 *   m = fp16(min), d = fp16((max - min) / 15), code = rint((x - m) / d) in
 *   [0, 15] (0 if d = 0; differences and quotients in fp32), value = code * d + m,
 * x clamped to +-65504 first; a NaN makes its group NaN.
 * Word layout: element e of a 32-bit word is at bits 4 * (e/2 + 4 * (e%2)).
 *   k      [n_pages][n_heads][page][4][dim/32] words: word [g][i] holds
 *          channels 32 i + 8 g + e
 *   v      [n_pages][n_heads][page/32][4][16][dim/16] words: word [g][c][i] of
 *          a block of 32 slots holds channel 16 i + c of slots
 *          16 (e/4) + 4 g + e%4
 *   k_par, v_par  [n_pages][n_heads][dim/group][page][2] fp16: d, m
 *   pos    [n_pages][n_heads][page] position of the slot's token in its sequence
 *   acc    [n_pages][n_heads][page] fp32 accumulated attention weight
 * The slots of a sequence are 0..length-1 for every head, in the order of their
 * tokens; heads may hold different tokens once a cache was evicted from.
 * Sequences with a common beginning may name the same pages for it where a call
 * only reads them: attention without acc_out, eviction's src.  What a call
 * writes must be named once in the table: the pages that as_cache_append puts
 * tokens on, those that hold slots below a length where attention gets acc_out
 * (a slot has one accumulated weight, of one sequence), eviction's dst.  Of a
 * slot that two sequences write, the contents are unspecified.
 */
typedef struct {
  int32_t n_pages;   /* P, pages of the pool                                     */
  int32_t n_heads;   /* key/value heads                                          */
  int32_t dim;       /* channels of a head: 64 or 128                            */
  int32_t group;     /* channels that share a scale: 32, 64 or 128, <= dim       */
  int32_t page;      /* slots of a page, a multiple of 32, <= 4096               */
  int32_t n_seqs;    /* B, rows of the page table                                */
  int32_t max_pages; /* entries of a row                                         */
  int32_t reserved;  /* 0                                                        */
  uint32_t* k;       /* aligned to 16 bytes, as are v, k_par and v_par           */
  uint32_t* v;
  void* k_par;
  void* v_par;
  int32_t* pos;      /* may be NULL where a call does not use it                 */
  float* acc;        /* likewise                                                 */
  const int32_t* page_table; /* [n_seqs][max_pages]                              */
} as_cache_t;

/*
 * Put n_tokens new tokens of every sequence into slots start[b]..: keys and
 * values quantised, positions set, accumulated weights set to 0.
 *   k, v        [n_seqs][n_tokens][n_heads][dim] of `type` (AS_BF16 or AS_F16),
 *               last two dimensions contiguous; *_seq and *_token strides in
 *               elements
 *   start       [n_seqs] first slot
 *   first_pos   [n_seqs] position of the first token, or NULL: start
 *   held_k, held_v  [n_seqs][n_tokens][n_heads][dim] fp32: the values that the
 *               cache holds now, or NULL
 * cache->pos and cache->acc may be NULL (not kept).
 */
int as_cache_append(const as_cache_t* cache, const void* k, const void* v, int32_t type,
                    int32_t n_tokens, int64_t k_seq, int64_t k_token, int64_t v_seq, int64_t v_token,
                    const int32_t* start, const int32_t* first_pos, float* held_k, float* held_v,
                    void* stream);

/*
 * Attention of n_queries new tokens of every sequence over its cache, which
 * holds them already as its last slots: query i sees the slots below
 * length - n_queries + i + 1.  Head j reads key/value head j / (heads / n_heads).
 *   o_i = sum_s p_is v_s,  p_is = exp(scale q_i.k_s) / sum_s' exp(scale q_i.k_s')
 * A query that sees nothing gets 0.
 *   q        [n_seqs][n_queries][n_q_heads][dim] of `type` (AS_BF16 or AS_F16),
 *            last two dimensions contiguous, q_seq and q_token strides in
 *            elements (multiples of 8), aligned to 16 bytes
 *   length   [n_seqs]
 *   scale    > 0, at most 2e38.  Logits (scale q.k) may reach 2^30 in magnitude;
 *            beyond that, where fp32 numbers lie 64 and more apart, a query's
 *            output and the weights that it gives are unspecified
 *   out      [n_seqs][n_queries][n_q_heads][dim] of `type`, contiguous, aligned
 *            to 8 bytes
 *   acc_in, acc_out  laid out as cache->acc: for every slot s below the
 *            length, acc_out = acc_in + sum of p_is over the queries and heads
 *            that read the key/value head (acc_in NULL: 0; the two may be the
 *            same array); other slots are not written.  No two sequences may
 *            share the pages of these slots.  acc_out NULL: no weights
 * At most 2^26 query rows, 65,535 sequences times heads, and 2^31 blocks of 32
 * slots over all sequences, heads and 16 rows (AS_E_LIMITS).
 * Products of codes and 16-bit numbers with fp32 sums; softmax in fp32; p times
 * a value's scale enters its product as two bf16 numbers (17 bits), and what
 * they leave of it is multiplied by code - 7.5.
 */
int64_t as_attention_kv4_workspace(const as_cache_t* cache, int32_t n_queries, int32_t n_q_heads,
                                   int32_t weights);
int as_attention_kv4(const as_cache_t* cache, const void* q, int32_t type, int32_t n_queries,
                     int32_t n_q_heads, int64_t q_seq, int64_t q_token, const int32_t* length,
                     float scale, void* out, const float* acc_in, float* acc_out, void* workspace,
                     int64_t workspace_bytes, void* stream);

/*
 * Copy what a budget keeps of every sequence and head to another cache: all
 * tokens where there are at most `keep`; otherwise those at the `recent` newest
 * positions (pos >= total[b] - recent) and, of the others, those of the largest
 * accumulated weight until there are `keep` (ties: the lowest slot; a NaN weight
 * comes last).  They go to slots 0.. of dst in their order, with codes, scales,
 * position and weight; codes behind the last one in its block of 32 slots of
 * dst->v become 0.  Out of place because sequences with a common beginning may
 * share src's pages; src and dst must not share a page that dst's table names.
 *   length       [n_seqs] tokens in src
 *   total        [n_seqs] tokens that the sequence has had (next position)
 *   keep, recent 1 <= keep <= dst's max_pages * page, at most 2^29 - 32;
 *                0 <= recent <= keep
 *   out_length   [n_seqs] tokens in dst: min(length, keep); an array of its own,
 *                length and total are read while it is written
 * src and dst agree in n_heads, dim, group and n_seqs; pos and acc are needed.
 */
int64_t as_cache_evict_workspace(const as_cache_t* src, int32_t keep);
int as_cache_evict(const as_cache_t* src, const as_cache_t* dst, const int32_t* length,
                   const int32_t* total, int32_t keep, int32_t recent, int32_t* out_length,
                   void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ALPASERVE_OPS_H */
