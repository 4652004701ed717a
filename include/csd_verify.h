/*
 * csd — operators of the target model's verifying pass over the drafts of all paths.
 *
 * Between csd_draft and csd_accept (csd.h) the target model sees, for every path of every problem, the
 * token that the path ends with and the draft tokens behind it.  The paths of a problem are samples of
 * one prompt, so their attention has a part that they share (the prompt's keys and values: held once,
 * read once for all paths) and a part of their own.  The operators here are what is special to that pass:
 *   csd_cache_*   keys and values of the prompts and of the paths, as 16-bit values or quantised to
 *                 8 bits as they are written, and read back;
 *   csd_attend    attention of all paths' new tokens over that cache;
 *   csd_targets   the model's token at every position, with the probability that it gave it: what
 *                 csd_accept compares with and what csd_append / csd_step take as tokens and probabilities.
 * and what stands around them in the model's own work:
 *   csd_rotate    rotary positions on queries and keys; csd_cache_write_rotated: with the write to the cache, in one launch
 *   csd_prompt_attend   attention of whole prompts to themselves, packed behind each other; csd_cache_write_packed
 *                 puts their keys and values into the cache
 *   csd_adjust    penalties for repeated tokens, biases and masks on the logits, before csd_targets.
 *
 * Conventions are those of csd.h: pointers named d_* (and csd_heads.data) are device memory of the caller, `stream` is a
 * hipStream_t as void*, calls only enqueue (except csd_cache_status), allocate nothing, can be captured in
 * a HIP graph, and return CSD_OK or a negative csd_error with nothing enqueued.  A csd_cache is not
 * thread-safe; calls on one cache are enqueued on one stream or ordered by the caller.
 */
#ifndef CSD_VERIFY_H_
#define CSD_VERIFY_H_

#include <stddef.h>
#include <stdint.h>

#include "csd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define CSD_BF16 0
#define CSD_F16 1
#define CSD_F32 2 /* csd_targets and csd_adjust only */

/* Limits of this build. */
#define CSD_MAX_VERIFY_STEP (CSD_MAX_DRAFT_LEN + 1) /* tokens a path and csd_attend call */
#define CSD_MAX_CACHE_TOKENS (1 << 24)              /* tokens of a prompt, of a path      */
#define CSD_MAX_HEADS 512
#define CSD_MAX_LAYERS 1024
#define CSD_MAX_ROW_TILES (1 << 21)   /* P * N * n_kv_heads * ceil(max_step * n_heads / n_kv_heads / 32) */
#define CSD_MAX_TARGET_ROWS (1 << 22) /* rows of a csd_targets or csd_adjust call */
#define CSD_MAX_PACKED_TOKENS (1 << 24)             /* tokens of packed sequences, and of a csd_rotate call */
#define CSD_MAX_SEQUENCES (1 << 20)
#define CSD_MAX_ROTATED_DIM 512

typedef struct csd_cache csd_cache; /* opaque, host-side, library-owned */

typedef struct {
  int32_t n_problems;  /* P > 0                                                            */
  int32_t n_paths;     /* N > 0, P * N <= 2^24                                             */
  int32_t prompt_cap;  /* tokens of a problem's prompt, which its paths share, >= 0        */
  int32_t path_cap;    /* tokens of a path's own behind the prompt, > 0                    */
  int32_t n_layers;    /* 1..CSD_MAX_LAYERS                                                */
  int32_t n_heads;     /* query heads, a multiple of n_kv_heads, up to CSD_MAX_HEADS       */
  int32_t n_kv_heads;  /* > 0; query head h reads key/value head h / (n_heads / n_kv_heads) */
  int32_t head_dim;    /* 64, 96, 128 or 256 (else CSD_ERR_UNIMPLEMENTED)                  */
  int32_t max_step;    /* most tokens a path of a csd_attend call, 1..CSD_MAX_VERIFY_STEP  */
  int32_t type;        /* CSD_BF16 or CSD_F16: queries, keys, values, outputs              */
  int32_t fp8;         /* 0: the cache holds values of `type`.  1: e4m3 codes (sign, 4 exponent
                          bits, 3 of mantissa, largest 448) and a scale for each token and kv
                          head, keys and values apart: with a the largest finite |x| of the
                          head_dim values, s = the least power of two with a <= 448 s, but at
                          least 2^-126 (1 where a = 0; half precision: 2^-32 where all values are
                          zero); code = x / s rounded to nearest even.
                          Infinities become +-448 s, NaN stays NaN.  A power of two loses
                          nothing in a floating format, and x / s and code * s are exact.
                          (Half precision: |x| of 63488 and more are held as 65536, an infinity
                          beside a > 57344 as 114688.  csd_attend works with these numbers;
                          csd_cache_read rounds them to half, to infinity.)                 */
} csd_cache_config;

/* Rows of tokens of heads: element d of head h of token t of row r is data[r * row_stride + t * token_stride + h * head_stride + d],
 * strides in elements; a row is a path, row p * N + i, or a problem's prompt.  data must be 16-byte aligned and the
 * strides multiples of 8 that are not negative (CSD_ERR_INVALID_ARG).  Views of a larger array, as a projection's output for queries,
 * keys and values together, are meant by this. */
typedef struct {
  const void* data;
  int64_t row_stride;
  int64_t token_stride;
  int64_t head_stride;
} csd_heads;

/* Size in bytes of the device workspace of a cache: the keys and values (the order in which they lie there is the
 * library's own), and scratch memory of csd_attend. */
int csd_cache_bytes(const csd_cache_config* cfg, size_t* out_bytes);

/* Makes a cache inside d_workspace (256-byte aligned, at least csd_cache_bytes), which must stay allocated and untouched until
 * csd_cache_destroy.  What is held for a token is unspecified until it is written; csd_attend never lets such
 * contents, whatever they are, into its results. */
int csd_cache_create(const csd_cache_config* cfg, void* d_workspace, size_t workspace_bytes, void* stream, csd_cache** out_cache);
int csd_cache_destroy(csd_cache* cache);

/* Writes keys and values of up to n tokens of every path (_prompt: of every problem's prompt) into `layer`.
 *   k, v      n tokens of each row, n_kv_heads heads each
 *   d_start   [P][N] ([P]) int32  position of a row's first token; NULL = 0
 *   d_counts  [P][N] ([P]) int32  how many of the n tokens row r really takes (clamped to [0, n]); NULL = n
 * Token t goes to position start + t, whatever was there: a loop that rejected drafts writes over them.  Tokens whose position
 * is outside of [0, capacity) are dropped and raise CSD_STATUS_CAPACITY (csd_cache_status). */
int csd_cache_write(csd_cache* cache, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* d_start,
                    const int32_t* d_counts, int32_t n, void* stream);
int csd_cache_write_prompt(csd_cache* cache, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* d_start,
                           const int32_t* d_counts, int32_t n, void* stream);

/* Reads them back, as values of the cache's type: d_k, d_v dense [P][N][n][n_kv_heads][head_dim] ([P][n]...), 16-byte aligned.
 * Rows as in csd_cache_write; zero for tokens beyond a row's count and for positions outside of the cache. */
int csd_cache_read(csd_cache* cache, int32_t layer, const int32_t* d_start, const int32_t* d_counts, int32_t n, void* d_k, void* d_v,
                   void* stream);
int csd_cache_read_prompt(csd_cache* cache, int32_t layer, const int32_t* d_start, const int32_t* d_counts, int32_t n, void* d_k,
                          void* d_v, void* stream);

/* Attention of every path's newest tokens.
 *   q             n tokens of each path, n_heads heads each
 *   d_prompt_len  [P]    int32  tokens of each prompt (clamped to [0, prompt_cap]); NULL = prompt_cap
 *   d_path_len    [P][N] int32  tokens of each path, the new ones among them (clamped to [0, path_cap])
 *   d_counts      [P][N] int32  how many of the n tokens are a path's (clamped to [0, n]); NULL = n
 * Token t of path (p, i) sees the prompt's first prompt_len[p] tokens and the path's first path_len - count + t + 1:
 *   d_out [P][N][n][n_heads][head_dim] = sum_x softmax_x(scale * q.k_x) v_x          dense, 16-byte aligned
 *   d_lse [P][N][n][n_heads] float     = ln sum_x exp(scale * q.k_x)                 may be NULL
 * A token that sees nothing gets zeros (lse -inf), and so do tokens beyond a path's count.  Nothing outside of what a token
 * sees, not even an infinity or a NaN, changes its result.
 * prompt_bound, path_bound: what no length exceeds as far as the caller knows, 0 = the capacities.  They size the
 * launch (how far a long axis is split); results are right for longer ones too.  n in [1, max_step]. */
int csd_attend(csd_cache* cache, int32_t layer, const csd_heads* q, const int32_t* d_prompt_len, const int32_t* d_path_len,
               const int32_t* d_counts, int32_t n, float scale, int32_t prompt_bound, int32_t path_bound, void* d_out, float* d_lse,
               void* stream);

/* The form of the launch that csd_attend makes of a call with these sizes (nothing is enqueued; prompt_bound, path_bound as there). */
typedef struct {
  int32_t joined;        /* 0: each path with its whole prompt.  1: parts of the prompts, of a problem's paths together, and of the
                            paths, which a second launch joins */
  int32_t solo;          /* a path's rows are a wave's, up to 32 of them, instead of a workgroup's, up to 128 */
  int32_t prompt_splits; /* parts of a prompt's tokens (0: not joined, or no prompt) */
  int32_t path_splits;   /* parts of a path's tokens */
  int32_t groups;        /* workgroups */
} csd_attend_form;
int csd_attend_form_of(const csd_cache_config* cfg, int32_t n, int32_t prompt_bound, int32_t path_bound, csd_attend_form* out_form);

/* The token that the model picks in each row of logits, and the probability that it gives it.
 *   d_logits [rows][vocab] of `type` (CSD_BF16, CSD_F16, CSD_F32), rows logit_stride elements apart
 *   d_noise  [rows][vocab] float, rows noise_stride elements apart; NULL = greedy
 *   token = the lowest index of the largest logit; with noise, of the largest logit * inv_temperature + noise
 *           (product and sum rounded to float one after the other): a sample of the softmax where the noise is
 *           -ln(-ln u), u uniform
 *   prob  = softmax(logits * inv_temperature)[token]: csd_append's probability (Eq. 5)
 * inv_temperature > 0 and finite.  Logits of -inf are never picked, NaN counts as -inf (as does a sum that is NaN); a row
 * with nothing to pick gets -1 and 0.  Where the largest is +inf, the +inf ones share the probability.
 *   d_tokens [rows] int32, d_probs [rows] float
 *   d_scratch: csd_targets_bytes of device memory, 16-byte aligned; may be NULL where that is 0. */
int csd_targets_bytes(int64_t rows, int32_t vocab, size_t* out_bytes);
int csd_targets(const void* d_logits, int32_t type, int64_t rows, int32_t vocab, int64_t logit_stride, const float* d_noise,
                int64_t noise_stride, float inv_temperature, int32_t* d_tokens, float* d_probs, void* d_scratch, size_t scratch_bytes,
                void* stream);

/* Rotary positions.  Pair i (of dim / 2) of a head at position t is turned by the angle 2 pi t turns[i]:
 *   (a, b) -> amplitude * (a cos - b sin, a sin + b cos), to 3 * 2^-35 of its terms, then rounded to 32 bits and to the type.
 * Positions are whole numbers of any sign. */
typedef struct {
  const double* d_turns; /* [dim / 2], device memory, 8-byte aligned: turns per token (csd_rotary_turns makes the usual ones)  */
  int32_t dim;           /* the first dim values of a head are rotated, the others copied: a multiple of 16, up to the head's   */
  int32_t interleaved;   /* 0: pair i is (i, i + dim / 2), 1: (2 i, 2 i + 1)                                                   */
  float amplitude;       /* finite; 1 as a rule                                                                               */
} csd_rotary;

/* The turns of a rotation, on the host: f_i = base^(-2i/dim) / (2 pi), and for contexts longer than those of the training f_i / factor;
 * with original > 0, the training's length, r = original * f_i turns over it, keep = (r - low) / (high - low) within [0, 1]:
 * f_i * (keep + (1 - keep) / factor), which leaves the fast pairs alone.  base > 1, factor > 0, original >= 0, high > low. */
int csd_rotary_turns(int32_t dim, double base, double factor, double original, double low, double high, double* out_turns);

/* Rotates `tokens` tokens of `heads` heads of `head_dim` values (a multiple of 8, up to CSD_MAX_ROTATED_DIM).
 *   x, out       element d of head h of token t is data[t * token_stride + h * head_stride + d] (row_stride is not used); 16-byte aligned, strides
 *                multiples of 8.  out may be x itself, with the same strides; else they must not overlap,
 *                nor out's heads each other.
 *   d_positions  [tokens] int32
 *   type         CSD_BF16 or CSD_F16 */
int csd_rotate(const csd_rotary* rotary, const csd_heads* x, const int32_t* d_positions, int64_t tokens, int32_t heads, int32_t head_dim,
               int32_t type, const csd_heads* out, void* stream);

/* csd_rotate of queries and keys and csd_cache_write of the rotated keys (rounded to the cache's type, as csd_rotate does) and the values, in one launch.
 *   q, k, v      n tokens of each path, n_heads, n_kv_heads and n_kv_heads heads
 *   d_positions  [P][N][n] int32
 *   d_q_out      [P][N][n][n_heads][head_dim] dense, 16-byte aligned: all n tokens' rotated queries, whatever the counts; must not overlap q, k, v */
int csd_cache_write_rotated(csd_cache* cache, int32_t layer, const csd_rotary* rotary, const csd_heads* q, const csd_heads* k, const csd_heads* v,
                            const int32_t* d_positions, const int32_t* d_start, const int32_t* d_counts, int32_t n, void* d_q_out, void* stream);

/* Sequences packed behind each other: sequence s has the tokens d_offsets[s] .. d_offsets[s + 1] - 1 of `tokens`; d_offsets ascends
 * (an empty sequence is fine).  Offsets are clamped to [0, tokens]; where they descend, results are unspecified, but nothing outside
 * of the tensors is touched.
 *
 * csd_cache_write_packed writes sequence p to the prompt of problem p, from position 0 on (P + 1 offsets): tokens beyond prompt_cap are dropped and
 * raise CSD_STATUS_CAPACITY.  k, v: tokens of n_kv_heads heads (row_stride is not used). */
int csd_cache_write_packed(csd_cache* cache, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* d_offsets, int64_t tokens,
                           void* stream);

/* Attention of each sequence to itself: token t sees tokens 0 .. t of its sequence.
 *   q, k, v  tokens of n_heads, n_kv_heads, n_kv_heads heads (row_stride is not used); n_heads is a multiple of n_kv_heads, up to CSD_MAX_HEADS
 *   d_out    [tokens][n_heads][head_dim] dense, 16-byte aligned = sum_x softmax_x(scale * q.k_x) v_x, must not overlap q, k, v
 *   d_lse    [tokens][n_heads] float = ln sum_x exp(scale * q.k_x), may be NULL
 * The same call gives the same bits; how a token's sums are ordered may depend on what else is packed.
 * Tokens of no sequence are not written.  Nothing that a token does not see, not even an infinity or a NaN, changes its result; where
 * all that it sees weighs nothing (every score -inf), it gets zeros and -inf.
 * head_dim 64, 96, 128 or 256 (else CSD_ERR_UNIMPLEMENTED), type CSD_BF16 or CSD_F16; scale finite, times log2 e too; token strides of k and v
 * up to 2^24 elements;
 * (tokens * n_heads / n_kv_heads / 128 + sequences) * n_kv_heads up to 2^23. */
int csd_prompt_attend(const csd_heads* q, const csd_heads* k, const csd_heads* v, int32_t type, int32_t n_heads, int32_t n_kv_heads,
                      int32_t head_dim, const int32_t* d_offsets, int32_t sequences, int64_t tokens, float scale, void* d_out, float* d_lse,
                      void* stream);

/* Logits of n positions of every path (n up to CSD_MAX_VERIFY_STEP) as they are sampled from.  Position t of path (p, i) has said the path's first
 * path_len - count + t + 1 tokens (as in csd_attend: the n newest are the pass's own), and the prompt's.  For a token that was said c
 * times by the path, in 32 bits, rounded once to the type:
 *   x  = the logit
 *   x  = x > 0 ? x / repetition : x * repetition   if c > 0 or the prompt has the token
 *   x  = x - (frequency * c + presence)            if c > 0
 *   x  = x + bias
 *   x  = -inf                                      if the mask's bit is 0
 * so a masked logit is -inf whatever it was.  A row of a position beyond its path's count becomes zeros. */
typedef struct {
  int32_t n_problems, n_paths, n, vocab; /* P, N, n, V                                                                          */
  int32_t type;                          /* CSD_BF16, CSD_F16 or CSD_F32                                                       */
  const void* d_logits;                  /* [P][N][n][V], rows logit_stride elements apart                                     */
  int64_t logit_stride;
  void* d_out;                           /* the same, rows out_stride apart; may be d_logits with the same stride              */
  int64_t out_stride;
  const int32_t* d_counts;               /* [P][N] how many of the n positions are a path's (clamped to [0, n]); NULL = n        */
  const float* d_penalties;              /* [P][3] repetition (> 0), presence, frequency; NULL: none, and no tokens are read     */
  const int32_t* d_tokens;               /* [P][N] rows of up to path_cap tokens, token_stride apart; NULL: none                */
  int64_t token_stride;
  int32_t path_cap;
  const int32_t* d_path_len;             /* [P][N] the new ones among them (clamped to [0, path_cap]); NULL only without tokens  */
  const int32_t* d_prompt;               /* [P] rows of up to prompt_cap tokens, prompt_stride apart; NULL: none               */
  int64_t prompt_stride;
  int32_t prompt_cap;
  const int32_t* d_prompt_len;           /* [P] (clamped to [0, prompt_cap]); NULL = prompt_cap                                  */
  const float* d_bias;                   /* [P][V], rows bias_stride apart (0: one for all); NULL: none                        */
  int64_t bias_stride;
  const uint32_t* d_mask;                /* [P][N][n] rows of (V + 31) / 32 words, mask_stride words apart (0: one for all); bit v % 32 of
                                            word v / 32 is 1 where token v may be picked; NULL: every token may be            */
  int64_t mask_stride;
} csd_adjustment;                        /* Tokens outside of [0, V) count for nothing.  Logits and out aligned to their elements, the rest to
                                            4 bytes; strides not negative, and rows of out must not overlap                   */
int csd_adjust(const csd_adjustment* adjustment, void* stream);

/* Waits for `stream` and copies the sticky CSD_STATUS_CAPACITY bit to *host_flags. */
int csd_cache_status(csd_cache* cache, uint32_t* host_flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CSD_VERIFY_H_ */
