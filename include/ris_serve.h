/*
 * ris_serve.h -- serving operators around the RIS hot path (C ABI, same
 * library and conventions as ris.h): prompts of different lengths packed into
 * one batch, a key/value cache held in 4 bits with the Hybrid-Anchor decode
 * step over it, and log probabilities of given tokens.
 *
 * As in ris.h every call is asynchronous on the given HIP stream, arguments
 * are validated on the host before anything is launched, the caller owns every
 * buffer, nothing is allocated or kept between calls, and no exception crosses
 * the ABI.  Every call may be captured into a HIP graph (kernel launches only).
 *
 * Packed sequences: cu_seqlens is a device int64[batch + 1] of ascending token
 * offsets; sequence b owns the tokens [cu_seqlens[b], cu_seqlens[b + 1]) and
 * may be empty.  Tokens below cu_seqlens[0] or from cu_seqlens[batch] on belong
 * to no sequence: they are not read, and what lies in their place in an output
 * stays as it was.  Offsets outside [0, T] are clipped, so a call stays inside
 * its buffers whatever cu_seqlens holds.
 *
 * Strides are in elements.  Rows of D elements are contiguous.
 */
#ifndef RIS_SERVE_H
#define RIS_SERVE_H

#include "ris.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------ */
/* RoPE on packed sequences                                                 */
/* ------------------------------------------------------------------------ */

/*
 * The rotation of ris_rope_from with positions that restart in every sequence:
 * token i of sequence b has position start[b] + i (start NULL: i).  src is
 * strided like ris_rope_from's, x is device [heads, T, D] contiguous of the
 * same dtype and must not overlap src unless it is src itself with head_stride =
 * T * D and token_stride = D.  One call rotates the query and key heads of a
 * projection output together (heads = Hq + Hkv), for whole prompts or, with
 * one token a sequence and start = their positions, for a decode step.  start
 * is device int64[batch]; positions must be in [0, 2^52].  The lengths are on
 * the device, so the factor must be given (> 0) for linear and YaRN.  The
 * rotated bits are those of ris_rope_from at the same positions.
 */
int ris_rope_packed(const void* src, int64_t head_stride, int64_t token_stride, void* x, int32_t dtype,
                    int32_t heads, int64_t T, int32_t D, const int64_t* cu_seqlens, const int64_t* start,
                    int32_t batch, const ris_rope_desc* desc, void* stream);

/* ------------------------------------------------------------------------ */
/* Attention over packed prompts                                            */
/* ------------------------------------------------------------------------ */

typedef struct {
    int32_t dtype_in;        /* ris_dtype of Q, K, V                            */
    int32_t dtype_out;       /* ris_dtype of out                                */
    int32_t Hq;              /* query heads                                     */
    int32_t Hkv;             /* KV heads; Hq % Hkv == 0                          */
    int32_t D;               /* head dimension: 64 or 128                       */
    int32_t batch;           /* sequences (>= 1)                                */
    int64_t T;               /* token rows of Q, K, V and out                   */
    int32_t causal;          /* 1 = token i attends to the tokens up to itself; */
                             /* 0 = to its whole sequence                       */
    float   scale;           /* score scale, up to 2^127; 0 = 1 / sqrt(D)       */
    int64_t q_head, q_token; /* element (h, t, d) of Q is at                    */
    int64_t k_head, k_token; /*   h * q_head + t * q_token + d; likewise K, V   */
    int64_t v_head, v_token; /*   and out.  Strides >= 0; every one of them and */
    int64_t o_head, o_token; /*   every base a multiple of 16 bytes; of out > 0 */
                             /*   where there is more than one row; K and V     */
                             /*   tokens less than 2^24 - 1024 apart            */
} ris_prompt_desc;

/*
 * The full-density baseline of ris_sparse_attn for a batch of prompts:
 *   out[h, t, :] = sum_j softmax_j(scale <Q[h, t], K[g, j]>) V[g, j],
 * g = floor(h / (Hq / Hkv)), j over the tokens of t's sequence up to t (or all
 * of them, causal = 0).  What lies in keys and values that a token does not
 * attend to, infinities and NaN included, does not reach its output; an infinity
 * of V that it attends to does, whatever its weight (with one of the other sign
 * or a NaN: NaN).  A token whose scores are -inf alone gets NaN.  float32
 * accumulation; with bf16 inputs the softmax weights enter the PV product
 * rounded to bf16, those below 2^-126 as 0.  out must not overlap the inputs, and
 * its rows must not overlap each other.
 */
int ris_prompt_attn(const void* Q, const void* K, const void* V, const int64_t* cu_seqlens, void* out,
                    const ris_prompt_desc* desc, void* stream);

/* ------------------------------------------------------------------------ */
/* Key/value cache held in 4 bits                                           */
/* ------------------------------------------------------------------------ */

/*
 * Keys and values as 4-bit floats (E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives) in blocks of 32 consecutive dimensions that share a power of two
 * (E8M0), the OCP MXFP4 element and scale types: 4.25 bits a value.
 *
 *   K4, V4: uint8 [batch, Hkv, max_len, D / 2]; byte i of a row holds dimension
 *           2 i in its low half and 2 i + 1 in its high half.
 *   S:      uint8 [batch, Hkv, max_len, 2, D / 32]; scale bytes of the row's
 *           keys, then of its values: 2^(byte - 127), 255 = NaN.
 *
 * K4 and V4 must be 16-byte aligned, S 8-byte aligned.
 */
typedef struct {
    int32_t dtype;           /* ris_dtype of the K and V rows                   */
    int32_t Hkv;             /* KV heads                                        */
    int32_t D;               /* head dimension: 64 or 128                       */
    int32_t batch;           /* sequences, of cu_seqlens and of the cache       */
    int64_t T;               /* token rows of K and V                           */
    int64_t max_len;         /* cache rows per (sequence, kv head), <= 2^31     */
    int64_t k_head, k_token; /* strides of K and V as in ris_prompt_desc;       */
    int64_t v_head, v_token; /*   multiples of 16 bytes, as are the bases       */
} ris_kv4_desc;

/*
 * Quantise packed rows into the cache: token i of sequence b goes to position
 * start[b] + i of cache sequence b (start NULL: i); a token whose position is
 * outside [0, max_len) is left out, and rows of the cache that no token goes to
 * stay as they were.  A block's scale is the least 2^e with no magnitude above
 * 7 * 2^e, e in [-124, 125]; magnitudes go to the nearest code of x / 2^e,
 * halfway to the even code, above 6 to 6 (so no value is off by more than 2^e,
 * below the range's upper end).  A block holding an infinity or NaN becomes NaN.
 */
int ris_kv4_store(const void* K, const void* V, const int64_t* cu_seqlens, const int64_t* start,
                  uint8_t* K4, uint8_t* V4, uint8_t* S, const ris_kv4_desc* desc, void* stream);

/* The way back: K and V rows (strided as described) receive the values that the
 * cache holds at the tokens' positions, exactly (every value is a bf16 number).
 * Tokens outside the cache are left as they were. */
int ris_kv4_load(const uint8_t* K4, const uint8_t* V4, const uint8_t* S, const int64_t* cu_seqlens,
                 const int64_t* start, void* K, void* V, const ris_kv4_desc* desc, void* stream);

/*
 * ris_decode_attn over the 4-bit cache: the same descriptor, sets, clipping and
 * empty-row rule, with K and V read as the values they stand for.  window >=
 * max_len attends to every key up to pos[b] (the dense step).  anchor_ptr and
 * anchor_idx may be NULL when anchor_stride is 0 (no anchor).  scale goes up to
 * 2^127.  The workspace is
 * ris_kv4_decode_workspace_bytes(desc) bytes, 16-byte aligned, and may not be
 * shared by calls that overlap in time.  Q must be 16-byte aligned.
 */
int64_t ris_kv4_decode_workspace_bytes(const ris_decode_desc* desc);
int ris_kv4_decode_attn(const void* Q, const uint8_t* K4, const uint8_t* V4, const uint8_t* S, const int64_t* pos,
                        const int64_t* anchor_ptr, const int32_t* anchor_idx, void* out, void* workspace,
                        int64_t workspace_bytes, const ris_decode_desc* desc, void* stream);

/* ------------------------------------------------------------------------ */
/* Log probabilities                                                        */
/* ------------------------------------------------------------------------ */

/* Most alternatives a row can list. */
#define RIS_MAX_TOP 64

typedef struct {
    int32_t dtype;           /* ris_dtype of the logits                         */
    int32_t n_targets;       /* given tokens per row, 0..65536                  */
    int32_t top_k;           /* alternatives per row, 0..RIS_MAX_TOP            */
    int64_t rows;            /* >= 1                                            */
    int64_t vocab;           /* logits per row, 1..2^31 - 1                     */
    int64_t row_stride;      /* elements between rows, >= vocab                 */
} ris_logprob_desc;

/* Bytes of device workspace ris_logprobs needs (host only; 0 is possible, and
 * then workspace may be NULL). */
int64_t ris_logprobs_workspace_bytes(const ris_logprob_desc* desc);

/*
 * Scoring from one pass over rows of logits x (any element alignment), as in the
 * paper's discriminative comparison of answer options: with p = softmax(x),
 *   logprob[r, i] = log p[targets[r, i]]       (targets int64 [rows, n_targets])
 *   entropy[r]    = -sum p log p               (NULL: not wanted)
 *   top_ids[r, :], top_logprob[r, :]           the top_k tokens of largest logit,
 *                                              descending, ties to the lower id.
 * A negative target is padding and gets 0; one >= vocab gets NaN.  A logit of
 * -inf has probability 0 (its term of the entropy is 0) and is never listed:
 * places left over hold id -1 and -inf.  A row of -inf alone has no
 * distribution: its log probabilities are -inf, its entropy is 0.  A NaN or
 * +inf makes its row's log probabilities and entropy NaN; such logits rank
 * first among the alternatives, NaN before +inf.  float32 arithmetic (the sums
 * of a row in some 2^17 terms each at most before they meet).  The workspace may not
 * be shared by calls that overlap in time; 16-byte aligned.
 */
int ris_logprobs(const void* logits, const int64_t* targets, float* logprob, float* entropy, int64_t* top_ids,
                 float* top_logprob, void* workspace, int64_t workspace_bytes, const ris_logprob_desc* desc,
                 void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RIS_SERVE_H */
