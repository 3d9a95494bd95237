/*
 * smoothrot_attention.h -- the attention block between the library's linear layers: a paged cache of keys and values (paper:
 * asymmetric INT4 with one group per head, "Quantization" settings; or fp16) and the attention over it.
 *
 * A serving step of a layer: the fused q|k|v projection (sr_w4a4_gemm, sr_w4a4_gemm_f6, sr_w4a4_linear_decode), then
 * sr_rope_kv_append on its columns, then sr_attn_decode (one new token per sequence) or sr_attn_prefill (prompts), then the
 * out-projection's quantiser (sr_fwht_quant_act, sr_fwht_quant_act_heads) on what that returns.
 *
 * The conventions of smoothrot.h hold (device pointers, stream, statuses, no allocation, 16-byte aligned bases, row strides
 * multiples of 8 where the elements are fp16), but for shapes: head_dim is 64 or 128 (SR_ERR_ARG otherwise), any number of
 * tokens, sequences and heads up to the limits given at each call (SR_ERR_SHAPE otherwise; heads below 65536), n_heads a multiple of
 * n_kv_heads (query head h reads key/value head h / (n_heads / n_kv_heads)).  Rows of several heads lie one head after the other,
 * [tokens, heads * head_dim].
 */
#ifndef SMOOTHROT_ATTENTION_H
#define SMOOTHROT_ATTENTION_H

#include "smoothrot.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SR_KV_F16 = 0, SR_KV_I4 = 1 };

/*
 * The cache: pages of page_size tokens, each page one head after the other.  Token i of a page is "slot" page * page_size + i.
 *   K, V                SR_KV_F16: fp16 [n_pages][n_kv_heads][page_size][head_dim]
 *                       SR_KV_I4:  uint8 [n_pages][n_kv_heads][page_size][head_dim / 2], packed like sr_kv_quant_asym's Q
 *   K_params, V_params  SR_KV_I4: fp32 [n_pages][n_kv_heads][page_size][2] (d, z): value = (code - z) * d, of the size of fp16
 *                       numbers, d > 0, |z| < 2^24; d = NaN for a row of NaN, which reaches the query heads that read it, in
 *                       its own sequence.  NULL for SR_KV_F16.
 * page_size a power of two, 16 <= page_size <= 2^20 (SR_ERR_ARG otherwise), n_pages >= 1, n_pages * page_size < 2^40.
 * The struct lies in host memory and is read during the call only.  Slots that no sequence holds may contain anything.
 */
typedef struct {
    void *K, *V;
    float *K_params, *V_params;
    int64_t n_pages, page_size, n_kv_heads, head_dim;
    int type;
} sr_kv_cache;

/*
 * New tokens: rotates queries and keys by the tokens' positions and writes keys and values into the cache.
 * Per token t and head, with c = cos_sin[positions[t]][i], s = cos_sin[positions[t]][head_dim / 2 + i]:
 *     y_a = x_a c - x_b s,   y_b = x_b c + x_a s      (a, b) = (i, i + head_dim / 2);  SR_ROPE_PAIRS: (2 i, 2 i + 1)
 *     y <- y H / sqrt(head_dim)                       SR_ROPE_HADAMARD: the transform inside the head on queries and keys
 *                                                     alike, which leaves q . k what it was (paper: head-wise online Hadamard)
 * in fp32 (every operation rounded), then rounded to fp16.  Values are not turned.  A 4-bit cache receives the codes of those
 * fp16 numbers under the formula of sr_kv_quant_asym with group = head_dim, d = (hi - lo) times the fp32 number nearest 1 / 15,
 * quotients by d correctly rounded (so d may differ from sr_kv_quant_asym's by a rounding, and a code on a rounding boundary).  A row
 * (one head of one token) with a NaN or an infinity, the transform's own overflow included, gets d = NaN, and so stands for NaN.
 *   Q_f16          fp16 [T, n_heads * head_dim], row stride ldq; may be NULL with n_heads = 0
 *   K_f16, V_f16   fp16 [T, n_kv_heads * head_dim], row strides ldk, ldv (e.g. columns of one fused projection)
 *   positions      int32 [T]; positions outside [0, max_pos) are taken as the nearest inside
 *   slots          int64 [T]: where the token goes.  A negative slot, or one beyond the cache, leaves the cache alone (padding
 *                  rows of a batch).  Slots that occur twice leave that slot's contents unspecified.
 *   cos_sin        fp32 [max_pos, head_dim]: cosines, then sines, of a position's head_dim / 2 angles; NULL: no rotation
 *                  (positions may then be NULL).  max_pos < 2^31.
 *   clip           in [2^-64, 1] (paper: 0.95; SR_KV_I4 only)
 *   Q_out          fp16 [T, n_heads * head_dim], row stride ldqo: the turned queries.  May be Q_f16 (same stride).
 *   K_out          NULL, or fp16 [T, n_kv_heads * head_dim], row stride ldko: the turned keys before quantisation.  May be
 *                  K_f16 (same stride).
 * T * (n_heads + 2 * n_kv_heads) < 2^27.
 */
enum { SR_ROPE_PAIRS = 1, SR_ROPE_HADAMARD = 2 };
SR_API int sr_rope_kv_append(const void *Q_f16, int64_t ldq, const void *K_f16, int64_t ldk, const void *V_f16, int64_t ldv,
                      int64_t T, int64_t n_heads, const int32_t *positions, const int64_t *slots,
                      const float *cos_sin, int64_t max_pos, int flags, float clip, const sr_kv_cache *cache,
                      void *Q_out, int64_t ldqo, void *K_out, int64_t ldko, void *stream);

/*
 * Rows of the cache as dense fp16 (4 bits: fp16((code - z) * d), rounded once) -- what sr_attn_prefill takes for the part of
 * a prompt that is cached already.
 *   slots          int64 [T], any order, repeats allowed; zeros for a slot outside the cache
 *   K_out, V_out   out, fp16 [T, n_kv_heads * head_dim], row strides ldko, ldvo.  T * 2 * n_kv_heads < 2^27.
 */
SR_API int sr_kv_gather(const int64_t *slots, int64_t T, const sr_kv_cache *cache,
                 void *K_out, int64_t ldko, void *V_out, int64_t ldvo, void *stream);

/*
 * Attention of one new token per sequence over its pages:
 *     o = sum_t p_t v_t,  p = softmax(scale * q . k_t)  over the tokens t < seq_lens[b]
 * with the values that the cache stands for (4 bits: (code - z) * d, not rounded); scores, maxima and sums in fp32, weights (4 bits:
 * p_t d) rounded to fp16 for the product with the values and divided by the sum of the p_t before it, o rounded once.  The tokens of all sequences are dealt out in equal shares and
 * the parts of a sequence joined, unless the table is narrow or the sequences many; the same call gives the same bits.
 *   Q_f16        fp16 [n_seqs, n_heads * head_dim], row stride ldq
 *   page_table   int32 [n_seqs, max_pages], row stride ld_table: page i holds tokens i * page_size .. of the sequence.  Entries
 *                behind the length are not looked at; the tokens of an entry outside [0, n_pages) are left out.
 *   seq_lens     int32 [n_seqs], new token included; taken as 0 if negative and as max_pages * page_size if larger.
 *                A sequence without tokens gives zeros.
 *   scale        0 < scale <= 2^64
 *   O_f16        out, fp16 [n_seqs, n_heads * head_dim], row stride ldo
 *   workspace    sr_attn_decode_workspace_bytes(...) bytes on the device that is current, 256-byte aligned (may be NULL where
 *                that is 0).  Contents need no initialisation; calls that share one must not overlap (captured graphs included).
 * Lengths are not known on the host: whether there are shares (and a workspace) follows n_seqs, the heads, the cache's type and
 * max_pages * page_size, so a table that is no wider than the longest sequence needs is best.  From 1025 sequences, or 8 pairs of
 * sequence and key/value head per compute unit, on there are no shares: a very long sequence is then better passed in a call of its own.
 * max_pages * page_size <= 2^30, n_seqs < 2^20, n_seqs * n_heads < 2^24.
 *   type         of the cache: SR_KV_F16 or SR_KV_I4.  0 for arguments that sr_attn_decode refuses.
 */
SR_API size_t sr_attn_decode_workspace_bytes(int64_t n_seqs, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                      int64_t max_pages, int64_t page_size, int type);
SR_API int sr_attn_decode(const void *Q_f16, int64_t ldq, int64_t n_seqs, int64_t n_heads, const sr_kv_cache *cache,
                   const int32_t *page_table, int64_t max_pages, int64_t ld_table, const int32_t *seq_lens, float scale,
                   void *O_f16, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention of whole prompts, packed one behind the other:
 *     o_i = sum_j p_j v_j,  p = softmax(scale * q_i . k_j)  over the keys j of row i's own sequence
 * and, if causal, over j <= i + (keys of the sequence - queries of the sequence): the last query sees every key, so that a
 * chunk of a prompt is passed with the keys of the chunks before it in front.  A row that sees no key gives zeros.  Scores,
 * maxima and sums in fp32, weights rounded to fp16 and divided by the sum of the rounded ones, o rounded once.
 *   Q_f16          fp16 [T_q, n_heads * head_dim], row stride ldq
 *   K_f16, V_f16   fp16 [T_k, n_kv_heads * head_dim], row strides ldk, ldv (may be NULL with T_k = 0)
 *   cu_q, cu_k     int32 [n_seqs + 1]: sequence s holds rows cu_q[s] .. cu_q[s + 1] - 1 of Q and cu_k[s] .. of K and V (ascending;
 *                  cut to [0, T_q] and [0, T_k]).  Rows of no sequence are left as they were.
 *   scale          0 < scale <= 2^64
 *   O_f16          out, fp16 [T_q, n_heads * head_dim], row stride ldo.  May be Q_f16 (same stride).
 * T_q, T_k <= 2^31 - 2^10, row strides < 2^23, (T_q / 64 + n_seqs) * n_heads < 2^31.  A non-finite key or value reaches rows of its own
 * sequence only.
 */
SR_API int sr_attn_prefill(const void *Q_f16, int64_t ldq, const void *K_f16, int64_t ldk, const void *V_f16, int64_t ldv,
                    const int32_t *cu_q, const int32_t *cu_k, int64_t n_seqs, int64_t T_q, int64_t T_k,
                    int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, int causal, float scale,
                    void *O_f16, int64_t ldo, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SMOOTHROT_ATTENTION_H */
