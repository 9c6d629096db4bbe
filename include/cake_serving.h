/*
 * cake_serving.h -- C ABI of the serving operators beside the clustering calls of cake_kmeans.h: what a program needs
 * that clusters the keys of an attention layer and then attends to some of them.
 *   rmsnorm_quant   residual addition, root-mean-square norm, 8-bit output with scales;
 *   gemm_fp8        product of two 8-bit matrices with scales per 128-column block (and 128 x 128 block of the weights);
 *   kv_append       rotation of queries and keys by position, keys and values written to a paged cache;
 *   qk_norm_append  the same with a norm of each query and key head ahead of the rotation;
 *   kv_read         cached keys and values read back by slots;
 *   paged_decode    attention of one new token per sequence over the paged cache;
 *   paged_chunk     attention of a chunk of new tokens per sequence over the paged cache;
 *   prompt_attention  attention of whole prompts, packed one behind the other.
 * The paper names a grouped-query decode and a block-scaled 8-bit product among its other kernels, without their source or interface;
 * these calls follow neither.
 *
 * Conventions are those of cake_kmeans.h (device pointers, caller-owned buffers, asynchronous on `stream`, CAKE_* return
 * codes, nothing allocated), and
 *   - cake_e4m3 is a raw 8-bit float: sign, 4 exponent bits, 3 mantissa bits, no infinities, largest value 448;
 *   - strides are counted in elements; the innermost dimension is always contiguous;
 *   - `ws` scratch is 256-byte aligned; its first word is the sticky device status (cake_kmeans_device_status).  The caller
 *     zeroes the first CAKE_SERVING_HEADER_BYTES bytes once, before the first call that uses the buffer; the calls leave
 *     them ready for the next call, of any size.  Calls that run concurrently must use distinct workspaces.  After a status
 *     of CAKE_ERR_TIMEOUT (a bounded wait in a kernel expired) the header is zeroed again before the next call.
 */
#ifndef CAKE_SERVING_H_
#define CAKE_SERVING_H_

#include "cake_kmeans.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef unsigned char cake_e4m3;

#define CAKE_SERVING_HEADER_BYTES 16640   /* status words and arrival counters at the head of every serving workspace */

/*
 * Per row t of T:  s = x[t] + residual[t];  y = s * rsqrt(mean(s^2) + eps) * weight;  then an 8-bit copy of y with scales:
 * scale_g = max(max|y over group g| / 448, 2^-100), q = y / scale_g rounded to nearest even.  Sums are held in 32 bits; y is
 * not rounded before it is quantised, and the norm is that of the unrounded s.  (The quotient is formed as (s * weight) * (factor /
 * scale), with an approximate reciprocal: q may be the neighbouring e4m3 value where y / scale lies within the roundings of its factors of a tie)
 *   x            [T][H] bf16, rows x_stride apart, in
 *   residual     [T][H] bf16, rows residual_stride apart, in, may be NULL
 *   weight       [H] bf16, in, may be NULL (all ones)
 *   group        128: one scale per 128 columns (the last group may be shorter); 0: one scale per row
 *   out_residual [T][H] bf16 contiguous, out, may be NULL: s rounded.  May be the buffer of x or of residual where that is
 *                contiguous too (a row is read before it is written; no other overlap)
 *   out_y        [T][H] bf16 contiguous, out, may be NULL: y rounded.  May be the buffer of x likewise
 *   out_q        [T][H] e4m3 contiguous, out, may be NULL;  out_scale [T][ceil(H/128) or 1] fp32, with out_q
 *   flags        CAKE_RMSNORM_NONE: no norm (y = s * weight): quantises alone
 * H <= 32768 (CAKE_ERR_UNSUPPORTED beyond).  Pointers are aligned to their elements; rows and bases that are multiples of
 * 16 bytes with H % 8 == 0 take the wide loads.  A row that holds an infinity or a NaN gives NaN in q where y is not finite.
 */
enum { CAKE_RMSNORM_NONE = 1 };
CAKE_API int cake_rmsnorm_quant(const cake_bf16* x, long long x_stride, const cake_bf16* residual, long long residual_stride,
                                const cake_bf16* weight, long long T, int H, float eps, int group, cake_bf16* out_residual,
                                cake_bf16* out_y, cake_e4m3* out_q, float* out_scale, cake_stream_t stream, unsigned flags);

/*
 * out[m][n] = sum over blocks kb of 128 columns of  x_scale[m][kb] * w_scale[n / 128][kb] * sum_{k in kb} X[m][k] W[n][k].
 * The product of a block is accumulated in 32 bits on the tensor cores, the blocks are scaled and added up in 32 bits, in
 * an order that depends on the sizes alone.
 *   X        [M][K] e4m3, rows x_stride apart, in        x_scale [M][ceil(K/128)] fp32 contiguous, in
 *   W        [N][K] e4m3, rows w_stride apart, in        w_scale [ceil(N/128)][ceil(K/128)] fp32 contiguous, in
 *   out      [M][N] rows out_stride apart, bf16, or fp32 with CAKE_GEMM_OUT_FP32, out
 *   ws       at least cake_gemm_fp8_workspace_bytes(M, N, K) bytes.  That number is not monotonic in M (a product of fewer rows may
 *            split its contraction where one of more does not): a buffer for products of several sizes has the largest
 *            of their numbers, or CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES, which no size exceeds
 * K % 16 == 0, x_stride % 16 == 0, w_stride % 16 == 0, X and W 16-byte aligned (CAKE_ERR_ALIGN).  M = 0 does nothing.
 */
enum { CAKE_GEMM_OUT_FP32 = 1 };
#define CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES 19415296   /* the header and 74 tiles of 256 x 256 fp32 */
CAKE_API int cake_gemm_fp8_workspace_bytes(long long M, int N, int K, size_t* out_bytes);
CAKE_API int cake_gemm_fp8(const cake_e4m3* X, long long x_stride, const float* x_scale, const cake_e4m3* W, long long w_stride,
                           const float* w_scale, long long M, int N, int K, void* out, long long out_stride, void* ws,
                           size_t ws_bytes, cake_stream_t stream, unsigned flags);

/*
 * A paged cache of keys and values: page p, token t of the page, head h: k + p*k_page_stride + t*k_token_stride +
 * h*k_head_stride, D contiguous elements there (the order of tokens and heads inside a page is the caller's).  Slot
 * s is token s % page_size of page s / page_size.
 *   type     CAKE_KV_BF16 or CAKE_KV_E4M3 (an element x of head h is held as e4m3(x / scale[h]), the quotient taken as x * (1 / scale[h]))
 *   k_scale, v_scale  [Hkv] fp32, device, normal numbers, may be NULL (all ones)
 * Base pointers are 16-byte aligned and every stride is a multiple of 16 bytes (CAKE_ERR_ALIGN).
 * D: 64, 96, 128 or 256 (CAKE_ERR_UNSUPPORTED otherwise).
 */
enum { CAKE_KV_BF16 = 0, CAKE_KV_E4M3 = 1 };
typedef struct cake_paged_cache {
    void* k;
    void* v;
    const float* k_scale;
    const float* v_scale;
    long long num_pages;
    long long k_page_stride, k_token_stride, k_head_stride;
    long long v_page_stride, v_token_stride, v_head_stride;
    int page_size, Hkv, D, type;
} cake_paged_cache;

/*
 * Writes the keys and values of T tokens to their slots, keys (and queries) rotated by their positions: of each head the
 * first `rot` elements, in pairs (i, i + rot/2), or (2i, 2i + 1) with CAKE_APPEND_INTERLEAVED:
 *   (a, b) -> (a cos - b sin, b cos + a sin),  cos = cos_sin[pos][i], sin = cos_sin[pos][rot/2 + i].
 * Arithmetic in 32 bits, one rounding at the store.
 *   cache      host pointer to the description above (read during the call)
 *   k, v       [T][Hkv][D] bf16, tokens k_stride / v_stride apart, heads D apart, in
 *   q          [T][Hq][D] bf16, tokens q_stride apart, in, may be NULL; out_q [T][Hq][D] bf16 contiguous, out (may be q's buffer)
 *   slots      [T] int64, in: the slot of each token.  A negative slot: keys and values of the token are not written (its
 *              queries are).  A slot beyond the cache: not written, and the device status becomes CAKE_ERR_BAD_INDEX
 *   positions  [T] int32, in;  cos_sin [max_positions][rot] fp32 contiguous, in.  rot = 0: no rotation, both may be NULL.
 *              A position outside [0, max_positions): nothing of the token is written, device status CAKE_ERR_BAD_INDEX
 * A slot that occurs twice among the T is left with elements of both tokens, in no particular mixture (the key of one beside the
 * value of the other, or parts of heads); no other slot is touched.  ws: CAKE_SERVING_HEADER_BYTES bytes.
 */
enum { CAKE_APPEND_INTERLEAVED = 1 };
CAKE_API int cake_kv_append(const cake_paged_cache* cache, const cake_bf16* k, long long k_stride, const cake_bf16* v,
                            long long v_stride, const cake_bf16* q, long long q_stride, int Hq, cake_bf16* out_q,
                            const long long* slots, const int* positions, const float* cos_sin, long long max_positions, int rot,
                            long long T, void* ws, size_t ws_bytes, cake_stream_t stream, unsigned flags);

/*
 * Attention of one query token per sequence and head over the sequence's cached tokens:
 *   out[b][h] = sum_t p_t v_t,  p = softmax over t of  scale * q[b][h] . k_t,  query head h reads key-value head h / (Hq / Hkv).
 *   q           [B][Hq][D] bf16, sequences q_stride apart, heads q_head_stride apart, in
 *   page_table  int32, in: token t of sequence b (and key-value head g) is in page
 *               page_table[b*table_stride + g*table_head_stride + t / page_size], token t % page_size of it;
 *               table_head_stride = 0: one table for all heads.  Only entries of the tokens attended to are read; max_pages
 *               bounds the entries of a row.  A page outside [0, num_pages): its tokens are left out, device status
 *               CAKE_ERR_BAD_INDEX
 *   seq_lens    int32, in: tokens of sequence b (and head g): seq_lens[b*lens_stride + g*lens_head_stride]; a length
 *               beyond max_pages * page_size is cut to it (device status CAKE_ERR_BAD_INDEX)
 *   window      0: all tokens; w > 0: the last w of them
 *   out         [B][Hq][D] bf16 contiguous, out;   out_lse [B][Hq] fp32, out, may be NULL: log of the sum of exponentials
 *   ws          at least cake_paged_decode_workspace_bytes(...) bytes
 * A row without tokens (length zero, or none that weighs anything) gives zeros, and -inf in out_lse.  Scores, their maximum and
 * sum, and the weighted sum of values are held in 32 bits (a value that is infinite, in a bf16 cache, may give NaN instead of
 * infinity); memory behind the last token is never read.  Weights are held with 11 bits or more; with an 8-bit cache, those
 * below 2^-25 of the row's heaviest to 2^-36 of it, and elements of a query below 2^-14 of its largest to 2^-25 of that.
 * One launch; two where the query heads of a key-value head have more than 512 elements in all (256 with bf16 heads of 256) and
 * the page table's width, cut by the window, leaves room for rows in many parts: a max_pages no larger than the longest row
 * needs saves the second.  The result depends on the inputs and their sizes, not on timing.
 */
CAKE_API int cake_paged_decode_workspace_bytes(long long B, int Hq, int Hkv, int D, size_t* out_bytes);
CAKE_API int cake_paged_decode(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_paged_cache* cache,
                               const int* page_table, long long table_stride, long long table_head_stride, int max_pages,
                               const int* seq_lens, long long lens_stride, long long lens_head_stride, long long B, int Hq,
                               float scale, int window, cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes,
                               cake_stream_t stream);

/*
 * Attention of many query tokens.  A sequence b has the query tokens starts[b] up to starts[b + 1] of the T that lie one behind the
 * other; with n of them and L keys, token i is at position p = L - n + i among the keys and sees
 *   causal:      the keys up to its own position, [0, p + 1)
 *   window w>0:  the last w of those, [max(0, p - w + 1), p + 1)
 *   otherwise:   all L keys
 *   out[token][h] = sum_t p_t v_t,  p = softmax over the keys t that it sees of  scale * q[token][h] . k_t,
 * query head h reads key-value head h / (Hq / Hkv).
 *   q          [T][Hq][D] bf16, tokens q_stride apart, heads q_head_stride apart, in
 *   starts     [B + 1] int32, device, in: 0 <= starts[b] <= starts[b + 1] <= T; a sequence for which that does not hold is left out
 *              (device status CAKE_ERR_BAD_INDEX).  Tokens of no sequence are left as they were in out and out_lse
 *   out        [T][Hq][D] bf16 contiguous, out;   out_lse [T][Hq] fp32 contiguous, out, may be NULL: log of the sum of exponentials;
 *              neither overlaps an input
 *   ws         at least cake_attention_workspace_bytes(Hq, Hkv, D) bytes: any number of sequences and tokens
 *   scale      any number; zero weighs all keys alike.  NaN (here, or in an 8-bit cache's k_scale) makes every row NaN that sees something
 * A token that sees nothing (or nothing that weighs anything) gives zeros, and -inf in out_lse.  Keys and values that a token does
 * not see do not touch its row, infinities and NaN among them (a row that meets such values in a tile of 128 keys beside its own is computed
 * again from its keys: right, and slow, 2 to 3 us a key for 32 such rows; beyond about a million keys that one block has of them the wait for it may
 * run out: device status CAKE_ERR_TIMEOUT).  A row whose weighted sum of finite values passes 32 bits is computed again likewise.
 * An infinite value that a token sees may give NaN instead of infinity.  Scores, their maximum and sum, and the weighted sum of values are held in 32 bits.  The weights are
 * rounded to bf16 for the product with the values (8-bit caches: to f16, 11 bits down to 2^-25 of a row's heaviest, in steps of 2^-35
 * of it below), their sum is not.  8-bit caches: queries are divided by a power of two per head and rounded to f16 (exact down to 2^-14 of the head's largest element).  D: 64, 96, 128 or 256
 * (CAKE_ERR_UNSUPPORTED otherwise).  q, k, v and out are 16-byte aligned and strides multiples of 8 elements, at least D
 * (CAKE_ERR_ALIGN, CAKE_ERR_SHAPE); the stride of a dimension of one element is not looked at.  One launch where no item
 * can be shared by blocks (fewer than eight tiles of 128 keys: Tk, or the table's width, or the window), two otherwise.  The result depends on the
 * inputs and their sizes, not on timing.
 */
CAKE_API int cake_attention_workspace_bytes(int Hq, int Hkv, int D, size_t* out_bytes);
/*
 * Packed prompts: keys and values lie one sequence behind the other.
 *   k, v       [Tk][Hkv][D] bf16, in, strides as for q
 *   k_starts   [B + 1] int32, device, in: as starts, of the keys (<= Tk); NULL: starts (Tk >= T then, or sequences are left out)
 *   flags      CAKE_ATTENTION_CAUSAL; window needs it (CAKE_ERR_UNSUPPORTED)
 */
enum { CAKE_ATTENTION_CAUSAL = 1 };
CAKE_API int cake_prompt_attention(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_bf16* k, long long k_stride,
                                   long long k_head_stride, const cake_bf16* v, long long v_stride, long long v_head_stride,
                                   const int* starts, const int* k_starts, long long B, long long T, long long Tk, int Hq, int Hkv, int D,
                                   float scale, int window, cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes,
                                   cake_stream_t stream, unsigned flags);
/*
 * A chunk of new tokens per sequence over a paged cache that holds their keys and values already (causal).
 *   page_table, seq_lens   as for cake_paged_decode: seq_lens counts the chunk's tokens too (they are the last ones); per key-value
 *              head with table_head_stride, lens_head_stride.  Only entries of keys that some token of the chunk's block of
 *              neighbouring tokens sees are read, and no memory of other keys.  A page outside [0, num_pages): its keys are left
 *              out, device status CAKE_ERR_BAD_INDEX; a length beyond max_pages * page_size is cut to it (likewise)
 */
CAKE_API int cake_paged_chunk(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_paged_cache* cache,
                              const int* page_table, long long table_stride, long long table_head_stride, int max_pages,
                              const int* seq_lens, long long lens_stride, long long lens_head_stride, const int* starts, long long B,
                              long long T, int Hq, float scale, int window, cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes,
                              cake_stream_t stream);

/*
 * The norm of each query and key head, the rotation of cake_kv_append, and its write to the cache, in one pass:
 *   y = x * rsqrt(mean over the head's D elements of x^2 + eps) * weight, then rotated as there.  Values are neither.  Arithmetic
 * in 32 bits, one rounding at the store.
 *   q          [T][Hq][D] bf16, tokens q_stride apart, heads D apart, in;  k, v [T][Hkv][D] likewise
 *   q_weight, k_weight  [D] bf16, in, may be NULL (all ones)
 *   out_q      [T][Hq][D] bf16 contiguous, out (may be q's buffer where that is contiguous too)
 *   out_k      [T][Hkv][D] bf16 contiguous, out, may be NULL (may be k's buffer likewise): the keys beside the cache, of tokens with a
 *              negative slot too, for the attention of a prompt whose keys need not be read back
 * cache, slots, positions, cos_sin, rot, flags and what an index out of range does: as for cake_kv_append.  A position out of range
 * leaves out_q and out_k of that token as they were.  ws: CAKE_SERVING_HEADER_BYTES bytes.
 */
CAKE_API int cake_qk_norm_append(const cake_paged_cache* cache, const cake_bf16* q, long long q_stride, int Hq, const cake_bf16* k,
                                 long long k_stride, const cake_bf16* v, long long v_stride, const cake_bf16* q_weight,
                                 const cake_bf16* k_weight, float eps, cake_bf16* out_q, cake_bf16* out_k, const long long* slots,
                                 const int* positions, const float* cos_sin, long long max_positions, int rot, long long T, void* ws,
                                 size_t ws_bytes, cake_stream_t stream, unsigned flags);

/*
 * Reads keys and values of N tokens back from their slots: out[n][h] = bf16(cache[slots[n]][h] * scale[h]) (a bf16 cache's as they are).
 *   slots      [N] int64, in, any order, repeats allowed.  A negative slot gives zeros; a slot beyond the cache likewise, and the
 *              device status becomes CAKE_ERR_BAD_INDEX
 *   out_k, out_v  bf16, out, either may be NULL: token n and head h at n * out_stride + h * out_head_stride, D contiguous elements
 *              (tokens outermost, or a matrix [N][D] for each head, as the clustering takes them).  16-byte aligned, strides
 *              multiples of 8 elements and at least D
 * ws: CAKE_SERVING_HEADER_BYTES bytes.
 */
CAKE_API int cake_kv_read(const cake_paged_cache* cache, const long long* slots, long long N, cake_bf16* out_k, cake_bf16* out_v,
                          long long out_stride, long long out_head_stride, void* ws, size_t ws_bytes, cake_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* CAKE_SERVING_H_ */
