/*
 * kvx_latent.h -- latent attention over a paged pool of one shared vector a token,
 * on AMD MI355X (gfx950).
 *
 * The model.  A token's cache entry is a latent vector c of latent_dim values and one
 * rotated key r of rope_dim values; all query heads share both.  Head h has two weights,
 * W_uk[h] (nope_dim x latent_dim) and W_uv[h] (v_dim x latent_dim), and attends with
 *   key    k = (W_uk[h] c, r)     value  v = W_uv[h] c.
 * Its scores and outputs can be had in two forms that are equal in exact arithmetic:
 *   expanded  keys and values are formed for every cached token and head, then attended;
 *   absorbed  the query is taken into the latent space, q' = (W_uk[h]^T q_nope, q_rope),
 *             attends to the entries (c, r) themselves, and W_uv[h] is applied to the
 *             weighted sum of latents.
 * A query costs about (2 latent_dim + rope_dim) / (nope_dim + rope_dim + v_dim) times as
 * much per key in the absorbed form, and the expansion of every key is saved: that form
 * suits single tokens, drafted tokens and short turns; long suffixes suit the other.
 *
 * The pages, the page table and the batch are those of kvx.h: pages of 16 tokens, request r
 * with a prefix of P_r tokens in the pool and a suffix of E_r tokens.  kvx_cache.h and
 * kvx_radix.h serve a latent pool as they serve a KV pool, except for the host tier of a cache:
 * a latent pool has no spill, reload or raw page moves, so its cache is one without
 * (kvx_cache_create).  The conventions at the head of kvx.h hold here too (status codes, checks
 * before any work, streams, one pool's calls in order, scratch that grows, page ids and
 * KVX_VALIDATE).  Besides:
 *   - A call runs on the pool's device and leaves the caller's current device as it was.  A
 *     stream of another device is refused (KVX_EINVAL).
 *   - A stream that is being captured into a HIP graph is refused (KVX_EUNSUPPORTED): the
 *     plan of a call is made on the host, from the lengths of its batch.
 *   - Results (q_out, out, lse) overlap no input of their call and not each other (KVX_EINVAL),
 *     but for q_out in place of q.
 *   - Scores are float32, also times sm_scale and log2 e: one below -3.4e38 counts as -inf, a
 *     weight of zero, and one above 3.4e38 makes its row's result and lse NaN.  A row whose scores are
 *     all -inf gives zeros and an lse of -inf.
 *   - Cache rows that attention reads are finite.  A row that is not may reach any query
 *     row of its request, those before it too.  Slots past a request's P_r + E_r tokens
 *     reach none, whatever they hold.
 */
#ifndef KVX_LATENT_H
#define KVX_LATENT_H

#include "kvx.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kvx_latent_pool kvx_latent_pool; /* opaque; owned by the library */

enum kvx_latent_dtype {
    KVX_LATENT_BF16 = 0, /* c and r as bf16 */
    KVX_LATENT_FP8 = 1   /* c as e4m3 codes with a power of two for each 64 of them, r as bf16 */
};

enum kvx_latent_form {
    KVX_LATENT_AUTO = 0,     /* by the batch's lengths, request by request: whichever is estimated to be faster */
    KVX_LATENT_ABSORBED = 1,
    KVX_LATENT_EXPANDED = 2
};

/* Device layout of a pool, for tests and tools.  A page holds 16 tokens in page_bytes
 * contiguous bytes.  bf16: [16][latent_dim + rope_dim].  fp8: codes [16][latent_dim], then
 * bf16 keys [16][rope_dim], then scale bytes, 2^(byte - 127): the byte of slot s and group g
 * (of 64 values) is at
 * ((s % 8) * 2 + g % 2) * (latent_dim / 64) + s / 8 * (latent_dim / 128) + g / 2. */
typedef struct {
    void *base; /* device */
    int64_t num_pages;
    int64_t page_bytes;
    int32_t page_size;
    int32_t latent_dim;
    int32_t rope_dim;
    int32_t dtype;         /* enum kvx_latent_dtype */
    int32_t key_offset;    /* bytes from a page's start to its rotated keys (bf16: of token 0's) */
    int32_t scale_offset;  /* bytes to the scale bytes; 0 for bf16 */
} kvx_latent_layout;

/*
 * Allocate a pool of `num_pages` pages of `page_size` tokens (must be 16), zeroed.
 *   latent_dim  256 or 512.    rope_dim  64.    dtype  enum kvx_latent_dtype.
 * Synchronous.  Errors: EINVAL, EUNSUPPORTED (sizes), ENOMEM, EHIP.
 */
int latent_pool_create(int64_t num_pages, int32_t page_size, int32_t latent_dim, int32_t rope_dim, int32_t dtype,
                       kvx_latent_pool **out);

/* Free a pool (waits for the device to go idle first).  NULL is a no-op. */
int latent_pool_destroy(kvx_latent_pool *pool);

/* Fill *out with the pool's device layout.  Errors: EINVAL. */
int latent_pool_layout(const kvx_latent_pool *pool, kvx_latent_layout *out);

/* As kv_pool_set_split_keys, for latent_attention and the absorbed form: key ranges are
 * split every `keys` tokens (a multiple of 64; 0 = automatic).  More where the parts would
 * be too many.  Errors: EINVAL. */
int latent_pool_set_split_keys(kvx_latent_pool *pool, int32_t keys);

/*
 * Write the suffix's cache entries: suffix token i of request r goes to slot t % 16 of
 * logical page t / 16, t = P_r + i.
 *   kv         device bf16, row i at kv + i * kv_stride: latent_dim values of c, then
 *              rope_dim values of r (both as they shall be cached)
 *   kv_stride  elements between rows: a multiple of 8, >= latent_dim + rope_dim
 * bf16 pool: the bits are copied.  fp8 pool: for each 64 consecutive values of c, e is the
 * smallest integer with max|c| <= 448 * 2^e, held to [-117, 119], and each value is stored
 * as e4m3(clamp(c * 2^-e, -448, 448)), rounded to nearest even, NaN as NaN.  A power of two
 * makes every stored value code * 2^e a bf16 value: reading rounds nothing.
 * Slots not written by the batch keep their contents; so do rows past the last suffix
 * token.  Errors: EINVAL, EUNSUPPORTED (capturing stream), ERANGE (validation mode),
 * ENOMEM, EHIP.  R = 0 or T = 0: no-op.
 */
int store_latent(kvx_latent_pool *pool, const kvx_batch *batch, const void *kv, int64_t kv_stride,
                 kvx_stream_t stream);

/*
 * store_latent with the steps before it fused in, for the suffix token at position t:
 *   c  is normalised when rope->k_norm is given (device bf16 [latent_dim]):
 *      c * k_norm / sqrt(mean(c^2) + norm_eps);
 *   r  turns as store_kv_rope turns a head (theta or inv_freq, style; rotary_dim must be
 *      rope_dim), and so do the last rope_dim values of every query head.
 * Arithmetic is float32, with every angle reduced to one turn in float64 first; each result
 * is rounded once (on an fp8 pool, c once, to its code).
 *   rope         q_norm must be NULL
 *   q, q_out     device bf16 [T, num_q_heads, q_dim], q_dim a multiple of 8 in
 *                [rope_dim, 4096]; q_out may be q itself, where only the rotated values are
 *                touched, but may not overlap it otherwise (EINVAL); unused when
 *                num_q_heads = 0
 * Otherwise as store_latent.
 */
int store_latent_rope(kvx_latent_pool *pool, const kvx_batch *batch, const kvx_rope *rope, const void *q,
                      int32_t num_q_heads, int32_t q_dim, void *q_out, const void *kv, int64_t kv_stride,
                      kvx_stream_t stream);

/*
 * Read cache entries back: row i of request r's E_r rows is token P_r + i, as bf16
 * [latent_dim + rope_dim], dequantised (exactly) on an fp8 pool.
 *   out         device bf16, row i at out + i * out_stride; values between rows are kept
 *   out_stride  elements between rows: a multiple of 8, >= latent_dim + rope_dim
 * Errors as store_latent.
 */
int load_latent(kvx_latent_pool *pool, const kvx_batch *batch, void *out, int64_t out_stride, kvx_stream_t stream);

/*
 * Attention to the cache entries themselves: for each request r, suffix row i and head h,
 *   o = softmax_j(sm_scale * q . (c_j, r_j)) c_j   over tokens j = 0 .. P_r + i
 * of the request's logical sequence (store_latent of the suffix must precede it on the
 * stream).  The core of the absorbed form, for callers who keep W_uk and W_uv in weights
 * of their own.
 *   q            device bf16 [T, num_q_heads, latent_dim + rope_dim]
 *   num_q_heads  1 to 1024; a request's E_r * num_q_heads is at most 2^31 - 1025, its P_r + E_r at
 *                most 2^31 - 2^23 (EUNSUPPORTED)
 *   sm_scale     > 0, at most 2e38
 *   out          device bf16 [T, num_q_heads, latent_dim] (round to nearest even)
 *   lse          device fp32 [T, num_q_heads] natural-log sum of exp of the scaled scores,
 *                or NULL
 * Products take bf16 operands (the softmax weights are rounded to bf16) and accumulate in
 * float32.  Errors: as store_latent.  R = 0 or T = 0: no-op.
 */
int latent_attention(kvx_latent_pool *pool, const kvx_batch *batch, const void *q, int32_t num_q_heads,
                     float sm_scale, void *out, float *lse, kvx_stream_t stream);

typedef struct {
    const void *w_uk;    /* device bf16 [num_q_heads][nope_dim][latent_dim] */
    const void *w_uv;    /* device bf16 [num_q_heads][v_dim][latent_dim] */
    int32_t num_q_heads; /* 1 to 1024, with the limits of latent_attention */
    int32_t nope_dim;    /* 64 or 128 */
    int32_t v_dim;       /* equal to nope_dim */
} kvx_latent_proj;

/*
 * Latent attention from per-head queries to per-head outputs: for each request r, suffix
 * row i and head h,
 *   o = softmax_j(sm_scale * q . k_j) v_j,  k_j = (W_uk[h] c_j, r_j),  v_j = W_uv[h] c_j,
 * over tokens j = 0 .. P_r + i.
 *   q     device bf16 [T, num_q_heads, nope_dim + rope_dim] (the last rope_dim rotated)
 *   out   device bf16 [T, num_q_heads, v_dim] (round to nearest even)
 *   lse   device fp32 [T, num_q_heads], or NULL
 *   form  enum kvx_latent_form.  The expanded form takes at most 2^31 - 1 tokens P_r + E_r in
 *         all, each request's rounded up to 64 (EUNSUPPORTED); past that the automatic choice is
 *         the absorbed form for every request
 * Intermediate rows -- expanded keys and values, or queries and sums in the latent space --
 * are rounded to bf16 once each, so the two forms differ by such roundings, and the scores
 * behind lse carry one.  Uses library-owned device workspaces: for the expanded form the keys
 * and values of as many heads at a time as 2 GiB holds (at least one), and the rotated keys; for the absorbed form
 * 2 (2 latent_dim + rope_dim) + 4 bytes for each of its suffix tokens and heads; for either up
 * to 2 GiB of partial results.
 * Errors: as store_latent.  R = 0 or T = 0: no-op.
 */
int latent_extend_attention(kvx_latent_pool *pool, const kvx_batch *batch, const kvx_latent_proj *proj,
                            const void *q, float sm_scale, void *out, float *lse, int32_t form,
                            kvx_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* KVX_LATENT_H */
