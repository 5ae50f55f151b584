/*
 * gnr_iter.h -- C ABI of the operators of one batch iteration on MI355X: what a simulated server stands for.
 *
 * An iteration of a server advances every decode of its batch by one token and the prefill in service by a chunk (Sec. 2.2
 * of the paper). Its duration, c0 + c_pre*prefill_tokens + c_dec*n_decode in gnr_sim.h, is what these operators take: the
 * new tokens' keys and values are written to a paged cache (iter_kv_write), every token is run over its own request's
 * cache (iter_attention), the adapter of each request's class is added to the projections that all classes share
 * (iter_adapters), and a request that is routed from its prefill's server to another takes its cache along
 * (iter_kv_read there, iter_kv_write here).
 *
 * Beside these: the positions of queries and keys (iter_rotary, and iter_rotary_write, which puts the keys and values into the cache
 * as well), and pages that change places or are shared and then written (iter_copy_pages).
 *
 * The library is libgnr_sim.so, the errors are gnr_sim.h's. Every function returns SIM_OK or a negative sim_err; none
 * throws, aborts or prints. Device pointers are marked; everything else is host memory and read before the call returns.
 * Work is enqueued on `hip_stream` (a hipStream_t, NULL = default stream) of the current device, to which the device
 * pointers have to belong; no function waits, allocates or copies, so each can be captured into a graph, which then reads
 * whatever the arrays hold when it is launched. Results are the same from run to run: nothing is summed by atomics.
 *
 * What the host can see is checked before anything is launched (SIM_EINVAL). What only the device sees (batch bounds,
 * page and adapter numbers) is checked by the kernels: they touch no memory outside the arrays whatever the numbers are,
 * treat what is out of bounds as absent, and add bits of enum iter_status to a word of the caller's.
 */
#ifndef GNR_ITER_H
#define GNR_ITER_H

#include "gnr_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ITER_MAX_REQUESTS 1024  /* requests of one batch */
#define ITER_MAX_TOKENS (1 << 21) /* its tokens; its rows (tokens times query heads of a kv head): 16 times as many */
#define ITER_MAX_ADAPTERS 2048  /* adapters loaded */
#define ITER_MAX_RANK 128
#define ITER_MAX_LAYERS 1024    /* caches of iter_copy_pages */

/* Element types. FP8 (e4m3: 4 exponent bits, 3 of mantissa, largest value 448, no infinity) and FP4 (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives; two elements to a byte, the first in its lower half) are cache types only. */
enum iter_type { ITER_BF16 = 0, ITER_FP16 = 1, ITER_FP8 = 2, ITER_FP4 = 3 };

/* BATCH: q_start does not ascend within [0, tokens], or a kv_len is negative or longer than its row of the page table (or 2^30).
 * PAGE: a page number outside the cache. ADAPTER: an adapter number outside [-1, adapters). */
enum iter_status { ITER_BAD_BATCH = 1, ITER_BAD_PAGE = 2, ITER_BAD_ADAPTER = 4 };

/* Keys or values of a paged cache: element (page, head, place, d) is data[page*page_stride + head*head_stride +
 * place*place_stride + d], strides in elements, non-negative (place_stride and exp_place_stride at most 2^24), the data and every row 16-byte aligned. Of an FP8 cache the row (page, head,
 * place) stands for its codes times 2^(exp - 127), where exp is the byte at exp[page*exp_page_stride + head*exp_head_stride +
 * place*exp_place_stride] (1..254). Of an FP4 cache every 32 elements of a row have a byte of their own, which follow each other: that of the elements from 32*i on is i
 * bytes further on (1..254; what a byte of 0 reads as is not said), and one of 255 stands for 32 that are no numbers; strides count elements, two of which are a byte. Other caches have no exponents (NULL). */
typedef struct {
  void *data;                                              /* device */
  uint8_t *exp;                                            /* device */
  int64_t page_stride, head_stride, place_stride;
  int64_t exp_page_stride, exp_head_stride, exp_place_stride;
} iter_plane;

/* The cache of one layer. head_dim: 64, 128 or 256; page (tokens of a page): a power of two up to 65536. A slot is the number
 * page * page_size + place of a token's rows. */
typedef struct {
  int type;                                                /* enum iter_type */
  int kv_heads, head_dim, page;
  int64_t pages;
  iter_plane k, v;
} iter_cache;

/* Rows of tokens: element (token, head, d) at data[token*token_stride + head*head_stride + d], 16-byte aligned rows. */
typedef struct {
  void *data;                                              /* device */
  int64_t token_stride, head_stride;
} iter_rows;

/* Writes the keys and values of `tokens` tokens ([tokens][kv_heads][head_dim] each, type BF16 or FP16) into the slots
 * `slots` (device, distinct; a slot outside the cache is no place: that token is not kept). An FP8 cache takes every
 * row in units of 2^e: e is the least whole number from -126 on with max|x| <= 448 * 2^e (0 for a row of zeros), a code is
 * x * 2^-e rounded to nearest even. A power of two costs no accuracy (codes are floating point themselves), and reading
 * back is exact in 16 bits wherever the value is in range. A row that holds a NaN or an infinity is stored as NaN throughout.
 * An FP4 cache takes every 32 elements of a row in units of a 2^e of their own in the same way, with max|x| <= 6 * 2^e; 32 that hold a NaN or an infinity are stored as NaN (and
 * magnitudes of BF16 from 3.5 * 2^126 on are nearest to a code that reads as infinite).
 * Any other cache has to be of the rows' type. */
int iter_kv_write(const iter_cache *cache, int type, const iter_rows *k, const iter_rows *v, const int64_t *slots,
                  int64_t tokens, void *hip_stream);

/* Reads the rows of `slots` (device) back as values of `type` (BF16 or FP16; for other caches than FP8 and FP4 the cache's). A
 * slot outside the cache gives zeros. */
int iter_kv_read(const iter_cache *cache, int type, const iter_rows *k, const iter_rows *v, const int64_t *slots,
                 int64_t tokens, void *hip_stream);

/* A batch: request r brings the tokens q_start[r] .. q_start[r+1]-1 (one for a decode, a chunk for a prefill, none is
 * fine; a batch of tokens has a request), which are the last ones of the kv_len[r] that its cache holds; token j of a request lies at place j % page of
 * page page_table[r*table_stride + j / page]. All arrays on the device, q_start with requests + 1 entries ascending from 0 to `tokens`.
 * max_q is what the host expects of the longest chunk: it selects kernels, results depend on it being right in nothing but their rounding. */
typedef struct {
  int requests;
  int64_t tokens, max_q;
  const int32_t *q_start, *kv_len, *page_table;            /* device */
  int64_t table_stride, table_width;                       /* entries of a row of the page table, and those in use */
} iter_batch;

/* Device bytes of the workspace iter_attention needs (16-byte aligned; what is in it does not matter and does not last). */
int iter_attention_bytes(const iter_cache *cache, const iter_batch *batch, int heads, size_t *out_bytes);

/* Attention of the batch's tokens over their requests' caches: q and out are [tokens][heads][head_dim] of `type` (BF16 or
 * FP16; the cache's type or, for an FP8 or FP4 cache, either), heads a multiple of kv_heads, and query head h reads kv head
 * h / (heads / kv_heads). Keys and values of an FP8 or FP4 cache are what iter_kv_read gives in `type`: for FP16
 * infinite from 65520 on and rounded to multiples of 2^-24, which takes nothing from rows that were written from FP16 and stayed below 63488 (FP4: 57344; rows of larger or smaller BF16
 * values belong to BF16 queries). The token at position p = kv_len - q_len + i of its request sees positions max(0, p - window + 1) .. p
 * (window = 0: 0 .. p): out = sum_j w_j v_j / sum_j w_j, w_j = exp(scale * q.k_j). A token that sees nothing gets zeros. What lies
 * where a token does not look (NaN included) does not matter. Scores, sums and outputs are held in 32 bits. For
 * the matrix product with the values the weights are the sum of two numbers of `type` each where a request has up to 16 rows (its tokens times query heads of a kv head), and
 * rounded to one number, relative to the largest of their row, where it has more. Rows of tokens outside every request (of a batch with
 * bounds out of range) are not written. out must not overlap q, nor be the same rows. There is no backward pass. */
int iter_attention(const iter_cache *cache, const iter_batch *batch, int type, int heads, const iter_rows *q,
                   const iter_rows *out, double scale, int64_t window, void *workspace, size_t bytes, uint32_t *status,
                   void *hip_stream);

/* Low-rank adapters, beside a projection that all requests share: for the tokens t of request r with a = adapter[r],
 * out[t] = base[t] + scale[a] * up[a] (down[a] x[t]), out[t] = base[t] for a = -1. x is [tokens][width_in], base and out
 * [tokens][width_out] (rows 16-byte aligned; out may be base itself or apart from it, and either may be or overlap x), down [adapters][rank][width_in] and up
 * [adapters][width_out][rank] without gaps, all of `type`; scale fp32. Widths and rank: multiples of 8, rank up to ITER_MAX_RANK. */
typedef struct {
  int adapters, rank;
  int64_t width_in, width_out;
  const void *down, *up;                                   /* device */
  const float *scale;                                      /* device */
} iter_adapter_set;

/* Device bytes of the workspace iter_adapters needs for any such call (whether it uses them goes by the batch and by whether out overlaps x). */
int iter_adapters_bytes(const iter_adapter_set *set, int64_t tokens, size_t *out_bytes);
int iter_adapters(const iter_adapter_set *set, int type, int requests, int64_t tokens, const int32_t *q_start,
                  const int32_t *adapter, const void *x, int64_t x_stride, const void *base, int64_t base_stride,
                  void *out, int64_t out_stride, void *workspace, size_t bytes, uint32_t *status, void *hip_stream);

/* Positions: of every pair of elements (a, b) of a row, a' = m (a cos t - b sin t) and b' = m (b cos t + a sin t). Pair i of dims / 2 is the elements (i, i + dims / 2), or
 * (2 i, 2 i + 1) if `interleaved`; elements from `dims` on stay as they are. t = position * turns[i] / 2^64 of a full turn: turns[i] is the part of a turn that a position is worth,
 * as a whole number of 2^-64, of which whole turns may be left out, so that angles are exact modulo a turn at any position (a number of 64 bits, of either sign). `dims` is a multiple of 16 up to the
 * head's. m, `magnitude`, is finite. `inverse` turns the other way: for m = 1 it undoes the turn, and it is what gradients of the results take back to x. Angles, sines and products are held in 32 bits
 * or more, sines and cosines within 2^-23. */
typedef struct {
  int dims, interleaved, inverse;
  float magnitude;
  const int64_t *turns;                                    /* device, dims / 2 */
} iter_turns;

/* Rows of `heads` heads of head_dim (64, 128 or 256) elements of `type` (BF16 or FP16), turned: out may be x itself (the same rows) or apart from it: in other memory, beside it in
 * the rows of one matrix, or with heads or tokens that alternate with x's at common strides. */
int iter_rotary(int type, int heads, int head_dim, const iter_turns *turns, const int64_t *positions, int64_t tokens, const iter_rows *x,
                const iter_rows *out, void *hip_stream);

/* iter_rotary of the queries (`heads` heads; q_out may be q itself or apart from q, k and v; none: heads = 0) and of the keys, and iter_kv_write of these and the values, in one launch: the
 * same bits as one after the other, the keys rounded to `type` before they are stored. */
int iter_rotary_write(const iter_cache *cache, int type, int heads, const iter_turns *turns, const int64_t *positions, const iter_rows *q, const iter_rows *q_out,
                      const iter_rows *k, const iter_rows *v, const int64_t *slots, int64_t tokens, void *hip_stream);

/* Copies pages of the caches of `n_layers` layers, which are alike but for their addresses: of every page source[i] the first places[i] places (places = NULL: all of them) to page
 * target[i]. A source may have several targets. Page numbers out of range, a target that is named twice or is a source as well, and places outside [0, page] are refused
 * (SIM_EINVAL) before anything is copied. The three lists are host memory and become part of what is launched: a captured call copies the same pages whenever it is replayed. Needs 16 bytes of
 * host memory for a copy while it checks more than 64 (SIM_ENOMEM). */
int iter_copy_pages(const iter_cache *layers, int n_layers, const int64_t *source, const int64_t *target, const int64_t *places, int64_t count,
                    void *hip_stream);

/* sizeof of iter_turns (for binding checks). */
int iter_turns_size(size_t *out_bytes);

/* sizeof of the other five ABI structs, in the order plane, cache, rows, batch, adapter set (for binding checks). */
int iter_abi_sizes(size_t *out5);

#ifdef __cplusplus
}
#endif
#endif
