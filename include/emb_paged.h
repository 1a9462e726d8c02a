/*
 * emb_paged.h -- C ABI of libembpaged.so: a paged key/value cache for several requests, what
 * fills it and the attention that reads it (GB300, sm_103a).
 *
 * Paper: "Embodied.cpp: A Portable Inference Runtime of Embodied AI Models on
 * Heterogeneous Robots" (arXiv 2607.02501). It runs every model family through one backbone
 * execution path (Section 3.2) whose prefix is computed once and attended to by many steps
 * (Section 3.1), and defines none of these operators; the standard definitions are used.
 *
 * A serving step over several requests (robots, cameras, dialogues):
 *   emb_paged_slots      once per step: every new token gets a place in the cache
 *   per layer, behind the q/k/v projection of emb_qlayer_seq:
 *     emb_qk_norm_rope   queries and keys normalised and rotated, keys and values stored
 *     emb_paged_attention  the new tokens attend to their request's whole history
 *
 * The cache of one layer is two arrays, K and V, bf16 [n_pages][page_size][n_kv_heads][head_dim].
 * A request's tokens lie in the pages that its row of the block table names, in order: token
 * `pos` of request r at page table[r][pos / page_size], place pos % page_size. Its slot is
 * page * page_size + place.
 *
 * Conventions are those of emb_qmm.h (device pointers owned by the caller, no allocation, no
 * host synchronisation, argument errors before anything is enqueued, programmatic dependent
 * launch; calls can be recorded with emb_chain_record_begin). Like the norm, rotary and attention calls of
 * emb_qmm.h, they let the next launch start while work ahead of them may still run (emb_qlayer_seq_chained). Lengths, tables, slots and
 * positions are read on the device, so a recorded call follows them from replay to replay.
 * What they hold cannot fault: each entry point says what an impossible value does.
 */
#ifndef EMB_PAGED_H
#define EMB_PAGED_H

#include "emb_qmm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Section 3.2, principle 2 (buffer reuse: the caller owns the cache, this call hands out its pages).
 * Block table, slots and positions of a step. Request r (of n_req) has cached[r] tokens in the
 * cache and gets added[r] new ones (negative counts are taken as 0). With P = page_size,
 * have_r = ceil(cached[r] / P), want_r = ceil((cached[r] + added[r]) / P), both at most max_pages:
 *   table[r][have_r .. want_r) = the next want_r - have_r entries of free_pages, taken in request
 *     order from entry *used on (-1 past entry n_free); the rest of `table` is left as it is;
 *   *used_out = *used + all pages taken, more than n_free if the list ran out;
 *   q_start[r] = sum of added[0 .. r), q_start[n_req] the total;   kv_len[r] = cached[r] + added[r];
 *   new token i of request r, token t = q_start[r] + i of the step, sits at positions[t] = cached[r] + i
 *     and slots[t] = table[r][pos / P] * P + pos % P, or -1 if that entry is negative or past max_pages;
 *   tokens from q_start[n_req] to n_tokens (padding of a recorded step): positions 0, slots -1.
 * A step whose total is above n_tokens gives its tokens past n_tokens neither slot nor page.
 * cached, added: int32 [n_req]; free_pages: int32 [n_free]; used, used_out: int32 [1] (different buffers);
 * table: int32 [n_req][max_pages], in and out; q_start: int32 [n_req + 1]; kv_len: int32 [n_req];
 * slots: int64 [n_tokens]; positions: int32 [n_tokens]. The sums of lengths fit in int32.
 * The same inputs give the same outputs, so a call may be repeated.
 * 1 <= n_req <= 65536, 0 <= n_tokens < 2^31, 0 <= n_free < 2^31, 1 <= page_size <= 65536,
 * 1 <= max_pages < 2^31; n_req * max_pages < 2^46. Pointers aligned to their type; slots, positions and free_pages may be
 * NULL when they have no entries. No output may overlap another buffer.
 * Errors: EMB_EINVAL, EMB_EALIGN, EMB_ECUDA. */
EMB_API emb_status emb_paged_slots(const int32_t* cached, const int32_t* added, int64_t n_req,
                                   const int32_t* free_pages, int64_t n_free, const int32_t* used,
                                   int64_t page_size, int32_t* table, int64_t max_pages, int32_t* q_start,
                                   int32_t* kv_len, int64_t* slots, int32_t* positions, int64_t n_tokens,
                                   int32_t* used_out, emb_stream_t stream);

/* Section 3.2 (the shared backbone layer around the linears), principle 2 (fusion: one pass from the
 * projections to the cache).
 * Per-head RMSNorm of queries and keys (Zhang and Sennrich, 2019; skipped where the gamma is NULL), rotary
 * embedding (Su et al., 2021; rotate-half pairs) with one or several position axes, and the cache write.
 * For token t, every query head and every key head x [head_dim]:
 *   y_i = x_i / sqrt(mean_i x_i^2 + eps) * gamma_i  (fp32; y = x without gamma);
 *   pair i < rot_dim / 2 is (y_i, y_(i + rot_dim / 2)), rotated by positions[axis_of_pair[i]][t] *
 *     base^(-2 i / rot_dim): (a, b) -> (a cos - b sin, b cos + a sin); elements from rot_dim on stay y;
 *   one bf16 rounding at the end.
 * Queries go to q_out [n_tokens][n_heads][head_dim]. Keys and the values (unchanged) go to slot slots[t]
 * of k_cache and v_cache; a token whose slot is negative or beyond the cache stores neither. The
 * non-negative slots of a call are distinct.
 * q, k, v: bf16, heads of a token contiguous, tokens q_stride, k_stride, v_stride elements apart (a
 * packed projection's row, or heads * head_dim), multiples of 8 and at least a token's elements.
 * gammas: fp32 [head_dim]. positions: int32 [n_axes][pos_stride], 1 <= n_axes <= 4. axis_of_pair: HOST memory,
 * uint8 [rot_dim / 2] with entries below n_axes, read during the call; NULL: axis 0 for every pair.
 * Angles are formed as two floats: the cosine and sine are within 1e-6 for |position| < 2^24, 1e-5 beyond, for base >= 1 (below,
 * pairs turn faster than one radian a position, and the bounds grow with that).
 * 1 <= n_tokens < 2^31; head_dim % 8 == 0, 8..256; rot_dim % 8 == 0, 0..head_dim; n_heads, n_kv_heads 1..4096;
 * base > 0, eps >= 0. Device pointers 16-byte aligned, but positions (4) and slots (8). No output may
 * overlap another buffer. Errors: EMB_EINVAL, EMB_EALIGN, EMB_ECUDA. */
EMB_API emb_status emb_qk_norm_rope(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                                    const uint16_t* v, int64_t v_stride, int64_t n_tokens, int64_t n_heads,
                                    int64_t n_kv_heads, int64_t head_dim, const float* q_gamma,
                                    const float* k_gamma, float eps, const int32_t* positions,
                                    int64_t pos_stride, int64_t n_axes, const uint8_t* axis_of_pair,
                                    int64_t rot_dim, float base, const int64_t* slots, uint16_t* q_out,
                                    uint16_t* k_cache, uint16_t* v_cache, int64_t n_pages, int64_t page_size,
                                    emb_stream_t stream);

/* Bytes of workspace that emb_paged_attention needs, whatever the call. */
#define EMB_PAGED_WORKSPACE ((size_t)64 << 20)

/* Section 3.1 ("prefix once, head many": new tokens attend to what the cache holds) and Section 3.2 (the
 * shared backbone layer).
 * Scaled dot-product attention (Vaswani et al., 2017) of the new tokens of n_req requests over their
 * cached tokens, their own included (stored before this call). Request r has the queries
 * q_start[r] .. q_start[r + 1) of Q and n = kv_len[r] keys; its last query sits at position n - 1, so query i of
 * m at p = n - m + i. With f = prefix[r] (0 where prefix is NULL), it sees the keys j in [lo, hi):
 *   hi = min(n, max(p + 1, f)): causal, but the first f tokens are visible to every query
 *     (f >= n: no mask);   lo = max(0, p - window + 1) if window > 0, else 0.
 *   s_j = scale * q.k_j;  with cap > 0, s_j = cap * tanh(scale * q.k_j / cap);
 *   O[t][h] = sum_j softmax_j(s_j) v_j, fp32 sums, one bf16 rounding; zeros for a query that sees no key.
 * Query head h reads key/value head h / (n_heads / n_kv_heads). Keys and values outside a query's range have
 * no part in its output, whatever they hold (NaN included). A visible key whose score is NaN or +infinity
 * makes its queries' outputs NaN; a score of -infinity has weight zero; a visible value that is not finite makes
 * that element of its queries' outputs infinite or NaN. The scores are held in base 2 (scale *
 * log2(e) rounded to fp32 once; capped ones within a relative 2^-20, with caps of up to 64 within 2^-22 of the cap), the weights by the hardware's power of two (relative error about 2^-22; below 2^-126 of
 * the largest they are zero). Up to 16 query rows (max_q queries times heads per key/value head), the
 * weights enter the value product as bf16 hi + lo (2^-16); above, they may be rounded once to bf16 (2^-9 each).
 * kv_len above max_pages * page_size counts as that; q_start past n_tokens as n_tokens, and a decreasing
 * q_start as no queries (rows of O that more than one request then claims, or a request and the padding, hold what any of
 * them gives; if the requests claim more queries than n_tokens in all, the rows of all are undefined); a page id outside [0, n_pages) as a page of zeros. Rows of O from q_start[n_req] to
 * n_tokens (padding) are zeroed.
 * Q, O: bf16 [n_tokens][n_heads][head_dim]; k_cache, v_cache as above, 16-byte aligned; table: int32
 * [n_req][max_pages]; q_start: int32 [n_req + 1], starting at 0; kv_len, prefix: int32 [n_req]. max_q: the most queries
 * that a request of the call has, as far as the host knows; it picks the kernel, any value >= 1 is right.
 * head_dim 64, 128 or 256, page_size 16, 32, 64, 128 or 256, n_heads / n_kv_heads at most 64 (else
 * EMB_EUNSUPPORTED). 1 <= n_req <= 65536; 1 <= n_tokens < 2^31; n_heads <= 4096; scale and cap finite, cap >= 0; window >= 0;
 * max_pages * page_size <= 2^31 - 512. A call whose key tiles could number 2^31 is EMB_EUNSUPPORTED.
 * workspace: EMB_PAGED_WORKSPACE bytes (EMB_ENOSPC if ws_bytes says less), 256-byte aligned, zero-filled before its
 * first use; a call leaves it ready for the next one unless emb_paged_status reports EMB_ETIMEOUT: then zero
 * its first 4 KB again. One workspace serves one stream at a time; calls on other streams with a workspace of their own may
 * run beside it (calls whose CTAs wait for one another are cooperative launches). Results are bitwise reproducible for
 * the same lengths. No output may overlap another buffer.
 * Errors: EMB_EINVAL, EMB_EALIGN, EMB_ENOSPC, EMB_EUNSUPPORTED, EMB_ECUDA. */
EMB_API emb_status emb_paged_attention(const uint16_t* Q, const uint16_t* k_cache, const uint16_t* v_cache,
                                       int64_t n_pages, int64_t page_size, const int32_t* table,
                                       int64_t max_pages, const int32_t* q_start, const int32_t* kv_len,
                                       const int32_t* prefix, int64_t n_req, int64_t n_tokens, int64_t max_q,
                                       uint16_t* O, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                       float scale, float cap, int64_t window, void* workspace,
                                       size_t ws_bytes, emb_stream_t stream);

/* Section 3.2 (the deployment boundary reports device-side failures to the host).
 * As emb_device_status, for the waits of this library's kernels: reads and clears its status word on
 * `stream`, then synchronises `stream`. EMB_OK, or EMB_ETIMEOUT if a bounded wait expired since the last call
 * (the outputs of the calls since then are undefined). */
EMB_API emb_status emb_paged_status(emb_stream_t stream);

/* Section 3.2 (deployment boundary; test support for the failure path above).
 * One CTA publishes its part of a shared item in a ready workspace of emb_paged_attention and waits for another's, which
 * never comes, giving up after timeout_ns nanoseconds (1e3 .. 1e9): emb_paged_status then returns EMB_ETIMEOUT, and the
 * workspace's first 4 KB are to be zeroed. Errors: EMB_EINVAL, EMB_EALIGN, EMB_ENOSPC, EMB_ECUDA. */
EMB_API emb_status emb_paged_selftest_wait_timeout(void* workspace, size_t ws_bytes, int64_t timeout_ns, emb_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* EMB_PAGED_H */
