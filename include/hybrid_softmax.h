/*
 * hybrid_softmax.h -- C ABI of the softmax layers of a hybrid model (sm_103a).
 *
 * A model retrofitted with block-hybrid attention keeps most of its layers on
 * exact attention over a paged key-value cache: in a denoising step such a
 * layer normalises and rotates the queries and keys of the active block, writes
 * the block's keys and values into the cache, and attends to the whole prefix
 * plus the block, without a mask inside the block.  The entry points here carry
 * those layers beside the block-hybrid ones of hybrid.h, and keep its
 * conventions: the caller owns every buffer, nothing is allocated, every call is
 * asynchronous on its stream, argument checks run on the host
 * (HYBRID_ERR_INVALID_ARG, HYBRID_ERR_UNSUPPORTED), and what only the device can
 * see (a page, slot, length or position out of range, a wait that gave up)
 * never traps: it sets a bit of the device error word, which hybrid_check()
 * reports (HYBRID_ERR_DEVICE, HYBRID_ERR_TIMEOUT).  Tensor pointers are
 * device pointers, 16-byte aligned (int and float arrays: 4-byte).
 *
 * Of hybrid_cfg they read head_dim d in {64, 128}, n_q_heads Hq and n_kv_heads
 * Hkv (1 <= Hkv <= Hq <= 256, Hq a multiple of Hkv; query head h reads key head
 * h / G, G = Hq / Hkv), io_dtype (float32 or bfloat16, the type of every tensor
 * below that has no type of its own) and, in hybrid_paged_attn, block_size B
 * (1 <= B <= 128 new tokens per request; 1 is plain decoding).  feat_dim is not
 * read.  All arithmetic is float32 with one rounding of each output to io_dtype
 * (bfloat16 attention: see hybrid_paged_attn).
 *
 * Paged cache (one K and one V array per layer, shared tables):
 *   K_cache, V_cache  [n_pages][Hkv][page_size][d]
 *   block_table       [n_req][max_pages] int: page of tokens j * page_size ...
 *   slot of a token   page * page_size + (position % page_size), an int
 * A page of one head is contiguous, so a page is read as one box per head.
 */
#ifndef HYBRID_SOFTMAX_H_
#define HYBRID_SOFTMAX_H_

#include "hybrid.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int page_size;   /* tokens per page: 16, 32, 64 or 128 */
    int n_pages;     /* pages of the pool; n_pages * page_size <= 2^31 - 1 */
    int max_pages;   /* entries per row of block_table (pages of the longest request);
                        max_pages * page_size <= 2^31 - 256 */
} hybrid_page_cfg;

/* ------------------------------------------------------------------------
 * Block tables and slot maps.
 *
 * The free pages form a ring: free_pages [n_pages] int, and a pair of ints
 * {head, count}: the free ones are free_pages[(head + i) % n_pages], i < count.
 * Calls read one pair and write another, so a call can be replayed.  No output may
 * share memory with an input or another output (HYBRID_ERR_INVALID_ARG). */

/* Room for n_new[r] >= 0 new tokens of each request, which has lens[r] already:
 * pages are taken from the ring's head, request by request in order, and
 *   block_table  the entries of the pages taken are written, others left alone
 *   slots        [n_slots] int: slots of the new tokens, packed by request;
 *                -1 beyond the last
 *   positions    [n_slots] int or null: lens[r] + 0, 1, ...; 0 beyond the last
 *   tok_offsets  [n_req + 1] int or null: request r's tokens are
 *                [tok_offsets[r], tok_offsets[r + 1]) of slots
 *   lens_out     [n_req] int: lens + n_new
 *   ring_out     the ring after the call
 * A request that cannot be served (a negative number, more than max_pages pages,
 * too few free pages, tokens beyond n_slots) is left as it is: its length stays,
 * its tokens get slot -1, and hybrid_check() reports HYBRID_ERR_DEVICE.  A request
 * that needs no new page is served whatever the pool holds.  n_req <= 65536. */
hybrid_status hybrid_page_append(const hybrid_page_cfg *pg, int n_req, const int *lens, const int *n_new,
                                 const int *free_pages, const int *ring_in, int *block_table, int *slots,
                                 int *positions, int n_slots, int *tok_offsets, int *lens_out, int *ring_out,
                                 cudaStream_t stream);

/* Give the pages of n_rows finished requests (rows [n_rows] of block_table, each
 * at most once) back to the ring's tail, in the order of rows and of their table
 * entries.  lens [n_req] are the requests' lengths; the caller sets those of the
 * released rows to 0 before the next append.  Entries are written into
 * free_pages in place, outside the live part of ring_in.  A row or length out of
 * range is skipped, a table entry out of range left out, and what would overfill the
 * ring dropped; all are reported by hybrid_check().  n_rows <= 65536. */
hybrid_status hybrid_page_release(const hybrid_page_cfg *pg, int n_req, const int *rows, int n_rows,
                                  const int *lens, const int *block_table, int *free_pages, const int *ring_in,
                                  int *ring_out, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * Norms of queries and keys for each head, and rotary positions, in one pass.
 *
 *   n = x / sqrt(mean(x^2) + eps) * w      (over the d features of a head; skipped
 *                                           where the weight is null)
 *   a pair (a, b) of the first rot_dim features of n, with angle t:
 *   (a cos t - b sin t, b cos t + a sin t) * scale
 * Pair i is features (2i, 2i+1) if interleaved, else (i, i + rot_dim/2); its angle
 * at position p is 2 pi p freqs[i] / 2^64.  freqs holds turns per position as
 * 64-bit binary fractions, so p * freqs[i] modulo 2^64 is the exact fraction of a
 * turn in wrapping integer arithmetic, for every position that an int holds. */
typedef struct {
    int rot_dim;       /* leading features rotated: a multiple of 16, 0 <= rot_dim <= d */
    int interleaved;   /* 0: pairs (i, i + rot_dim/2); 1: pairs (2i, 2i + 1) */
    float scale;       /* factor on cosine and sine */
    float eps;         /* added to the mean square */
} hybrid_rope_cfg;

typedef enum {
    HYBRID_ROPE_NONE = 0,     /* theta_i = base^(-2i / rot_dim) radians per position */
    HYBRID_ROPE_LINEAR = 1,   /* theta_i / factor (position interpolation) */
    HYBRID_ROPE_NTK = 2,      /* base * factor^(rot_dim / (rot_dim - 2)) in place of base */
    HYBRID_ROPE_YARN = 3      /* by parts: theta_i (1 - g) / factor + theta_i g, with
                                 g = clamp((r_i - beta_slow) / (beta_fast - beta_slow), 0, 1),
                                 r_i = orig_len theta_i / 2 pi; scale = 0.1 ln(factor) + 1.
                                 The ramp is linear in the turns r_i.  (A model whose ramp is
                                 linear in the pair's index i between the two bounds has other
                                 frequencies between them: it brings freqs of its own.) */
} hybrid_rope_kind;

typedef struct {
    int kind;          /* hybrid_rope_kind */
    double base;       /* > 1 */
    double factor;     /* >= 1: the context's extension */
    double orig_len;   /* > 0: the context before it (YaRN) */
    double beta_fast;  /* YaRN: pairs with more turns than this over orig_len keep their frequency */
    double beta_slow;  /* YaRN: pairs with fewer are interpolated; 0 <= beta_slow < beta_fast */
} hybrid_rope_scaling;

/* The rot_dim / 2 entries of freqs (HOST array; the caller copies it to the
 * device once) and the factor for hybrid_rope_cfg.scale.  Host-only. */
hybrid_status hybrid_rope_freqs(const hybrid_rope_scaling *sc, int rot_dim, unsigned long long *freqs,
                                float *scale);

/* Q [n_tok][Hq][d], K [n_tok][Hkv][d] with q_stride, k_stride elements between
 * tokens (slices of one projection's output; a multiple of 16 bytes, at least one
 * token's heads) -> Qo, Ko dense.
 *   wq, wk     [d] io_dtype, or null: no norm
 *   positions  [n_tok] int;  freqs [rot_dim / 2] (8-byte aligned); both unread,
 *              and may be null, when rot_dim is 0
 * Qo may be Q, and Ko K, where the input is dense; they must not overlap otherwise. */
hybrid_status hybrid_qk_norm_rope(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q,
                                  size_t q_stride, const void *K, size_t k_stride, int n_tok, const void *wq,
                                  const void *wk, const int *positions, const unsigned long long *freqs, void *Qo,
                                  void *Ko, cudaStream_t stream);

/* The same, with the keys and the values V [n_tok][Hkv][d] (v_stride) written to
 * slots[t] of the paged cache.  A negative slot writes nothing (padding); a slot
 * beyond the pool writes nothing and is reported by hybrid_check().  Slots that
 * are written must differ.  pg->max_pages is not read. */
hybrid_status hybrid_qk_norm_rope_cache(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope,
                                        const hybrid_page_cfg *pg, const void *Q, size_t q_stride, const void *K,
                                        size_t k_stride, const void *V, size_t v_stride, int n_tok, const void *wq,
                                        const void *wk, const int *positions, const unsigned long long *freqs,
                                        const int *slots, void *Qo, void *K_cache, void *V_cache,
                                        cudaStream_t stream);

/* Bytes of workspace of hybrid_qk_norm_rope_backward (partial sums of the weight
 * gradients); 0 for an unsupported cfg or n_tok < 0. */
size_t hybrid_qk_norm_rope_workspace_bytes(const hybrid_cfg *cfg, int n_tok);

/* Gradients of sum(dQo * Qo) + sum(dKo * Ko), from the inputs of the forward pass
 * and dQo, dKo (dense, io_dtype):
 *   dn = rotation by -t of dy, times scale;  u = w dn;  xh = x r
 *   dx = r (u - xh mean(u xh)),  dw = sum over tokens and heads of dn xh
 * dQ, dK are written with the strides of Q, K.  dwq, dwk [d] float32 are
 * overwritten; each is null exactly where its weight is.  Partial sums are added
 * in a fixed order: the same inputs give the same bits.  workspace: 16-byte
 * aligned, need not be initialised.  No output may overlap an input. */
hybrid_status hybrid_qk_norm_rope_backward(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q,
                                           size_t q_stride, const void *K, size_t k_stride, const void *dQo,
                                           const void *dKo, int n_tok, const void *wq, const void *wk,
                                           const int *positions, const unsigned long long *freqs, void *workspace,
                                           size_t workspace_bytes, void *dQ, void *dK, float *dwq, float *dwk,
                                           cudaStream_t stream);

/* ------------------------------------------------------------------------
 * Attention over the paged cache.
 *
 *   O[r][i][h] = sum_j p_j v_j,  p = softmax over the visible j of q . k_j / sqrt(d)
 * for the B = cfg->block_size queries of every request, Q and O [n_req][B][Hq][d]
 * dense.  kv_len [n_req] int counts the cached tokens, the active block's own
 * included (its keys and values are in the cache); every query of a request sees
 * the same keys j < kv_len, those with
 *     window == 0,  or  j >= kv_len - window,  or  j < n_sink.
 * (window >= 0 tokens up to the end of the context, and n_sink >= 0 first tokens that
 * stay visible; n_sink is ignored without a window.)  A request without a visible
 * key gets zeros.  What lies in the cache at other places (NaN included) has no
 * effect, and pages and table entries that hold no visible key are not read.
 * Infinities and NaN of visible keys and values give what the formula gives; a p_j
 * below 2^-126 of the largest may count as zero (and zero times infinity is NaN).
 * The work of all requests is cut evenly over the GPU whatever their lengths are;
 * parts of one request are joined in a fixed order, so the same inputs give the
 * same bits on every call.  bfloat16: products on the tensor cores with float32
 * accumulation, probabilities rounded to bfloat16 for the product with V (their
 * sum is taken in float32).
 * kv_len beyond max_pages * page_size (or negative) is clamped, and a page out of
 * range read as page 0; both are reported by hybrid_check(), the request's output
 * is then unspecified.
 *   workspace  16-byte aligned, >= hybrid_paged_attn_workspace_bytes; need not be
 *              initialised; calls that may overlap on the GPU need one each
 * n_req <= 65536, and n_req * (ceil(max_pages * page_size / 128) + 2) * Hkv * B *
 * ceil(Hq / (8 Hkv)) < 2^29 (HYBRID_ERR_UNSUPPORTED above a limit; with several rows to
 * a tile the second one lies higher). */
size_t hybrid_paged_attn_workspace_bytes(const hybrid_cfg *cfg, const hybrid_page_cfg *pg, int n_req);
hybrid_status hybrid_paged_attn(const hybrid_cfg *cfg, const hybrid_page_cfg *pg, const void *Q,
                                const void *K_cache, const void *V_cache, const int *block_table,
                                const int *kv_len, int n_req, int window, int n_sink, void *O, void *workspace,
                                size_t workspace_bytes, cudaStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HYBRID_SOFTMAX_H_ */
