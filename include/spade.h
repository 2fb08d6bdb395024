/*
 * spade.h -- C ABI of the speculative-verify library for AMD Instinct MI355X
 * (gfx950).
 *
 * The library implements the cloud side of speculative decoding as SPADE
 * (arXiv 2608.13076) uses it: the verifier M_p scores d draft tokens in one
 * forward pass over d+1 positions (Algorithm 1, the "Cloud" step), accepts
 * the longest verified prefix, replaces the first rejected draft by a draw
 * from p'(x) = norm(max(0, p(x) - q(x))) (Sec. III-C, "Verification
 * criterion"), and updates the context (m <- m + k + 1).  The draft length d
 * is called gamma below.
 *
 * Conventions shared by every call
 * --------------------------------
 * - All device memory belongs to the caller: weights, workspace, KV cache,
 *   inputs and outputs.  The library never allocates or frees device memory;
 *   its handles own small host structures only.
 * - Pointers prefixed d_ are device pointers, h_ are host pointers.
 * - `stream` is a hipStream_t passed as void* (NULL = the null stream).  Every
 *   call that takes a stream is asynchronous and stream-ordered unless its
 *   comment says it synchronises.
 * - Calls return SPADE_OK or a negative spade_status and never throw.  On
 *   error nothing is launched and spade_last_error() holds a message (per
 *   thread).
 * - Token ids are int32 in [0, vocab).  Out-of-range ids found on the device
 *   are clamped and flagged in the device error word (spade_get_device_error).
 * - A model and the KV handles built on it must be used from one stream at a
 *   time: calls share the workspace.
 * - Schedule choices that do not change any result (tilings, k-splits,
 *   attention merge, correction slices) and the measurement hooks are
 *   declared in spade_tuning.h.
 */
#ifndef SPADE_H
#define SPADE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct spade_model_s* spade_model;
typedef struct spade_kv_s* spade_kv;

typedef enum {
  SPADE_OK = 0,
  SPADE_EINVAL = -1,       /* bad argument (null pointer, range, shape)        */
  SPADE_ECAPACITY = -2,    /* batch, gamma or KV capacity exceeded             */
  SPADE_EHIP = -3,         /* a HIP runtime call failed                        */
  SPADE_EUNSUPPORTED = -4, /* shape the kernels do not handle (see config)     */
  SPADE_EDEVICE = -5       /* device error word non-zero                       */
} spade_status;

enum { SPADE_GREEDY = 0, SPADE_SAMPLE = 1 };
enum { SPADE_F32 = 0, SPADE_BF16 = 1, SPADE_I4 = 2 /* kv_dtype only */ };

/* Bits of the device error word. */
enum {
  SPADE_DERR_TOKEN = 1u,    /* a token id was outside [0, vocab); clamped      */
  SPADE_DERR_NAN = 2u,      /* a logit was NaN                                  */
  SPADE_DERR_RESIDUAL = 4u, /* max(0, p - q) had no mass; drew from p instead   */
  SPADE_DERR_NOQ = 8u,      /* a sampling request got no draft_probs; greedy    */
  SPADE_DERR_CAPACITY = 16u, /* a request's length left fewer than gamma + 1 free
                                positions (lens written outside the library's
                                calls); clamped, that call's outputs are invalid */
  SPADE_DERR_COMMIT = 32u,  /* spade_kv_commit read an n_accepted outside
                               [0, gamma] of the last verify call; clamped      */
  SPADE_DERR_TREE = 64u     /* a parent was outside [-1, i); taken as -1        */
};

/* Weight tensors, row-major [out_features, in_features] unless noted. */
enum {
  SPADE_WQ = 0,     /* [d_model, d_model]                                  */
  SPADE_WK = 1,     /* [d_model, d_model]                                  */
  SPADE_WV = 2,     /* [d_model, d_model]                                  */
  SPADE_WO = 3,     /* [d_model, d_model]                                  */
  SPADE_WGATE = 4,  /* [d_ffn, d_model]                                    */
  SPADE_WUP = 5,    /* [d_ffn, d_model]                                    */
  SPADE_WDOWN = 6,  /* [d_model, d_ffn]                                    */
  SPADE_G_ATTN = 7, /* [d_model] float32 gain of the attention RMSNorm     */
  SPADE_G_FFN = 8,  /* [d_model] float32 gain of the feed-forward RMSNorm  */
  SPADE_EMBED = 9,  /* [vocab, d_model]                                    */
  SPADE_G_FINAL = 10, /* [d_model] float32 gain of the final RMSNorm       */
  SPADE_LM_HEAD = 11  /* [vocab, d_model]                                  */
};

/*
 * The verifier: a pre-RMSNorm decoder (Sec. III-A: embedding, L blocks
 * x_{l+1} = x_l + f_l(x_l) with f_l = attention then feed-forward, LM head,
 * softmax).  Attention is multi-head with rotary position embedding
 * (rotate-half pairing of feature i with i + head_dim/2, angle
 * pos * rope_theta^(-2i/head_dim)), grouped-query when n_kv_heads <
 * n_heads: query head h attends with K/V head h / (n_heads / n_kv_heads),
 * and Wk, Wv have n_kv_heads * head_dim rows; the feed-forward is SwiGLU
 * (silu(h W_gate^T) * (h W_up^T)) W_down^T; RMSNorm(x) = x / sqrt(mean(x^2)
 * + rms_eps) * g; no biases; the LM head is untied.
 *
 * weight_dtype: SPADE_BF16 or SPADE_F32 for every matrix (gains are float32).
 * kv_dtype: storage type of K and V (RoPE is applied before storing).
 * SPADE_I4 holds them in 4 bits, as spade_kvq_append does (below); prompts
 * then go through 16 rows per request and forward, a request's results depend
 * on the other requests of a call in their last bits, and the running weights
 * and eviction of spade_kv_track_weights and spade_kv_evict are available.
 * n_kv_heads: 0 (the default: n_heads) or a divisor of n_heads.
 * Supported: head_dim 64 or 128; d_model = n_heads * head_dim; d_model and
 * d_ffn multiples of 256 (bf16 weights) or 128 (f32); any vocab >= 2; at most
 * 15 drafts per request (gamma + 1 <= 16 rows).
 */
typedef struct {
  int32_t n_layers, d_model, n_heads, head_dim, d_ffn, vocab;
  int32_t weight_dtype, kv_dtype;
  float rms_eps, rope_theta;
  int32_t n_kv_heads;
} spade_config;

/* Bytes of the library's weight arena (its own tiled layout; filled by
 * spade_model_load_tensor).  0 if the config is unsupported. */
size_t spade_weight_bytes(const spade_config* cfg);

/* Bytes of the workspace for calls with up to max_batch requests of up to
 * max_gamma drafts each and caches of up to max_len positions.  With a bf16
 * cache and head_dim 128 its activation arrays also hold a prefill forward:
 * min(2048, max_batch * max_len rounded up to 16) rows (about 220 MB at the
 * 7B shape, 363 MB at the 33B shape). */
size_t spade_workspace_bytes(const spade_config* cfg, int max_batch, int max_gamma, int max_len);

/* Bytes of a KV cache holding max_batch requests of max_len positions.  With
 * S = max_len rounded up to a multiple of 256 and KVH the K/V heads, K and V
 * are each [n_layers][max_batch][KVH][S / 256] blocks of head_dim x 256
 * elements.  In a bf16 cache a block holds the B operands of the attention's
 * products in MFMA order, as 1 KB fragments.  K (S = Q K^T): fragments
 * [16][head_dim / 32], fragment (u, s) covering positions 16 u .. + 15 and
 * features 32 s .. + 31 of the block, its 16-byte piece 16 j + i holding
 * features 32 s + 8 j .. + 7 of position 16 u + i.  V (O = P V): fragments
 * [head_dim / 16][8], fragment (t, s) covering features 16 t .. + 15 and
 * positions 32 s .. + 31, its piece 16 j + i holding positions 32 s + 8 j .. + 7
 * of feature 16 t + i.  In a float32 cache a K block is [256][head_dim] (a row
 * per position) and a V block [head_dim][256].  So one wave's fragment load is
 * 1 KB contiguous and one 256-key chunk of K or V one contiguous block.
 * max_len <= 16384.  A 4-bit cache takes head_dim + 8 bytes per position and
 * K/V head (max_len rounded up to 32) and 4 per request. */
size_t spade_kv_bytes(const spade_config* cfg, int max_batch, int max_len);

/* Create a model over caller-owned device buffers: d_weights of
 * spade_weight_bytes() and d_workspace of spade_workspace_bytes() bytes
 * (256-byte aligned).  Synchronises once: writes the RoPE table and clears the
 * workspace's counters and error word on the current device. */
spade_status spade_model_create(const spade_config* cfg, void* d_weights, void* d_workspace,
                                int max_batch, int max_gamma, int max_len, spade_model* out);

/* Copy one tensor (kind = SPADE_WQ .. SPADE_LM_HEAD; layer ignored for the
 * three global tensors) from a row-major device buffer into the arena,
 * re-tiling matrices for the GEMM kernels.  d_src holds bf16 bits (uint16) or
 * float32 as weight_dtype says; gains are always float32.  The source may be
 * freed once the stream has passed this call. */
spade_status spade_model_load_tensor(spade_model m, int kind, int layer, const void* d_src, void* stream);

/* Wrap a caller-owned KV buffer of spade_kv_bytes(cfg, max_batch, max_len)
 * bytes plus device int32 arrays lens[max_batch] (cached positions per
 * request) and pending[max_batch] (the token whose row has not been computed
 * yet: the last prompt token, then each round's correction).  lens and
 * pending start at 0.  With kv_dtype SPADE_I4 it clears the evicted counts in
 * the buffer and synchronises. */
spade_status spade_kv_create(spade_model m, void* d_kv, int max_batch, int max_len,
                             int32_t* d_lens, int32_t* d_pending, spade_kv* out);

/* Set lens[0..B) and pending[0..B) from host arrays (a snapshot restore).  A
 * request set to length 0 starts over: its evicted positions no longer count.
 * Lengths from before a spade_kv_evict do not fit the rows that it moved. */
spade_status spade_kv_set_state(spade_kv kv, int B, const int32_t* h_lens,
                                const int32_t* h_pending, void* stream);

/* Read lens and pending to the host.  Synchronises the stream. */
spade_status spade_kv_get_state(spade_kv kv, int B, int32_t* h_lens, int32_t* h_pending, void* stream);

/* Snapshot lens/pending [B] into caller device buffers (device-to-device) and
 * remember the host-side capacity bound; spade_kv_restore copies them back and
 * restores that bound.  Rows past the restored lengths are stale and get
 * overwritten, so verify -> commit -> restore replays a round exactly.  Not
 * across a spade_kv_evict, which moves the rows, nor across a spade_kv_set_state
 * by which a request with evicted positions starts over (SPADE_EINVAL). */
spade_status spade_kv_snapshot(spade_kv kv, int B, int32_t* d_lens, int32_t* d_pending, void* stream);
spade_status spade_kv_restore(spade_kv kv, int B, const int32_t* d_lens, const int32_t* d_pending,
                              void* stream);

/* Prefill request b: run d_tokens[0 .. n_tokens-2] through the verifier,
 * appending their K/V at positions lens[b] .. lens[b] + n_tokens - 2, and make
 * d_tokens[n_tokens-1] the pending token (no logits are produced).  This is
 * the context y_{1:m} of Algorithm 1's input. */
spade_status spade_prefill(spade_model m, spade_kv kv, int b, const int32_t* d_tokens,
                           int n_tokens, void* stream);

/*
 * spade_verify -- one cloud verification of gamma drafts for B requests
 * (Algorithm 1, Cloud step; Sec. III-C).
 *
 * For request b the rows [pending_b, d_b,1 .. d_b,gamma] are appended at
 * positions lens[b] .. lens[b] + gamma and run through the verifier in one
 * pass; row i gives p_i = softmax(logits_i / T), the distribution of the token
 * after d_b,i (row gamma: after the last draft).  Then, left to right:
 *   greedy (mode SPADE_GREEDY): d_b,i+1 is accepted iff it is the argmax of
 *     row i (ties: lowest id);
 *   sampling (SPADE_SAMPLE): accepted iff u_b,i * q_b,i(d) < p_b,i(d), in
 *     float32, i.e. with probability min(1, p/q).
 * n_accepted[b] = k, the number accepted before the first rejection (0..gamma).
 * correction[b] = the token that follows the k accepted drafts:
 *   greedy: the argmax of row k;
 *   sampling, k < gamma: a draw from norm(max(0, p_k - q_k));
 *   sampling, k = gamma: a draw from p_gamma (no draft distribution there).
 * Draws use Gumbel-max, argmax_v (log w_v + G_v), with G_v = -log(-log U_v),
 * U_v = ((x_v >> 41) + 0.5) * 2^-23 and x_v output v (0-based) of a SplitMix64
 * stream seeded with the float32 bits of u_b,gamma.
 *
 * d_draft_tokens  int32 [B, gamma] (may be NULL when gamma == 0)
 * d_draft_probs   float32 [B, gamma, vocab] draft distributions q, already
 *                 tempered, used as given; may be NULL if no request samples
 *                 or gamma == 0 (a sampling request without q is verified
 *                 greedily and flags SPADE_DERR_NOQ)
 * d_uniforms      float32 [B, gamma + 1] in [0, 1); NULL if no request samples
 * d_mode          uint8 [B], SPADE_GREEDY or SPADE_SAMPLE
 * temperature     finite and > 0; applied to sampling requests (greedy ignores it)
 * d_n_accepted    int32 [B] out
 * d_correction    int32 [B] out
 * d_logits        float32 [B, gamma + 1, vocab] out (raw logits), or NULL
 *
 * The KV rows of all gamma+1 positions are written but lens is unchanged, so
 * the call can be repeated (idempotent) until spade_kv_commit.  Requires
 * lens[b] + gamma + 1 <= max_len, checked against the host-side upper bound
 * of lens (refreshed from the device, synchronising the stream, when the
 * bound alone fails), and B <= max_batch, gamma <= max_gamma.  A device
 * length the bound did not cover (lens written outside the library) is
 * clamped on the device and flagged SPADE_DERR_CAPACITY.
 * A captured call covers lens[b] + gamma + 1 up to the largest bound at the
 * capture, rounded up to whole chunks of 256 positions (bf16 cache of head_dim
 * 128) or 128 (others) and at most max_len; a longer request is clamped and
 * flagged likewise.
 */
spade_status spade_verify(spade_model m, spade_kv kv, int B, int gamma,
                          const int32_t* d_draft_tokens, const float* d_draft_probs,
                          const float* d_uniforms, const uint8_t* d_mode, float temperature,
                          int32_t* d_n_accepted, int32_t* d_correction, float* d_logits,
                          void* stream);

/* Prefill of B requests at once: request b caches h_n_tokens[b] - 1 prompt
 * tokens (row b of d_tokens, device int32 [B][ld], ld >= every count) after
 * its current length, and its last prompt token becomes pending -- the same
 * cache contents and state as spade_prefill of each request.  Each forward
 * takes rows from each of a range of consecutive requests (the GEMMs read
 * each weight once for all rows of the forward): with a bf16 cache and
 * head_dim 128 up to all of a request's prompt, within the workspace's
 * prefill rows (max_batch * max_len rounded up to 16, at most 2048, and at
 * least max_batch * 16); otherwise 16 per request.  A forward with bf16
 * weights too and more than 32 rows holds each request's own number of rows;
 * in others a request whose prompt runs out contributes placeholder rows,
 * written past its length and only where the cache has room.  Needs lens + h_n_tokens[b] <=
 * max_len (else SPADE_ECAPACITY; checked as by spade_verify, and so by
 * spade_prefill).  Counts are read from host memory
 * (h_n_tokens) before the call returns. */
spade_status spade_prefill_batch(spade_model m, spade_kv kv, int B, const int32_t* d_tokens, int ld,
                                 const int32_t* h_n_tokens, void* stream);

/* Probabilities softmax(logits / temperature) of `rows` rows of V logits,
 * float32, row-major [rows][V] in and out (device pointers, caller-owned; out
 * may be in itself, else must not overlap it).  The edge side of Algorithm 1 keeps, for every draft
 * token, the distribution q it was drawn from (Sec. III-C: the acceptance
 * test and the residual need q); with the draft model run through
 * spade_verify with gamma = 0, this turns that call's logits into q.
 * Stream-ordered; SPADE_EINVAL for null pointers, rows < 1, V < 2 or a
 * temperature that is not finite and > 0. */
spade_status spade_softmax(const float* d_logits, int rows, int V, float temperature, float* d_probs,
                           void* stream);

/* Context update after spade_verify (Algorithm 1: append the k accepted
 * tokens and the correction, m <- m + k + 1): lens[b] += n_accepted[b] + 1 and
 * pending[b] = correction[b] for b < B, on the device.  KV rows past the new
 * length are the rolled-back drafts; they are overwritten by the next round.
 * Needs a spade_verify on this cache since the last commit, prefill or state
 * change, covering at least B requests (else SPADE_EINVAL); each n_accepted is
 * clamped to [0, gamma] of that call (SPADE_DERR_COMMIT if it was outside).
 * The host-side upper bound of lens grows by gamma + 1; spade_verify reads the
 * device lengths back (one synchronisation) only when that bound would fail
 * its capacity check, so a long verify -> commit loop needs no host sync. */
spade_status spade_kv_commit(spade_kv kv, int B, const int32_t* d_n_accepted,
                             const int32_t* d_correction, void* stream);

/* Accept/reject and correction alone, from given logits (the last stage of
 * spade_verify).  d_logits float32 [B, gamma + 1, V]; other arguments as in
 * spade_verify.  Needs a model only for its workspace: V <= cfg.vocab. */
spade_status spade_accept_from_logits(spade_model m, int B, int gamma, int V, const float* d_logits,
                                      const int32_t* d_draft_tokens, const float* d_draft_probs,
                                      const float* d_uniforms, const uint8_t* d_mode,
                                      float temperature, int32_t* d_n_accepted,
                                      int32_t* d_correction, void* stream);

/* spade_accept_from_logits for callers that cannot allocate -- code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc --
 * and have no model: the same accept/reject and correction draw (the sliced
 * draw of a call that may sample) with the library's own static device
 * scratch (about 790 KB per device, held until the process ends) instead of
 * a model's workspace.  B <= 64 (else SPADE_ECAPACITY), gamma + 1 <= 16;
 * other arguments as in spade_accept_from_logits.  d_err: device uint32 the
 * call ORs the SPADE_DERR_* bits into (the caller clears it).  Calls no
 * allocating routine.  Calls on one device share its scratch: calls that
 * overlap on one device (different streams, no ordering) race. */
spade_status spade_accept_from_logits_noalloc(int B, int gamma, int V, const float* d_logits,
                                              const int32_t* d_draft_tokens, const float* d_draft_probs,
                                              const float* d_uniforms, const uint8_t* d_mode,
                                              float temperature, int32_t* d_n_accepted,
                                              int32_t* d_correction, uint32_t* d_err, void* stream);

/* Head norms of a model with 4-bit caches (SPADE_EUNSUPPORTED for others):
 * every query and key head is divided by its root mean square and multiplied
 * by its layer's gain before the rotation.  d_gain_q, d_gain_k: float32
 * [n_layers][head_dim], owned by the caller and read by every later call; both
 * NULL turns the norms off. */
spade_status spade_model_set_head_norms(spade_model m, const float* d_gain_q, const float* d_gain_k, float eps);

/* Running weights of a 4-bit cache (SPADE_EUNSUPPORTED for others): from now on
 * spade_verify and the prefill calls add the attention probability that every
 * cached position receives, summed over the query heads of its K/V head, to
 * d_weights, float32 [n_layers][max_batch][n_kv_heads][max_len], owned by the
 * caller (NULL: off).  Prompt rows all count (the last layer's too), of a
 * verify call the pending token's row, whose drafts may be rejected; a new
 * position starts at 0.  A repeated spade_verify adds its row again. */
spade_status spade_kv_track_weights(spade_kv kv, float* d_weights);

/* Keep, for every layer and K/V head of requests 0 .. B - 1 with more than
 * `budget` positions, the last `recent` and the budget - recent of the others
 * with the largest running weights (spade_kvq_evict, in place); lens[b] becomes
 * min(lens[b], budget).  Later rows keep counting their positions from the
 * start of the sequence, which may go on to the model's max_len: where it ends
 * before the cache is full, spade_verify and the prefill calls refuse too.  d_kept:
 * int32 [n_layers][max_batch][n_kv_heads][budget].  Rows of a verify call that
 * was not committed are lost.  A captured call counts once for the host's
 * bounds and snapshots, however often it is replayed. */
spade_status spade_kv_evict(spade_kv kv, int B, int budget, int recent, int32_t* d_kept, void* stream);

/*
 * K/V caches in 4 bits
 * --------------------
 * A cache of its own next to the model's: the attention state of a stack of
 * layers in a quarter of bfloat16's bytes, for a program that computes its
 * projections itself.  Every position and K/V head holds a key and a value of
 * head_dim features as codes n of 4 bits, with one scale s and one minimum m
 * (bfloat16) each:
 *   m = bf16(min_f x_f), s = bf16(max(max_f x_f - m, 0) * (1 / 15))  (in float32)
 *   n_f = clamp((x_f - m) / s to the nearest integer, ties to even, 0, 15)
 *   (0 where s = 0), and the cache stands for x_f ~ m + n_f s.
 * A row with a feature that is not finite, or whose m or max - m is not, is
 * held as NaN.  head_dim bytes and 8 more per position and K/V head (bfloat16
 * takes 4 head_dim).
 *
 * The calls share a shape, given by value of its fields at every call:
 *   n_layers, batch    layers and requests of the cache
 *   n_heads            query heads, a multiple of n_kv_heads (grouped-query:
 *                      query head h reads K/V head h / (n_heads / n_kv_heads))
 *   head_dim           64 or 128
 *   max_len            positions per request, at most 1048576
 * Layouts: a cache is n_layers x batch x n_kv_heads regions, whose inner order
 * is the library's; weights are float32 [n_layers][batch][n_kv_heads][max_len]
 * (the calls of one layer take that layer's part).  lens[b] counts the
 * positions request b holds: the calls read it, and only spade_kvq_evict
 * changes it (the caller adds the rows it keeps).  Requests are 0 .. B - 1.
 * Inputs of `dtype` SPADE_F32 or SPADE_BF16 are rows of contiguous heads, `ld`
 * elements from one row to the next (a multiple of 4), from addresses that
 * divide by 16 (SPADE_F32) or 8 (SPADE_BF16); other float arrays divide by 16.
 * Row i of request b is row b R + i.  d_rows: int32 [B], how many of its R
 * rows each request uses (clamped to [0, R]); NULL: all.  d_err: a device
 * uint32 that gets SPADE_DERR_CAPACITY ORed in where a length leaves the
 * range a call was given (nothing is read or written out of the cache then);
 * may be NULL.  All calls are asynchronous, allocate nothing and can be
 * captured.
 */
typedef struct {
  int32_t n_layers, batch, n_heads, n_kv_heads, head_dim, max_len;
} spade_kvq_shape;

/* Bytes of a cache (256-byte aligned; needs no initial contents). */
size_t spade_kvq_bytes(const spade_kvq_shape* shape);

/* Bytes of the workspace of spade_kvq_attend calls of up to max_rows rows (1
 * to 16) per request.  Calls that may overlap need a workspace each; it needs
 * no initial contents and keeps nothing between calls. */
size_t spade_kvq_workspace_bytes(const spade_kvq_shape* shape, int max_rows);

/* New rows of one layer: queries, keys and values as a projection leaves them.
 * Every query and key head is divided by its root mean square over head_dim
 * (x / sqrt(mean(x^2) + eps) * gain; d_gain_q / d_gain_k float32 [head_dim],
 * NULL: no norm), then rotated by its position as in the verifier (feature i
 * with i + head_dim / 2; d_rope float32 [rope_len][head_dim / 2][2], the cosine
 * and sine of every angle; NULL: no rotation).  Row i of request b is at
 * position (d_pos ? d_pos[b] : lens[b]) + i of the table (clamped to it,
 * flagged) and is stored as position lens[b] + i of the cache (dropped and
 * flagged at max_len and beyond).  Keys are normed and rotated in double and
 * rounded once to float32 before they are quantised, so their codes do not
 * depend on the order of a sum.  d_q NULL: no queries (d_q_out is not used);
 * else d_q_out gets the queries in `dtype` (it may be d_q itself with the same
 * distance of rows; any other overlap with d_q, d_k or d_v is refused), zeros
 * for rows that a request does not use.  d_weights (NULL: none): the new
 * positions' weights of this layer become 0.  R is any number of rows. */
spade_status spade_kvq_append(const spade_kvq_shape* shape, int layer, void* d_cache, int B, int R, int dtype,
                              const void* d_q, int64_t q_ld, const void* d_k, int64_t k_ld, const void* d_v,
                              int64_t v_ld, const float* d_gain_q, const float* d_gain_k, float eps,
                              const float* d_rope, int rope_len, const int32_t* d_pos, const int32_t* d_lens,
                              const int32_t* d_rows, void* d_q_out, int64_t q_out_ld, float* d_weights,
                              uint32_t* d_err, void* stream);

/* Causal attention of R rows per request (1 to 16) over one layer of the cache,
 * which already holds those rows at positions lens[b] .. lens[b] + R - 1
 * (spade_kvq_append): row i sees positions 0 .. lens[b] + i,
 *   out = softmax(scale q . k) v   per query head,
 * d_q and d_out [B R] rows of n_heads heads in `dtype` that do not overlap;
 * rows that a request does not use give zeros.  max_keys: the host's bound of
 * lens[b] + the rows in use, in [1, max_len] ([R, max_len] without d_rows), or
 * 0 for max_len.  A longer request is cut to it and flagged: its length, and of
 * more than max_keys rows those behind count as not in use.
 * d_weights_out (NULL: none): out = in + sum of the probabilities that the
 * first weight_rows rows in use of request b gave a position, over the query
 * heads of its K/V head, for the positions below lens[b] + rows; the others are
 * left as they were.  d_weights_in may be NULL (zeros) or d_weights_out.
 * Float32 calls keep their queries and the products of probabilities and
 * scales in 24 bits (three bfloat16 terms), bfloat16 calls those products in 16.
 * Sums and scores are float32, and the matrix instructions cut
 * the smaller of 32 products short: where no score scale q . k, nor its part scale
 * m sum_f q_f, exceeds 11 in size, outputs of float32 calls and probabilities
 * (also as weights) are good to 1e-6 of their size, beyond that to 1e-6 + 2^-22
 * of the largest.  Queries below 2^60 in size, values below 2^50 and spans max - m
 * of a value row above 2^-40 keep that precision; smaller spans lose bits, larger
 * numbers give infinities or NaN.  How the keys are divided among workgroups
 * follows the lengths of all requests, so the
 * last bits of a result do too; the same call gives the same bits.  scale: in
 * (0, 2^50]. */
spade_status spade_kvq_attend(const spade_kvq_shape* shape, int layer, const void* d_cache, int B, int R, int dtype,
                              const void* d_q, int64_t q_ld, float scale, const int32_t* d_lens,
                              const int32_t* d_rows, int max_keys, void* d_out, int64_t out_ld,
                              const float* d_weights_in, float* d_weights_out, int weight_rows, void* d_workspace,
                              size_t workspace_bytes, uint32_t* d_err, void* stream);

/* Rows of one layer as the values they stand for: positions start[b] + i (NULL:
 * i), i < R, as [B][R][n_kv_heads][head_dim] in `dtype`; zeros for rows past
 * d_rows[b] and for positions outside [0, max_len). */
spade_status spade_kvq_read(const spade_kvq_shape* shape, int layer, const void* d_cache, int B, int R,
                            const int32_t* d_start, const int32_t* d_rows, int dtype, void* d_k, void* d_v,
                            void* stream);

/* Eviction by accumulated attention weight.  Every (layer, request, K/V head)
 * of a request with more than `budget` positions keeps the last `recent` of
 * them and, of the others, the budget - recent with the largest weights (ties:
 * the lower position; NaN counts as larger than any number), closed up in
 * order; shorter requests keep all.  lens_out[b] = min(lens[b], budget).  The
 * positions' angles stay what they were, so later rows are appended with
 * d_pos counting the evicted positions too.
 * d_kept int32 [n_layers][batch][n_kv_heads][budget] gets the kept positions
 * of requests 0 .. B - 1, then -1.  The cache goes to d_cache_out of shape_out
 * (its batch >= B, its max_len >= budget, other fields equal), which is
 * another buffer, or d_cache itself with the same shape: then in place.
 * d_weights_out (NULL: none) gets the kept positions' weights, those behind
 * stay as they were; it may be d_weights if the shapes are the same.
 * d_lens_out may be d_lens.  0 <= recent <= budget, budget >= 1. */
spade_status spade_kvq_evict(const spade_kvq_shape* shape, const void* d_cache, const spade_kvq_shape* shape_out,
                             void* d_cache_out, int B, int budget, int recent, const float* d_weights,
                             float* d_weights_out, const int32_t* d_lens, int32_t* d_lens_out, int32_t* d_kept,
                             void* stream);

/*
 * Trees of drafts
 * ---------------
 * Verification of a tree instead of a chain, for a program that computes its
 * projections itself: R rows (nodes) per request, row i with a parent before it
 * (d_parents int32 [B][R], in [-1, i); -1: none; NULL: i - 1, a chain), row 0 the
 * root (the pending token).  The rows of a layer are appended to the cache behind
 * the lens[b] positions that it holds, attend to the context, to their ancestors
 * and to themselves, and a walk over the next tokens that the program has drawn
 * for every row (spade_sample) keeps the path that they follow.  So every kept
 * token is drawn from its own row's distribution, whatever the drafts are.
 *
 * The calls share a shape, given by value of its fields at every call:
 *   n_layers, batch    layers and requests of the cache
 *   n_heads            query heads, a multiple of n_kv_heads (grouped-query:
 *                      query head h reads K/V head h / (n_heads / n_kv_heads))
 *   head_dim           64 or 128
 *   max_len            positions per request, at most 1048576
 * A cache is laid out as a model's bfloat16 cache of these sizes (spade_kv_bytes),
 * so the buffer of one can be used: spade_prefill fills it.  Rows, their ld and
 * alignment, d_rows (int32 [B], rows in use, clamped to [0, R]; NULL: all) and
 * d_err as for spade_kvq_*; lens (int32 [B]) is changed by spade_tree_commit
 * alone.  All calls are asynchronous, allocate nothing and can be captured.
 */
typedef struct {
  int32_t n_layers, batch, n_heads, n_kv_heads, head_dim, max_len;
} spade_tree_shape;

/* Bytes of a cache (256-byte aligned; needs no initial contents). */
size_t spade_tree_bytes(const spade_tree_shape* shape);

/* Bytes of the workspace of spade_tree_attend calls of up to max_rows rows (1 to
 * 64) per request.  Calls that may overlap need a workspace each; it needs no
 * initial contents and keeps nothing between calls. */
size_t spade_tree_workspace_bytes(const spade_tree_shape* shape, int max_rows);

/* Rotation of queries and keys: the first rot_dim features of a head (a multiple
 * of 8, at most head_dim) are pairs j = 0 .. rot_dim / 2 - 1, features j and j +
 * rot_dim / 2, or 2 j and 2 j + 1 where interleaved is not 0.  At position p, pair
 * (x, y) becomes amplitude (x cos a - y sin a, y cos a + x sin a), a = p freq[j] in
 * double; the other features stay.  d_freq: device, float64 [rot_dim / 2], 8-byte
 * aligned (theta^(-2 j / rot_dim), or scaled for long contexts). */
typedef struct {
  const double* d_freq;
  int32_t rot_dim, interleaved;
  float amplitude;
} spade_rotary;

/* New rows of one layer: row i of request b is stored as position lens[b] + i of
 * the cache (dropped and flagged outside [0, max_len)), keys and values rounded
 * to bfloat16.  Queries and keys are rotated first (rotary NULL: not) by position
 * (d_pos ? d_pos[b] : lens[b]) + (d_depth ? d_depth[b R + i] : i): d_depth int32
 * [B][R], of a tree the number of ancestors.  d_q NULL: no queries (d_q_out is not
 * used); else d_q_out gets them in `dtype`, zeros for rows that a request does not
 * use (it may be d_q itself with the same distance of rows; any other overlap with
 * d_q, d_k or d_v is refused).  R is any number of rows. */
spade_status spade_tree_append(const spade_tree_shape* shape, int layer, void* d_cache, int B, int R, int dtype,
                               const void* d_q, int64_t q_ld, const void* d_k, int64_t k_ld, const void* d_v,
                               int64_t v_ld, const spade_rotary* rotary, const int32_t* d_pos, const int32_t* d_depth,
                               const int32_t* d_lens, const int32_t* d_rows, void* d_q_out, int64_t q_out_ld,
                               uint32_t* d_err, void* stream);

/* Attention of R rows per request (1 to 64) over one layer of the cache, which
 * already holds them at positions lens[b] .. lens[b] + R - 1: row i sees positions
 * 0 .. lens[b] - 1, its ancestors and itself,
 *   out = softmax(scale q . k) v   per query head.
 * d_q and d_out: [B R] rows of n_heads heads in `dtype` that do not overlap; rows
 * that a request does not use give zeros.  What a row does not see has no part in
 * its output, infinities and NaN among it; a value that is not finite makes its
 * feature of the rows that see it NaN or infinite, a key that is not finite their
 * scores.  (Sums can pass float32's range for values beyond 2^64.)  max_keys: the host's bound of lens[b] + the rows in use, in
 * [1, max_len] ([R, max_len] without d_rows), or 0 for max_len; a longer request is
 * cut to it and flagged, as by spade_kvq_attend.  scale: in [2^-50, 2^50].  Float32
 * calls keep queries and probabilities in 24 bits, bfloat16 calls the
 * probabilities in 16; scores and sums are float32.  How the keys are divided
 * among workgroups follows the lengths of all requests, so the last bits of a result
 * do too; the same call gives the same bits. */
spade_status spade_tree_attend(const spade_tree_shape* shape, int layer, const void* d_cache, int B, int R, int dtype,
                               const void* d_q, int64_t q_ld, float scale, const int32_t* d_parents,
                               const int32_t* d_lens, const int32_t* d_rows, int max_keys, void* d_out, int64_t out_ld,
                               void* d_workspace, size_t workspace_bytes, uint32_t* d_err, void* stream);

/* Rows of one layer: positions start[b] + i (NULL: i), i < R, as [B][R][n_kv_heads]
 * [head_dim] in `dtype`; zeros for rows past d_rows[b] and for positions outside
 * [0, max_len). */
spade_status spade_tree_read(const spade_tree_shape* shape, int layer, const void* d_cache, int B, int R,
                             const int32_t* d_start, const int32_t* d_rows, int dtype, void* d_k, void* d_v,
                             void* stream);

/* Keep the path that the drawn tokens follow, in all layers.  From row 0 on, the
 * walk goes to the lowest row i in use whose parent is the present row and whose
 * token d_tokens[b R + i] is d_next[b R + present], until there is none.
 *   n_accepted[b]  rows behind row 0 on the path (-1: the request uses no rows)
 *   path[b R + j]  the path's rows, 0 first; -1 behind the last
 *   correction[b]  d_next of the last of them: the new pending token (-1: no rows)
 * The path's rows become positions lens[b] .. lens[b] + n_accepted[b] of every
 * layer and head, lens_out[b] = lens[b] + n_accepted[b] + 1 (d_lens_out may be
 * d_lens).  The other rows are left where they were, as far as they are not
 * written over.  R: 1 to 64; all arrays int32. */
spade_status spade_tree_commit(const spade_tree_shape* shape, void* d_cache, int B, int R, const int32_t* d_tokens,
                               const int32_t* d_parents, const int32_t* d_next, const int32_t* d_rows,
                               const int32_t* d_lens, int32_t* d_lens_out, int32_t* d_n_accepted, int32_t* d_path,
                               int32_t* d_correction, uint32_t* d_err, void* stream);

/* Sampling
 * --------
 * One token per row of logits, and the distribution it was drawn from.  With l a
 * token's logit, T its row's temperature and d = (max l - l) / T in double, weight
 * exp(-d), the tokens in the order of their logits (equal ones by id) are kept
 * while
 *   d <= 32;
 *   the token is among the first top_k of those (top_k <= 0: no limit);
 *   the weight before it is below (top_p - 2^-40) of theirs (top_p >= 1: no limit;
 *     the first token always stays);
 *   exp(-d) >= min(min_p, 1).
 * Weights are good to 2^-34 of them: where the weight before a token is nearer than
 * that to what top_p allows, the token may be kept or not.  Equal logits have equal
 * weights, which add up without rounding: the 2^-40 is for those.
 * The token is argmax (-d + G) over the kept ones (ties: the lowest id), G_v the
 * noise of spade_verify's draws, seeded with the bits of the row's uniform; its
 * probability among them goes to d_chosen, all of them (0 for the others) to
 * d_probs.  T not above 0: the largest logit (ties: the lowest id), probability 1.
 * A NaN logit counts as -infinity and is flagged (SPADE_DERR_NAN), +infinity as the
 * largest finite number; of a row without a logit above -infinity (flagged too) the
 * token is 0, all probabilities are 0. */
typedef struct {
  float temperature;
  int32_t top_k;
  float top_p, min_p;
} spade_sampling;

/* Bytes of the workspace of spade_sample calls of up to `rows` rows of V tokens
 * (0: refused).  Calls that may overlap need a workspace each; it needs no initial
 * contents and keeps nothing between calls. */
size_t spade_sample_workspace_bytes(int rows, int V);

/* d_logits: [rows] of V numbers of `dtype` (SPADE_F32 or SPADE_BF16), ld elements
 * from one row to the next.  Request r has rows r rows_per_request .. ; its values
 * are those of d_temperature, d_top_k, d_top_p and d_min_p ([requests] on the
 * device; the last request may have fewer rows), where one is NULL the one in
 * `all` (NULL: 1, 0, 1, 0).  d_uniforms float32 [rows]; d_tokens int32 [rows];
 * d_chosen float32 [rows] or NULL; d_probs float32 [rows][V] or NULL (it may be
 * float32 logits with ld = V; any other overlap is refused).  2 <= V <= 1048576.
 * Asynchronous, allocates nothing, can be captured; the same call gives the same
 * bits. */
spade_status spade_sample(int rows, int V, int dtype, const void* d_logits, int64_t ld, int rows_per_request,
                          const spade_sampling* all, const float* d_temperature, const int32_t* d_top_k,
                          const float* d_top_p, const float* d_min_p, const float* d_uniforms, int32_t* d_tokens,
                          float* d_chosen, float* d_probs, void* d_workspace, size_t workspace_bytes,
                          uint32_t* d_err, void* stream);

/* Read and clear the device error word.  Synchronises the stream. */
spade_status spade_get_device_error(spade_model m, uint32_t* h_flags, void* stream);

/* Message of the last failed call on this thread ("" if none). */
const char* spade_last_error(void);

void spade_model_destroy(spade_model m);
void spade_kv_destroy(spade_kv kv);

#ifdef __cplusplus
}
#endif

#endif /* SPADE_H */
