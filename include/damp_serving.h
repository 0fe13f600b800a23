/*
 * damp_serving.h - the operators of libdamp that a server of recurrent-state
 * models needs around the state update of damp.h: linear attention with one
 * decay a head (prompts and single tokens), the verification of drafted
 * tokens, and the slots of a state pool as the pages of its cache.
 *
 * The conventions are those of damp.h: device pointers unless the comment
 * says "host", caller-owned memory, calls that only enqueue work on `stream`,
 * arguments checked on the host before anything is enqueued, statuses and
 * damp_last_error(). Nothing here allocates memory or synchronises (but for
 * the debugging aid DAMP_CHECK_SLOTS, as in damp.h), so every call can be
 * captured into a graph. Values that live on the device (slot ids, lengths,
 * tokens) are bounded by the kernels: no value makes a call touch memory
 * outside the arrays that it was given.
 *
 * How they go together: a recurrent state cannot be rolled back, so a
 * request that speculates drafts on a copy (damp_slots_fork, or the first
 * drafted step from one slot into another), the target reads its outputs for
 * all drafted tokens without keeping a state (damp_linear_prefill with
 * slot_out = DAMP_SLOT_ZERO), damp_verify_drafts counts the tokens that
 * stand, and damp_linear_prefill runs over those again with the counts,
 * still on the device, as its lengths.
 */
#ifndef DAMP_SERVING_H
#define DAMP_SERVING_H

#include "damp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Linear attention with one decay a head.
 *
 * Per value head h (key head hk = h / (HV / num_k_heads)), S its d_k x d_v
 * state in fp32:
 *   S_t = exp(g_t) S_{t-1} + k_t v_t^T
 *   o_t = scale * S_t^T q_t            (from the updated state)
 * with g_t one fp32 number per token and head (a log-decay; 0 keeps the
 * state, -inf forgets it, up to 88, whose factor fp32 just holds, grows it).
 * Over any number of tokens that grow, results are the recurrence's as long as
 * its own states and outputs stay in fp32 (prompts: states, |v_t| and
 * |q_t . k_j| below 2^111). The states live in a DAMP_STATE_FP32 pool with
 * d_k and d_v multiples of 8 up to 256, not necessarily equal. Other pools
 * return DAMP_ERR_UNSUPPORTED.
 *
 * Slots: request b starts from slot_in[b] and leaves its state in
 * slot_out[b].
 *  - slot_in[b] in [0, num_slots): that state. DAMP_SLOT_ZERO: the zero
 *    state (a new request; nothing is read). Any other value: a padded
 *    request, whose outputs are written as zeros and whose state is not.
 *  - slot_out[b] in [0, num_slots): the state after the last token is
 *    written there. Any other value: it is not kept.
 *  - slot_out = NULL means slot_out = slot_in. slot_in may repeat (several
 *    requests continuing one prompt); slot_out must not, and a slot that one
 *    request writes must not be read by another.
 *
 * Operands: q, k bf16 [tokens, num_k_heads, d_k] and v bf16 [tokens, HV, d_v],
 * heads contiguous, 16-byte aligned, with the given distance between tokens
 * in elements (a multiple of 8, at least one token's heads; so they may be
 * left where a fused projection wrote them). g fp32 [tokens, HV] with the
 * token distance g_stride >= HV, or g_stride = 0 for one decay a head.
 * Operands and states must be finite (g may be -inf): a NaN or an infinity
 * may reach any output of its own request, those of earlier tokens included,
 * and its state; it reaches no other request, and what lies outside the
 * requests' tokens is not read.
 * States, and outputs in fp32, are good to fp32. For outputs in bf16 a prompt's
 * fp32 intermediates (the state, the decayed scores and values) enter the
 * products with 16 bits: an output may be off by 2^-15 of the sum of its terms'
 * absolute values, beside its own rounding of up to 2^-8. That shows where the
 * terms nearly cancel; callers who need those outputs take o in fp32.
 * o [tokens, HV, d_v] contiguous in o_dtype (DAMP_DT_FP32 or DAMP_DT_BF16),
 * 16-byte aligned.
 * ---------------------------------------------------------------------- */

#define DAMP_SLOT_ZERO (-1)

/* One token for each of B requests (token b belongs to request b). B = 0 is
 * a no-op; B <= 65535. */
damp_status damp_linear_update(const damp_pool* pool, int32_t layer,
                               const int32_t* slot_in, const int32_t* slot_out,
                               int32_t B, int32_t num_k_heads, const uint16_t* q,
                               int64_t q_stride, const uint16_t* k,
                               int64_t k_stride, const uint16_t* v,
                               int64_t v_stride, const float* g,
                               int64_t g_stride, float scale, void* o,
                               int32_t o_dtype, void* stream);

/* Scratch of damp_linear_prefill for B requests of at most max_len tokens
 * (0 where it needs none, and for invalid arguments). Its contents matter
 * only during a call. More or longer requests may need less, since fewer
 * pieces of them fill the device: ask for each call's B and max_len. */
size_t damp_linear_prefill_workspace_bytes(const damp_pool* pool, int32_t B,
                                           int32_t max_len);

/* Prompts of B requests, packed along one token axis of n_tokens: request b
 * has the tokens seq_start[b] .. seq_start[b] + seq_len[b] - 1 (int32, device).
 * Requests need not be adjacent or in order, and must not overlap; what lies
 * between them is neither read nor written. A request of length 0 has no
 * outputs; its state still goes from slot_in to slot_out.
 *  max_len    host: no seq_len exceeds it (0 <= max_len <= n_tokens). A
 *             request is cut to max_len tokens and to the end of the token
 *             axis; one that starts outside [0, n_tokens] has length 0.
 *  workspace  damp_linear_prefill_workspace_bytes(pool, B, max_len) bytes,
 *             16-byte aligned (NULL where that is 0). Calls that may overlap
 *             need one each.
 * B = 0 is a no-op; B <= 65535; n_tokens < 2^31; token distances of at most
 * 2^24 - 16 (of g, 2^23 - 8) and HV d_v of at most 2^23 - 8 elements. */
damp_status damp_linear_prefill(const damp_pool* pool, int32_t layer,
                                const int32_t* slot_in, const int32_t* slot_out,
                                int32_t B, int64_t n_tokens, int32_t max_len,
                                const int32_t* seq_start, const int32_t* seq_len,
                                int32_t num_k_heads, const uint16_t* q,
                                int64_t q_stride, const uint16_t* k,
                                int64_t k_stride, const uint16_t* v,
                                int64_t v_stride, const float* g,
                                int64_t g_stride, float scale, void* o,
                                int32_t o_dtype, void* workspace,
                                size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Verification of drafted tokens.
 *
 * Request b drafted n_b = lens[b] tokens x_0 .. x_{n_b - 1}, each drawn from
 * its draft's distribution q_i; p_i are the target's distributions, p_{n_b}
 * the one after the last draft. With given uniform numbers u_0 .. u_K in [0, 1):
 *   draft i stands iff all before it do and u_i q_i(x_i) < p_i(x_i);
 *   a = the number of drafts that stand;
 *   next token ~ max(p_a - q_a, 0), normalised, if a < n_b, else ~ p_{n_b},
 *   drawn by u_K, which judges no draft (a number that refused one is not
 *   uniform any more),
 * which together distribute the tokens as the target does.
 *
 * Everything is decided in exact arithmetic, so results do not depend on an
 * order of summation: the product above is not rounded, and the next token is
 * the least x whose cumulative weight w(0) + .. + w(x) exceeds
 * floor(W floor(2^24 u_K) / 2^24), W the sum of all weights, with
 *   fix(y) = floor(2^40 min(max(y, 0), 1)), fix(NaN) = 0,
 *   w(x) = max(fix(p_a(x)) - fix(q_a(x)), 0) or fix(p_a(x)).
 * The distributions need not be normalised. If no token has weight the next
 * token is -1. A drafted token outside [0, V) never stands. u is cut to
 * [0, 1 - 2^-24]; NaN counts as 0.
 * ---------------------------------------------------------------------- */

/* Scratch of damp_verify_drafts (0 for invalid sizes). */
size_t damp_verify_workspace_bytes(int32_t B, int32_t V);

/*  p          [B, K + 1, V] in dtype (DAMP_DT_FP32 or DAMP_DT_BF16).
 *  q          [B, K, V] in dtype.
 *  tokens     int32 [B, K]: the drafted tokens.
 *  lens       int32 [B], cut to [0, K]; NULL = K for every request.
 *  u          fp32 [B, K + 1]; u[b, K] draws the next token.
 *  accepted   int32 [B]: a.
 *  out        int32 [B, K + 1]: the drafts that stand, the next token, then -1.
 *  workspace  damp_verify_workspace_bytes(B, V) bytes (or more), 16-byte
 *             aligned, its first 2^18 bytes zero before its first call; every
 *             call leaves those zero again, so that a workspace serves call
 *             after call, of any sizes that it has room for. Calls that may
 *             overlap need one each.
 * K = 0 draws one token from p (q and tokens are not used). B = 0 is a no-op;
 * B <= 65535, 0 <= K <= 1024, 1 <= V <= 2^22. */
damp_status damp_verify_drafts(const void* p, const void* q, int32_t dtype,
                               const int32_t* tokens, const int32_t* lens,
                               const float* u, int32_t B, int32_t K, int32_t V,
                               int32_t* accepted, int32_t* out, void* workspace,
                               size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Slots as pages of the state cache, in any pool (every layout).
 *
 * refs is an int32 [num_slots] device array of the caller's: how many hold a
 * slot (0 = free). Calls on one array must not overlap.
 * ---------------------------------------------------------------------- */

/* Takes the n lowest free slots in ascending order: out[i] (int32 [n]) is
 * the slot and its count becomes 1; -1 where no slot is left. (To the linear
 * calls -1 is DAMP_SLOT_ZERO: a caller that does not know that n slots are free
 * has to look before it passes the ids on.) */
damp_status damp_slots_alloc(int32_t* refs, int32_t num_slots, int32_t* out,
                             int32_t n, void* stream);

/* Adds one holder to (retain) or takes one from (release) each of the n named
 * slots; a slot named twice counts twice, entries outside [0, num_slots) are
 * skipped, and counts do not fall below 0. Retaining a free slot takes it. */
damp_status damp_slots_retain(int32_t* refs, int32_t num_slots,
                              const int32_t* slots, int32_t n, void* stream);
damp_status damp_slots_release(int32_t* refs, int32_t num_slots,
                               const int32_t* slots, int32_t n, void* stream);

/* Copies the states of slot src[i] into the slots dst[i * fan + j], j < fan
 * (int32 [n] and [n, fan]); `layer` selects one layer, or -1 for all. Each
 * source is read once. Entries outside [0, num_slots) are skipped, so fans
 * may be ragged. A slot may occur once among all of dst and not in src; src
 * may repeat. */
damp_status damp_slots_fork(const damp_pool* pool, int32_t layer,
                            const int32_t* src, const int32_t* dst, int32_t n,
                            int32_t fan, void* stream);

/* Scratch of damp_slots_compact (0 for an invalid pool). */
size_t damp_slots_compact_workspace_bytes(const damp_pool* pool);

/* Moves the live slots (refs > 0), L in number, of every layer into the slots
 * 0 .. L - 1 with the fewest copies: a live slot below L stays, and the i-th
 * live slot from L on (ascending) moves into the i-th free one below L.
 *  refs       counts, in and out: they move with their slots.
 *  map        int32 [num_slots]: where each slot's state is now, -1 for a
 *             free one.
 *  live       int32 [1]: L.
 *  workspace  damp_slots_compact_workspace_bytes(pool) bytes, 16-byte
 *             aligned; its contents matter only during the call. */
damp_status damp_slots_compact(const damp_pool* pool, int32_t* refs,
                               int32_t* map, int32_t* live, void* workspace,
                               size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DAMP_SERVING_H */
