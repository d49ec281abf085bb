/*
 * csbrnn_lm.h -- operators of recurrent language models beside the pruned products of csbrnn.h:
 * the gated delta rule (a recurrent cell whose state is a matrix), low-rank adapters of many
 * requests added to a shared projection's result, and the verification of drafted tokens.
 *
 * The conventions of csbrnn.h hold: int status codes, csb_last_error(), device pointers owned by
 * the caller (prefix d_), nothing allocated on the device, everything enqueued on `stream` (a
 * hipStream_t; NULL: the default stream) without host synchronisation, workspaces 256-byte
 * aligned with contents that need no initialisation.  The calls are kernel launches only: they may
 * be captured into a HIP graph and replayed with new contents in the captured buffers.
 * Offsets, lengths, slots and adapter numbers are device memory, so the host cannot check them:
 * the kernels do.  What lies outside its range reads and writes nothing out of bounds; what it
 * means is said at each operator.
 */
#ifndef CSBRNN_LM_H
#define CSBRNN_LM_H

#include "csbrnn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The gated delta rule.  Value head h has a state S of dk x dv numbers, a decay exp(g) and a step
 * beta per token, and reads key head h / (heads_v / heads_k).  Per token
 *     S <- exp(g) S;   u = beta (v - S^T k);   S <- S + k u^T;   o = scale S^T q.
 * Sequences are packed: sequence i has the tokens d_start[i] .. d_start[i + 1] - 1 of n_tokens
 * (d_start [n_seq + 1], ascending; NULL: n_seq sequences of n_tokens / n_seq tokens each), of which
 * the first d_len[i] are taken when d_len is given (at least 0; more than there are means all).
 * Element (token t, head, j) of q, k, v and out is at t * ld + head * width + j, g and beta of
 * (t, h) at t * ld + h; the leading dimensions leave the other operands of a fused projection in
 * place.  `type` is CSB_VAL_*; g, beta and states are binary32, and so is everything computed: the
 * state, all sums and the intermediate u have 24 bits, `out` is rounded once.
 * States: [n_states][heads_v][dk][dv].  Sequence i starts from state d_slot[i] of d_state_in and
 * leaves its last state in the same place of d_state_out (the same buffer or another that does not
 * overlap; NULL: not kept -- drafted tokens tried, and taken up later with d_len); d_slot NULL: state i.
 * d_state_in NULL, and a slot outside [0, n_states): starts from zeros; such a slot is not stored
 * either.  Two sequences of a call with one slot race.  A sequence of no tokens keeps its state.
 * Entries of `out` of tokens that no sequence takes are not written.  Offsets outside
 * [0, n_tokens] are taken as the nearer end.
 * Keys are expected at length one or less with beta in [0, 2], as layers of this kind make them:
 * longer ones let the state grow without bound, in the formula as here.  Infinite or NaN entries
 * of a token spread to the rest of its sequence and head, and nowhere else.  g = -infinity
 * forgets the state.
 */
typedef struct {
    int32_t type;                          /* CSB_VAL_*: q, k, v and out                     */
    int32_t heads_k, heads_v;              /* heads_v a multiple of heads_k                  */
    int32_t dk, dv;                        /* dk in [1, 256], dv >= 1                        */
    int32_t n_seq;
    int64_t n_tokens;
    const void *d_q, *d_k, *d_v;
    int64_t ldq, ldk, ldv;                 /* elements from one token to the next            */
    const float *d_g, *d_beta;
    int64_t ldg, ldbeta;
    const int32_t *d_start, *d_len;
    const float *d_state_in;
    float *d_state_out;
    const int32_t *d_slot;
    int32_t n_states;
    float scale;
    void *d_out;
    int64_t ldo;
} csb_delta_args;

/*
 * The rule token by token: one launch, every wavefront a part of a state's columns in registers.  For
 * the few tokens of a decoding step; right for any length.  Bitwise reproducible.
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range, heads_v
 * no multiple of heads_k, n_tokens no multiple of n_seq without d_start, an unknown type ->
 * CSB_EINVAL; dk > 256, n_tokens above 2^31 - 1, or more wavefronts than a launch takes (n_seq heads_v
 * ceil(dv / 32) of 2^24 and more) -> CSB_EUNSUPPORTED; launch failure -> CSB_EDEVICE.
 * n_seq = 0 does nothing.
 */
int csb_delta_recurrent(const csb_delta_args *args, void *stream);

/*
 * The same rule, the same arguments and errors, chunk by chunk: for prompts.  ldq, ldk, ldv or ldo of 2^23 or more,
 * dv above 2^20, or more workgroups than a launch takes (n_seq heads_v, rounded up to a multiple of 8, times ceil(dv / 16) of 2^22 and more;
 * (n_tokens / 64 + n_seq) ceil(heads_v / 4) of 2^24 and more) -> CSB_EUNSUPPORTED.
 * Faster than token by token from 16 to 32 tokens a sequence on; binary32 rows of dk above 128
 * and rows below 16 bytes are taken token by token here too.  A chunk of 64 tokens meets the state before its
 * decays: S^T k with the state before the chunk has to be a binary32 number.  Before a capture into a
 * graph call it once: a kernel's first launch raises its LDS limit.
 * d_ws: csb_delta_workspace_bytes(args) bytes (type, heads_*, dk, dv, n_seq and n_tokens are read; 0 for those
 * that the call refuses or takes token by token: d_ws may be NULL then).
 */
size_t csb_delta_workspace_bytes(const csb_delta_args *args);
int csb_delta_chunked(const csb_delta_args *args, void *d_ws, void *stream);

/*
 * Low-rank adapters of many requests, added to the result Y of a projection they share (the
 * layouts of csb_spmm*):   Y[:, n] += scale_a B_a (A_a X[:, n])   for every column n of a request
 * with adapter a.  X [cols][ldx] of `type` (entry (j, n) at d_X[j * ldx + n]), Y [rows][ldy]
 * binary32; d_A [n_adapters][rank][cols] and d_B [n_adapters][rows][rank] of `type`.
 * Request s has the columns d_start[s] .. d_start[s + 1] - 1 (d_start [n_seg + 1], ascending;
 * NULL: one column each, n_seg = batch) and adapter d_id[s]; a number outside [0, n_adapters): none,
 * its columns of Y stay as they are.  Adapter a uses its first d_rank[a] ranks (NULL: all;
 * values are taken into [0, rank]; what is stored past them is not used) and the factor d_scale[a]
 * (NULL: 1).  Columns that no request has stay as they are.  Offsets outside [0, batch] are taken as the nearer end.
 * Products of 16-bit numbers are exact in binary32 and A X is kept in binary32 on its way to B.
 * What is not finite in a column of X changes that column of Y only, and in a row of A or B the entries that it is a
 * factor of only; they are infinite or NaN (with a 16-bit type NaN where the formula has infinity).  Bitwise reproducible.
 * d_ws: csb_adapter_workspace_bytes(...) bytes.  Two launches.
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range,
 * n_seg != batch without d_start, an unknown type -> CSB_EINVAL; rank > 128, batch > 2^30, rows or cols above
 * 2^31 - 1, or more workgroups than a launch takes -> CSB_EUNSUPPORTED; launch failure ->
 * CSB_EDEVICE.  batch = 0 or n_seg = 0 does nothing.
 */
size_t csb_adapter_workspace_bytes(int64_t cols, int32_t batch, int32_t n_seg, int32_t rank);
int csb_adapter_add(int32_t type, const void *d_X, int64_t ldx, float *d_Y, int64_t ldy, int64_t rows,
                    int64_t cols, int32_t batch, const void *d_A, const void *d_B, int32_t n_adapters,
                    int32_t rank, const int32_t *d_rank, const float *d_scale, int32_t n_seg,
                    const int32_t *d_start, const int32_t *d_id, void *d_ws, void *stream);

/*
 * Verification of drafted tokens.  Request b brings d_count[b] drafts (NULL: n_draft; values are
 * taken into [0, n_draft]), tokens d_draft[b * n_draft + i].  Row (b, i) of the target's
 * probabilities is at d_p + (b * (n_draft + 1) + i) * ldp, that of the draft's at
 * d_q + (b * n_draft + i) * ldq, both of `type`; d_q NULL: drafts without probabilities (all of
 * the mass on the drafted token).  d_u [n_req][n_draft] and d_r [n_req]: numbers in [0, 1) given by the caller.
 * Draft x of row i is accepted if u q_i(x) < p_i(x) (the product rounded to binary32), up to
 * the first that is not; a token outside [0, vocab) is not accepted.  One more token then follows, from the
 * row where the drafts ended: with weights max(p - q, 0) if a draft was refused there, p if all
 * were accepted.  It is drawn by inversion, in whole numbers, so that it depends neither on the
 * order nor on the split of a sum: weight w counts floor(min(w, 1) 2^38) units (p - q rounded to
 * binary32; a NaN counts none), and the token is the lowest whose cumulated units exceed
 * floor(units of the row * floor(r 2^24) / 2^24).  Where no weight is left p's own units are
 * taken, and -1 is drawn where those are none either.
 * d_tokens [n_req][n_draft + 1] receives the accepted drafts, the drawn token and -1 behind it;
 * d_accepted [n_req] the number of accepted drafts.  d_ws: csb_verify_workspace_bytes(...) bytes.
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range, an
 * unknown type -> CSB_EINVAL; vocab > 2^24, n_req > 2^21, or more workgroups than a launch takes ->
 * CSB_EUNSUPPORTED; launch failure -> CSB_EDEVICE.  n_req = 0 does nothing; n_draft = 0 samples (d_q, d_draft and d_u may be NULL then).
 */
size_t csb_verify_workspace_bytes(int32_t n_req, int32_t vocab);
int csb_verify_drafts(int32_t type, const void *d_p, int64_t ldp, const void *d_q, int64_t ldq,
                      const int32_t *d_draft, const float *d_u, const float *d_r, const int32_t *d_count,
                      int32_t n_req, int32_t n_draft, int32_t vocab, int32_t *d_tokens, int32_t *d_accepted,
                      void *d_ws, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CSBRNN_LM_H */
