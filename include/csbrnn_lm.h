/*
 * csbrnn_lm.h -- operators of recurrent language models beside the pruned products of csbrnn.h:
 * the gated delta rule (a recurrent cell whose state is a matrix), the selective state space scan and the
 * short convolution in front of it, norms around a block, low-rank adapters of many requests added to a shared
 * projection's result, the verification of drafted tokens and the sampling of tokens from logits.
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

/*
 * The short causal convolution of a recurrent layer, channel by channel:
 *     out[t, c] = act(bias[c] + sum_{j < width} w[c][j] x[t - (width - 1) + j, c]),
 * act(v) = v / (1 + e^-v) with `silu`, else v.  Sequences (d_start, d_len, n_seq, n_tokens), slots and what happens to entries outside
 * of them are as with the delta rule.  Element (t, c) of x and out is at t * ld + c, both of `type` (CSB_VAL_*); w [channels][width] and
 * bias [channels] (NULL: zero) are binary32, sums too; `out` is rounded once and must not overlap x.
 * States hold the width - 1 inputs before a sequence's first token, oldest first, as they are:
 * [n_states][width - 1][channels] of `type`.  Sequence i starts from state d_slot[i] of d_state_in (d_slot NULL: state i; d_state_in NULL or
 * a slot outside [0, n_states): zeros) and leaves its last width - 1 inputs in the same place of d_state_out (the same buffer or
 * another that does not overlap; NULL: not kept).  With width 1 states have no entries, and are neither read nor written.
 * What is not finite in x or a state stays in its channel, in the width outputs that it is a factor of.
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range, out = x, n_tokens no multiple of n_seq
 * without d_start, an unknown type -> CSB_EINVAL; width > 8, n_tokens above 2^31 - 1, or more workgroups than a launch takes ->
 * CSB_EUNSUPPORTED; launch failure -> CSB_EDEVICE.  n_seq = 0 does nothing.  Bitwise reproducible, one launch.
 */
typedef struct {
    int32_t type;                          /* CSB_VAL_*: x, out and the states               */
    int32_t channels, width;               /* width in [1, 8]                                */
    int32_t silu;
    int32_t n_seq;
    int32_t n_states;
    int64_t n_tokens;
    const void *d_x;
    int64_t ldx;                           /* elements from one token to the next            */
    const float *d_w, *d_bias;
    const int32_t *d_start, *d_len;
    const void *d_state_in;
    void *d_state_out;
    const int32_t *d_slot;
    void *d_out;
    int64_t ldo;
} csb_conv_args;

int csb_short_conv(const csb_conv_args *args, void *stream);

/*
 * The selective state space scan.  Channel c has a state h of n numbers, decays A[c][0 .. n) (below zero in layers of this kind) and reads
 * B and C of group c / (channels / groups).  Per token, with s = dt[t, c] + dt_bias[c], or ln(1 + e^s) in its place with `softplus`:
 *     h[j] <- exp(s A[c][j]) h[j] + s x[t, c] B[t, group, j];   y = sum_j C[t, group, j] h[j] + D[c] x[t, c];
 *     out[t, c] = y, or y z[t, c] / (1 + e^-z[t, c]) where d_z is given.
 * Element (t, c) of x, dt, z and out is at t * ld + c, (t, group, j) of B and C at t * ld + group * n + j, all of `type`; A [channels][n],
 * D and dt_bias [channels] (NULL: zeros) and states are binary32, and so is everything computed; `out` is rounded once.  A step through softplus is off by 12 units of 2^-24 of
 * itself (with 16-bit operands by 1.25 |dt + dt_bias| more below zero), which states keep.  `out` may be x,
 * dt or z themselves (the same pointer and leading dimension); it must not overlap them otherwise, nor B and C.
 * Sequences, slots and states ([n_states][channels][n]) are as with the delta rule.  Long sequences are
 * split into chunks: the chunks' own states first, then outputs from what the chunks before leave, in two launches; else one launch.  Whether and how goes by n_tokens, n_seq,
 * channels and n of the call, so a sequence's last bits depend on how many others, and how long ones, share its call.  The same call is bitwise reproducible.
 * What is not finite stays in its channel (in B or C: its group's) from its token on; it is infinite or NaN there.  Products s A are expected at or below
 * zero: a chunk over which a state would grow by 2^128 counts as infinite growth.  Decays from -2.36e38 down, -infinity among them, count as the lowest numbers: with a
 * step of zero the state stays as it is, with others of 1e-36 and more nothing is left of it.
 * d_ws: csb_scan_workspace_bytes(args) bytes (channels, groups, n, n_seq and n_tokens are read; 0 where there is one launch or a
 * refusal: d_ws may be NULL then).
 * Few tokens, chunks or neither is decided by the mean length of a call's sequences, which is all that the host knows: a few long prompts take longer
 * in one call with many single tokens than in a call of their own (4096 channels, n = 16, bfloat16: a prompt of 2048 tokens among 255 single ones 1900 us, the two apart 76 and 34;
 * one of 8192 among 47 of 100, which are not split for it, 1050, apart 246 and 99).
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range, channels no multiple of groups, n_tokens no
 * multiple of n_seq without d_start, out at the address of B, C or of an x, dt, z with another leading dimension, an unknown type -> CSB_EINVAL; n > 128, n_tokens above 2^31 - 1,
 * or more workgroups than a launch takes -> CSB_EUNSUPPORTED; launch failure -> CSB_EDEVICE.  n_seq = 0 does nothing.
 */
typedef struct {
    int32_t type;                          /* CSB_VAL_*: x, dt, z, B, C and out              */
    int32_t channels, groups;              /* channels a multiple of groups                  */
    int32_t n;                             /* numbers of a channel's state, in [1, 128]      */
    int32_t softplus;
    int32_t n_seq;
    int64_t n_tokens;
    const void *d_x, *d_dt, *d_z, *d_B, *d_C;
    int64_t ldx, lddt, ldz, ldB, ldC;      /* elements from one token to the next            */
    const float *d_A, *d_D, *d_dt_bias;
    const int32_t *d_start, *d_len;
    const float *d_state_in;
    float *d_state_out;
    const int32_t *d_slot;
    int32_t n_states;
    int32_t reserved;                      /* 0                                              */
    void *d_out;
    int64_t ldo;
} csb_scan_args;

size_t csb_scan_workspace_bytes(const csb_scan_args *args);
int csb_selective_scan(const csb_scan_args *args, void *d_ws, void *stream);

/*
 * Norms around a block of a model.  Per token, with the block's output y, a gate, the residual stream x, all but one of y and x optional:
 *     q = y, or y act(gate) with `gate_first`;   p = norm_after(q), times act(gate) where the gate was not first;
 *     r = x + scale s[j] p[j]   (without x: scale s p; without y: x; s NULL: 1);   out = norm_before(r),
 * norm(v)[j] = (v[j] - m) / sqrt(mean((v - m)^2) + eps) w[j] + b[j] with m = mean(v) (CSB_NORM_MEAN), or m = 0 (CSB_NORM_RMS; w NULL: 1, b
 * NULL: 0), CSB_NORM_NONE: v itself; act(v) = v / (1 + e^-v) (CSB_GATE_SILU) or 1 / (1 + e^-v) (CSB_GATE_SIGMOID).
 * norm_after is taken over `groups` equal parts of a token's entries, each by itself.  Every operand has a type and an order of its own:
 * element (t, j) is at t * ld + j, or at j * ld + t with `columns`, which is how csb_spmm* take and leave their operands.
 * d_out of r and of norm_before(r) (both [n_tokens][width]; r may be NULL where norm_before is asked for) are each rounded once, and
 * norm_before is that of r before its rounding.  An output may be an input itself (same pointer, type, order and ld), and must not overlap one
 * otherwise.  Products and sums are binary32, a norm's sums binary64: entries of any finite size have their norm.  What is not finite in
 * a token's entries stays in that token (in its group where there are several): beside infinite entries CSB_NORM_RMS leaves zeros (times w, and b) of the finite ones and
 * NaN of them, CSB_NORM_MEAN NaN of all.
 * Errors: NULL, sizes, types or leading dimensions out of range, eps below zero or not finite, width no multiple of groups, a gate or norm_after without y, norms or gates
 * unknown, an output at the address of an input of another type, order or ld -> CSB_EINVAL; width / groups > 32768, norm_before with several groups, or more workgroups than a launch takes -> CSB_EUNSUPPORTED; launch failure ->
 * CSB_EDEVICE.  n_tokens = 0 does nothing.  Bitwise reproducible, one launch, no workspace.
 */
#define CSB_NORM_NONE 0
#define CSB_NORM_RMS 1
#define CSB_NORM_MEAN 2
#define CSB_GATE_SILU 0
#define CSB_GATE_SIGMOID 1
typedef struct {
    void *d;                               /* NULL: not there                                */
    int64_t ld;
    int32_t type;                          /* CSB_VAL_*                                      */
    int32_t columns;                       /* (t, j) at j * ld + t                           */
} csb_norm_operand;
typedef struct {
    int64_t n_tokens;
    int32_t width, groups;
    int32_t after, before;                 /* CSB_NORM_*                                     */
    int32_t gate_kind, gate_first;         /* CSB_GATE_*                                     */
    float scale, eps;
    csb_norm_operand y, gate, x, r, out;
    const float *d_after_w, *d_after_b, *d_scale, *d_before_w, *d_before_b;      /* [width], or NULL */
} csb_norm_args;

int csb_block_norm(const csb_norm_args *args, void *stream);

/*
 * Sampling.  Row i of logits is at d_logits + i * ld, of `type`; NaN counts as -infinity.  With m the row's largest logit and T
 * = d_temperature[i] (NULL: 1), token v has the weight floor(2^38 e^((logit - m) / T)) in whole units (2^38 for every logit that is m; the
 * exponential in binary64, to 2^-40 of itself).  T not above zero, or NaN: the first token of the order has all of the weight.  The order is by logit, largest first,
 * equal ones by their number, lowest first.  Kept are
 *     the first k = d_top_k[i] tokens of the order (NULL, or k < 1: all);
 *     of these, the ones with fewer units before them than floor(their units * floor(p 2^24) / 2^24), p = d_top_p[i], and the first (NULL, or p
 *     not below 1: all);
 *     of these, the ones of at least floor(min(q, 1) 2^38) units, q = d_min_p[i] (NULL, or q not above 0: all).
 * Token d_tokens[i] is drawn from what is kept by inversion, as csb_verify_drafts does: the lowest whose cumulated units, by number,
 * exceed floor(units of the row * floor(r 2^24) / 2^24), r = d_r[i] in [0, 1) given by the caller; -1 where every logit is -infinity or NaN.
 * d_probs (NULL: not wanted): row i of the distribution drawn from, at d_probs + i * ldprobs, of `type`: units over the row's units, rounded to binary32 and that to `type`, zero for
 * tokens that are not kept; what csb_verify_drafts takes as p and q.  With d_tokens NULL (d_r may be too) only that is made.  It may be the
 * logits themselves (same pointer and leading dimension), and must not overlap them otherwise.  Whole units: the result depends neither on the order nor on the split of a sum.
 * d_ws: csb_sample_workspace_bytes(n_rows, vocab) bytes (0 up to a vocabulary of 24576: d_ws may be NULL then).  One launch where a row has up to 98304
 * bytes, which needs no workspace either (d_ws may be NULL for 16-bit logits up to a vocabulary of 49152), else three to five.
 * Errors: NULL (the optional pointers excepted), sizes or leading dimensions out of range, an unknown type -> CSB_EINVAL; vocab > 2^24, n_rows > 2^21, or
 * more workgroups than a launch takes -> CSB_EUNSUPPORTED; launch failure -> CSB_EDEVICE.  n_rows = 0 does nothing.
 */
size_t csb_sample_workspace_bytes(int32_t n_rows, int32_t vocab);
int csb_sample(int32_t type, const void *d_logits, int64_t ld, const float *d_temperature, const int32_t *d_top_k,
               const float *d_top_p, const float *d_min_p, const float *d_r, int32_t n_rows, int32_t vocab,
               int32_t *d_tokens, void *d_probs, int64_t ldprobs, void *d_ws, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CSBRNN_LM_H */
