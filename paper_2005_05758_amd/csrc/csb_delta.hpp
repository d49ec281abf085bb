// The gated delta rule: what its kernels and their launchers share.
#pragma once

#include "csb_lm.hpp"

namespace csb {

struct DeltaDev {                              // the call's arguments as the kernels take them
    const void *q, *k, *v;
    const float *g, *beta;
    const int32_t *start, *len, *slot;
    const float *s_in;
    float *s_out;
    void *out;
    int64_t ldq, ldk, ldv, ldg, ldb, ldo, n_tokens, each;
    int32_t hk, hv, group, dk, dv, n_seq, n_states;
    float scale;
};

Refusal delta_sizes(const csb_delta_args *a);  // of sizes that neither form takes
int check_delta(const char *who, const csb_delta_args *a);
DeltaDev delta_dev(const csb_delta_args *a);
int launch_delta_recurrent(const csb_delta_args *a, hipStream_t st);

#ifdef __HIPCC__
// The tokens of sequence i and the place of its state (negative: none).
__device__ __forceinline__ void delta_sequence(const DeltaDev &a, int i, int64_t *first, int64_t *end, int64_t *slot) {
    sequence_range(a.start, i, a.each, a.n_tokens, first, end);
    if (a.len) *end = *first + clamp64(a.len[i], 0, *end - *first);
    const int32_t s = a.slot ? a.slot[i] : i;
    *slot = s >= 0 && s < a.n_states ? s : -1;
}
#endif

}  // namespace csb
