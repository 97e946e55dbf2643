// Arguments of lossless verification (dm_lossless.cu), shared with the C ABI.
#pragma once
#include "dm_internal.h"

namespace dm {

// Constants of exp(x / T) in fp64 (see weight() in dm_lossless.cu).
struct Exp64 {
    float c16;       // 16 log2(e) / T
    double step;     // T ln2 / 16
    double a[5];     // 1 / (n! T^n), n = 1..5
};

struct LosslessParams {
    const void *target, *draft_logits;   // [B][T + bonus][ld_target], [B][T][ld_draft] or null
    long long ld_target, ld_draft;
    const int32_t *draft, *draft_len;    // [B][T], [B] or null
    int B, T, bonus, V;
    double inv_temp, inv_draft_temp;
    float c, c_draft;                    // log2(e) / temperature
    const float *u_accept, *u_next;      // [B][T], [B]
    float* out_accept_prob;              // [B][T]
    int32_t *out_accept_len, *out_next;  // [B]
    Exp64 e, e_draft;                    // (the rest is set by the launch)
    double table[16];                    // 2^(j/16), j 2^16 taken from the high word
    int share;                           // entries of a CTA's part of a row
};

// Storage types DM_F32 or DM_BF16; draft_dtype is not looked at without draft logits.
int launch_lossless(LosslessParams P, int dtype, int draft_dtype, cudaStream_t stream);

}  // namespace dm
