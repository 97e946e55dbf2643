// Arguments of the row operators (dm_rows.cu), shared with the C ABI.
#pragma once
#include "dm_internal.h"

namespace dm {

constexpr int kRowsMaxTop = DM_MAX_TOP;   // alternatives, and teacher tokens, of a row
constexpr int kRowsMaxCluster = 8;        // CTAs that share a row
constexpr int kRowsMaxV = 1 << 30;

struct RowsParams {
    const void* logits;   // [rows][ld], entries 0..V-1 of a row
    long long ld;
    int V, rows;
    float inv_temp;       // 1 / T
    float c;              // log2(e) / T
    double inv_temp_d;
    float gap;            // 250 / c: what lies farther below the maximum is nothing
    int stash_vecs;       // 16-byte vectors in shared memory: a CTA's share, or the ring it streams through (set by the launch)
    int n_batches;        // batches of the longest share (set by the launch)
    int slot_batches, n_slots;   // batches of a thread that share one remembered maximum, and how many of those (set by the launch)
    const uint32_t* err;  // device error word of the kernel that wrote the logits, or null
    uint32_t* err_out;    // device error word of the call's context
    long long wait_limit; // clock cycles that a wait for the next row may take
    // logprobs
    const int32_t* tokens;
    int n_top;
    float *out_logprob, *out_lse, *out_entropy, *out_top_logprob;
    int32_t* out_top_ids;
    // gradients
    const float *g_logprob, *g_entropy;
    void* out_grad;
    long long ld_grad;
    // distill
    const int32_t* t_ids;
    const float *t_logprob, *weight;
    int k, tail;
    float* out_loss;
};

// dtype: DM_F32 or DM_BF16 (logits and their gradient).  Only enqueue work; DM_EUNSUPPORTED where a
// share of a row does not fit what a CTA needs to know about it in shared memory.
int launch_rows_logprobs(const RowsParams& P, int dtype, cudaStream_t stream);
int launch_rows_grad(const RowsParams& P, int dtype, cudaStream_t stream);
int launch_rows_distill(const RowsParams& P, int dtype, cudaStream_t stream);

// The gradient kernels whose rows stay in shared memory.  False: the row is too long for that, nothing
// was launched; true: *status is the outcome.
bool launch_rows_resident(const RowsParams& P, int dtype, bool distill, cudaStream_t stream, int* status);

}  // namespace dm
