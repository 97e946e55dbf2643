// Arguments of the dropout operator and its gradient (dm_dropout.cu), shared with the C ABI.
#pragma once
#include "dm_internal.h"

namespace dm {

struct DropoutParams {
    const void* in;        // x[rows][ld_in], or the copies' gradient [rows * K][ld_in]
    void* out;             // copies [rows * K][ld_out], or the gradient of x [rows][ld_out]
    long long ld_in, ld_out, rows;
    int T, K, d;
    int shared_masks;      // 1: the mask key ignores the position
    uint32_t seq_base_lo, key0, key1, thr;
    float scale;           // 1 / (1 - p)
    // set by the launch: chunks of a row, runs of paths, paths of a run, warps' tasks
    int n_chunks, n_groups, group_paths;
    long long n_tasks;
};

int launch_dropout(DropoutParams P, int dtype, bool grad, cudaStream_t stream);

}  // namespace dm
