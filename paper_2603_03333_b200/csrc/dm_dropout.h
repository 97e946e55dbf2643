// Arguments of the dropout operator and its gradient (dm_dropout.cu), shared with the C ABI.
#pragma once
#include "dm_internal.h"

namespace dm {

// Division of numbers below 2^31 by a fixed d: n / d = n m >> (31 + s) with s = ceil(log2 d), m = ceil(2^(31+s) / d), since
// m d - 2^(31+s) < d <= 2^s.
struct Divisor {
    uint32_t d = 1, m = 0x80000000u, s = 31;
    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by) {
        while ((1ull << (s - 31)) < d) ++s;
        m = (uint32_t)(((1ull << s) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((unsigned long long)n * m) >> s); }
};

struct DropoutParams {
    const void* in;        // x[rows][ld_in], or the copies' gradient [rows * K][ld_in]
    void* out;             // copies [rows * K][ld_out], or the gradient of x [rows][ld_out]
    long long ld_in, ld_out, rows;
    int T, K, d;
    int shared_masks;      // 1: the mask key ignores the position
    uint32_t seq_base_lo;
    // set by the launch: threshold and 1 / (1 - p), the generator's round keys (read as constants, they cost no instruction);
    // paths of a run; warps' tasks, and how to get from one to chunk, run of paths, row and position
    uint32_t thr;
    float scale;
    uint32_t key[10][2];
    int group_paths;
    uint32_t n_tasks;
    Divisor by_chunks, by_groups, by_T;
};

int launch_dropout(DropoutParams P, const MaskKey& mk, int dtype, bool grad, cudaStream_t stream);

}  // namespace dm
