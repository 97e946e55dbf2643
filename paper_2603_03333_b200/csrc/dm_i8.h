// Products of 8-bit integer matrices with scales (dm_i8_sm100.cu), shared with the C ABI.
#pragma once
#include "dm_internal.h"

namespace dm {

constexpr int kI8MaxDepth = 131071;   // terms of a sum: 131071 * 128 * 128 < 2^31

struct QuantizeParams {
    const void* x;
    long long ld, n_rows;
    int n;
    int8_t* q;
    long long ld_q;
    float* scale;
};
int launch_quantize_i8(const QuantizeParams& P, int dtype, cudaStream_t stream);

struct I8Args {
    const int8_t *a, *w;          // [n_rows][ld_a], [V][ld_w]: 16-byte aligned rows
    long long ld_a, ld_w;
    const float *a_scale, *w_scale;
    int n_rows, V, d;
    void* out;                    // [n_rows][ld_out]
    int out_dtype;
    long long ld_out;
    uint32_t* err;
    long long wait_limit;
    bool behind_quantize;         // the kernel ahead in the stream wrote a and a_scale and nothing else, and was launched without overlap
};
int launch_matmul_i8(const I8Args& A, cudaStream_t stream);

}  // namespace dm
