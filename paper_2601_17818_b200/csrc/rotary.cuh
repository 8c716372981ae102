// Rotary positions with several axes (rotary.cu).
#pragma once

#include <cuda_bf16.h>

#include "kv_attention.cuh"

namespace vitcop {

struct RotaryArgs {
    const __nv_bfloat16 *q, *k;                            // either may be null, with no heads then
    __nv_bfloat16 *q_out, *k_out;
    int64_t qs[3], ks[3], qo[3], ko[3];                    // strides of samples, heads, rows
    const int32_t *position, *token, *seq_len, *axis;
    const double* inv_freq;
    int B, Hq, Hk, N, d, axes, n_pos, F, inverse;
    int tokens;                                            // of a CTA (this and the next are the launcher's)
    Divisor heads, pieces;                                 // of a token, of a row
};
constexpr int kMostFrequencies = 256;                      // of a row
int launch_rotary_axes(RotaryArgs args, cudaStream_t stream);

}  // namespace vitcop
