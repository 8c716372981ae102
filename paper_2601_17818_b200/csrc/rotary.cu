// Rotary positions with several axes: q and k of a layer turned in one kernel, every row by the positions of its token.
//
// Frequency e turns elements e and e + F of a row by position[axis[e]] * inv_freq[e] (the other way round for gradients: the transpose of
// a rotation).  Angles are taken in 64 bits, as turns of which the whole ones are dropped: a position of 20000 leaves fp32 three digits of its
// angle, here it leaves what sine and cosine of an fp32 in [-1, 1] half turns are off by.  A CTA takes a few tokens: their cosines and sines
// once, to shared memory, for all heads of q and k; then every thread turns 8 elements and the 8 that are F behind them, 16 bytes each.  Both
// halves of a row are whole sectors wherever heads and tokens lie, as long as they are multiples of 32 bytes (8 frequencies, or a stride at an odd multiple of 16 bytes,
// take twice the sectors), so that no order of the two is slower than the other.
// Tables are not read as constants (a kernel in front that is still running when this one is launched may be what writes them), nor past the L1: all tokens of an SM want them,
// narrow rows (as the gradient's of 2 x 2943 rows of 32 heads of 64) 10.6 us instead of 11.1.
// Bound by HBM: 4 x 4672 tokens, 32 heads of 128 in all, 49.7 us (0.94 of the copy rate; one pair of pieces a thread at a time 54.2); 8 x 704 kept rows of
// 64 heads 31.2 us (0.90); one token 2.6 us.  Not by it where rows are few or narrow: 2 x 2943 rows of 32 heads of 64, half turned, 10.6 us (0.70), whose CTAs wait for token,
// position and angles, one after the other, before their first row and then have two rounds of rows.
#include <algorithm>

#include <cuda_bf16.h>

#include "rotary.cuh"

namespace vitcop {
namespace {

constexpr int kThreads = 256, kMostTokens = 16, kPieces = 1024, kAtOnce = 2;

// (a b) rounded to bf16, the first in the lower half
__device__ __forceinline__ uint32_t pair_of(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Token of row r of sample b, or -1: the row stays as it is.
__device__ __forceinline__ int token_of(const RotaryArgs& k, int b, int r) {
    if (r >= k.N || (k.seq_len && r >= __ldcg(k.seq_len + b))) return -1;
    return k.token ? min(__ldcg(k.token + (int64_t)b * k.N + r), k.n_pos - 1) : r;
}

__global__ void __launch_bounds__(kThreads, 6)
rotary_axes_kernel(const __grid_constant__ RotaryArgs k) {
    extern __shared__ float turns[];                       // [tokens][F] cosines, then as many sines
    __shared__ int tokens[kMostTokens];
    grid_dependency_wait();
    grid_dependency_launch_dependents();
    const int row0 = blockIdx.x * k.tokens, b = blockIdx.y, tid = threadIdx.x, F = k.F;
    if (tid < k.tokens) tokens[tid] = token_of(k, b, row0 + tid);
    __syncthreads();
    float* const sines = turns + k.tokens * F;
    for (int i = tid; i < k.tokens * F; i += kThreads) {
        const int t = i / F, e = i - t * F, token = tokens[t];
        if (token < 0) continue;
        const int axis = min(max(k.axis[e], 0), k.axes - 1);
        const int at = __ldcg(k.position + ((int64_t)axis * k.B + b) * k.n_pos + token);
        const double turn = (double)at * (k.inv_freq[e] * 0.15915494309189535);        // (1 / 2 pi)
        float s, c;
        sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
        turns[i] = c;
        sines[i] = k.inverse ? -s : s;
    }
    __syncthreads();
    // pieces of a row: 8 elements and their partners, then 8 at a time of what is only copied; a thread fetches two in front of working on either
    const int turned = F / 8, pieces = (int)k.pieces.d, heads = k.Hq + k.Hk, total = k.tokens * heads * pieces;
    for (int i0 = tid; i0 < total; i0 += kAtOnce * kThreads) {
        uint4 x[kAtOnce], y[kAtOnce];
        __nv_bfloat16* to[kAtOnce];
        int at[kAtOnce];                                   // of its cosines; < 0: a copy
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            const int i = i0 + n * kThreads;
            to[n] = nullptr;
            if (i >= total) continue;
            const int rest = quotient(i, k.pieces), piece = i - rest * pieces, t = quotient(rest, k.heads), h = rest - t * heads;
            if (tokens[t] < 0) continue;
            const bool is_q = h < k.Hq;
            const int64_t hh = is_q ? h : h - k.Hq, r = row0 + t;
            const int e = piece < turned ? piece * 8 : F + piece * 8;
            const __nv_bfloat16* const src = (is_q ? k.q + b * k.qs[0] + hh * k.qs[1] + r * k.qs[2] : k.k + b * k.ks[0] + hh * k.ks[1] + r * k.ks[2]) + e;
            to[n] = (is_q ? k.q_out + b * k.qo[0] + hh * k.qo[1] + r * k.qo[2] : k.k_out + b * k.ko[0] + hh * k.ko[1] + r * k.ko[2]) + e;
            at[n] = piece < turned ? t * F + e : -1;
            x[n] = __ldcs(reinterpret_cast<const uint4*>(src));
            if (piece < turned) y[n] = __ldcs(reinterpret_cast<const uint4*>(src + F));
        }
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            if (!to[n]) continue;
            if (at[n] < 0) {
                __stcs(reinterpret_cast<uint4*>(to[n]), x[n]);
                continue;
            }
            const float4 c0 = *reinterpret_cast<const float4*>(turns + at[n]), c1 = *reinterpret_cast<const float4*>(turns + at[n] + 4);
            const float4 s0 = *reinterpret_cast<const float4*>(sines + at[n]), s1 = *reinterpret_cast<const float4*>(sines + at[n] + 4);
            const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
            const uint32_t xw[4] = {x[n].x, x[n].y, x[n].z, x[n].w}, yw[4] = {y[n].x, y[n].y, y[n].z, y[n].w};
            uint32_t u[4], v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a0 = bf16lo(xw[j]), a1 = bf16hi(xw[j]), b0 = bf16lo(yw[j]), b1 = bf16hi(yw[j]);
                u[j] = pair_of(a0 * c[2 * j] - b0 * s[2 * j], a1 * c[2 * j + 1] - b1 * s[2 * j + 1]);
                v[j] = pair_of(b0 * c[2 * j] + a0 * s[2 * j], b1 * c[2 * j + 1] + a1 * s[2 * j + 1]);
            }
            __stcs(reinterpret_cast<uint4*>(to[n]), make_uint4(u[0], u[1], u[2], u[3]));
            __stcs(reinterpret_cast<uint4*>(to[n] + F), make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

}  // namespace

int launch_rotary_axes(RotaryArgs k, cudaStream_t stream) {
    const int heads = k.Hq + k.Hk;
    k.heads = divisor(heads);
    k.pieces = divisor(k.F / 8 + (k.d - 2 * k.F) / 8);
    const int64_t row = (int64_t)heads * k.pieces.d;
    k.tokens = std::min(k.N, (int)std::max<int64_t>(1, std::min<int64_t>(kMostTokens, (kPieces + row / 2) / row)));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((k.N + k.tokens - 1) / k.tokens), (unsigned)k.B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)k.tokens * k.F * 2 * sizeof(float);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    KernelTimeScope timed("rotary_axes_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, rotary_axes_kernel, k));
}

}  // namespace vitcop
