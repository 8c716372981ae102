// Rotary positions with several axes: q and k of a layer turned in one kernel, every row by the positions of its token.
//
// Frequency e turns elements e and e + F of a row by position[axis[e]] * inv_freq[e] (the other way round for gradients: the transpose of
// a rotation).  Angles are taken in 64 bits, as turns of which the whole ones are dropped: a position of 20000 leaves fp32 three digits of its
// angle, here it leaves what sine and cosine of an fp32 in [-1, 1] half turns are off by.  A CTA takes a few tokens: their cosines and sines
// once, to shared memory, for all heads of q and k; then every thread turns 8 elements and the 8 that are F behind them, 16 bytes each.  Both
// halves of a row are whole sectors wherever heads and tokens lie, so that no order of the two is slower than the other.
// Bound by HBM.
#include <cuda_bf16.h>

#include "rotary.cuh"

namespace vitcop {
namespace {

constexpr int kThreads = 256, kMostTokens = 16;

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

__global__ void __launch_bounds__(kThreads)
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
        const int axis = min(max(__ldg(k.axis + e), 0), k.axes - 1);
        const int at = __ldcg(k.position + ((int64_t)axis * k.B + b) * k.n_pos + token);
        const double turn = (double)at * (__ldg(k.inv_freq + e) * 0.15915494309189535);        // (1 / 2 pi)
        float s, c;
        sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
        turns[i] = c;
        sines[i] = k.inverse ? -s : s;
    }
    __syncthreads();
    // pieces of a row: 8 elements and their partners, then 8 at a time of what is only copied
    const int turned = F / 8, pieces = turned + (k.d - 2 * F) / 8, heads = k.Hq + k.Hk;
    const int first = blockIdx.z * k.heads, count = min(k.heads, heads - first), total = k.tokens * count * pieces;
    for (int i = tid; i < total; i += kThreads) {
        const int rest = i / pieces, piece = i - rest * pieces, t = rest / count, h = first + rest - t * count;
        if (tokens[t] < 0) continue;
        const bool is_q = h < k.Hq;
        const int64_t hh = is_q ? h : h - k.Hq, r = row0 + t;
        const __nv_bfloat16* const src = is_q ? k.q + b * k.qs[0] + hh * k.qs[1] + r * k.qs[2] : k.k + b * k.ks[0] + hh * k.ks[1] + r * k.ks[2];
        __nv_bfloat16* const dst = is_q ? k.q_out + b * k.qo[0] + hh * k.qo[1] + r * k.qo[2] : k.k_out + b * k.ko[0] + hh * k.ko[1] + r * k.ko[2];
        if (piece >= turned) {
            const int e = 2 * F + (piece - turned) * 8;
            *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(src + e);
            continue;
        }
        const int e = piece * 8;
        const uint4 x = *reinterpret_cast<const uint4*>(src + e), y = *reinterpret_cast<const uint4*>(src + F + e);
        const float4 c0 = *reinterpret_cast<const float4*>(turns + t * F + e), c1 = *reinterpret_cast<const float4*>(turns + t * F + e + 4);
        const float4 s0 = *reinterpret_cast<const float4*>(sines + t * F + e), s1 = *reinterpret_cast<const float4*>(sines + t * F + e + 4);
        const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
        uint32_t u[4], v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a0 = bf16lo(xw[j]), a1 = bf16hi(xw[j]), b0 = bf16lo(yw[j]), b1 = bf16hi(yw[j]);
            u[j] = pair_of(a0 * c[2 * j] - b0 * s[2 * j], a1 * c[2 * j + 1] - b1 * s[2 * j + 1]);
            v[j] = pair_of(b0 * c[2 * j] + a0 * s[2 * j], b1 * c[2 * j + 1] + a1 * s[2 * j + 1]);
        }
        *reinterpret_cast<uint4*>(dst + e) = make_uint4(u[0], u[1], u[2], u[3]);
        *reinterpret_cast<uint4*>(dst + F + e) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

}  // namespace

int launch_rotary_axes(RotaryArgs k, cudaStream_t stream) {
    const int heads = k.Hq + k.Hk;
    k.tokens = k.N < 4 ? k.N : 4;
    k.heads = heads;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((k.N + k.tokens - 1) / k.tokens), (unsigned)k.B, (unsigned)((heads + k.heads - 1) / k.heads));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)k.tokens * k.F * 2 * sizeof(float);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    KernelTimeScope timed("rotary_axes_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, rotary_axes_kernel, k));
}

}  // namespace vitcop
