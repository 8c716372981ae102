// Attention of query rows over the K/V cache in 4 bits: out = softmax(scale q K^T) V over the rows that a query sees.
//
// A CTA takes one query row; its warps share out the tokens, keep their own maximum, sum and output of the softmax, and join them.
#include "f32x2.cuh"
#include "kv_cache.cuh"

namespace vitcop {
namespace {

constexpr int kAttWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ld_bf16(const uint8_t* p) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }

template <int D>
__global__ void __launch_bounds__(kAttWarps * 32)
cache_attention_kernel(CacheQueries io, const uint8_t* cache, int Hq, int H, int Tq, int Ncap, const int32_t* cache_len,
                       float scale, int causal, float* lse, int* status) {
    using L = CacheBlock<D>;
    constexpr int G = L::G;
    grid_dependency_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = VITCOP_OK;
    const int tq = blockIdx.x % Tq, bq = blockIdx.x / Tq, hq = bq % Hq, b = bq / Hq, h = hq / (Hq / H);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int len = cache_len ? max(0, min(cache_len[b], Ncap)) : Ncap;
    const int limit = causal ? max(0, len - Tq + tq + 1) : len;
    const uint8_t* const head = cache + ((int64_t)b * H + h) * (Ncap / kCacheBlock) * L::kBytes;
    float q[G], o[G] = {}, mx = -__builtin_huge_valf(), sum = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) q[g] = __bfloat162float(io.q[b * io.qb + hq * io.qh + tq * io.qt + g * 32 + lane]) * scale;
    for (int j = warp; j < limit; j += kAttWarps) {
        const uint8_t* const block = head + (int64_t)(j / kCacheBlock) * L::kBytes;
        const int row = j % kCacheBlock;
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int byte = block[L::kKCodes + row * (D / 2) + lane / 8 * 4 * G + g * 4 + lane % 8 / 2];
            const float c = (float)((byte >> (lane % 2 * 4) & 15) - 8);
            s = fmaf(q[g], fmaf(c, ld_bf16(block + L::kKScale + (row * G + g) * 2), ld_bf16(block + L::kKCentre + (row * G + g) * 2)), s);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        const float top = fmaxf(mx, s), keep = mx == top ? 1.f : exp2f((mx - top) * kLog2e), p = exp2f((s - top) * kLog2e);
        mx = top;
        sum = fmaf(sum, keep, p);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int byte = block[L::kVCodes + row * (D / 2) + lane / 4 * 2 * G + g * 2 + lane % 4 / 2];
            const float c = (float)((byte >> (lane % 2 * 4) & 15) - 8);
            const float v = fmaf(c, ld_bf16(block + L::kVScale + (row * G + g) * 2), ld_bf16(block + L::kVCentre + (g * 32 + row) * 2));
            o[g] = fmaf(o[g], keep, p * v);
        }
    }
    __shared__ float wmax[kAttWarps], wsum[kAttWarps], wout[kAttWarps][D];
    if (lane == 0) {
        wmax[warp] = mx;
        wsum[warp] = sum;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) wout[warp][g * 32 + lane] = o[g];
    __syncthreads();
    float top = -__builtin_huge_valf(), total = 0.f;
    for (int w = 0; w < kAttWarps; ++w) top = fmaxf(top, wmax[w]);
    float f[kAttWarps];
    for (int w = 0; w < kAttWarps; ++w) {
        f[w] = wmax[w] == top ? 1.f : exp2f((wmax[w] - top) * kLog2e);
        total += wsum[w] * f[w];
    }
    for (int e = threadIdx.x; e < D; e += kAttWarps * 32) {
        float v = 0.f;
        for (int w = 0; w < kAttWarps; ++w) v = fmaf(wout[w][e], f[w], v);
        io.out[b * io.ob + hq * io.oh + tq * io.ot + e] = __float2bfloat16_rn(limit > 0 ? v / total : 0.f);
    }
    if (lse && threadIdx.x == 0) lse[((int64_t)b * Hq + hq) * Tq + tq] = limit > 0 ? top + logf(total) : -__builtin_huge_valf();
}

}  // namespace

size_t cache_attention_workspace_bytes(int, int, int, int, int, int) { return kStatusBytes; }

int launch_cache_attention(const CacheQueries& io, const void* cache, int B, int Hq, int H, int Tq, int d, int Ncap,
                           const int32_t* cache_len, float scale, bool causal, float* lse, void* workspace, cudaStream_t stream) {
    if ((int64_t)B * Hq * Tq > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(B * Hq * Tq));
    cfg.blockDim = dim3(kAttWarps * 32);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    KernelTimeScope timed("cache_attention_kernel", stream);
    auto kern = d == 64 ? cache_attention_kernel<64> : d == 128 ? cache_attention_kernel<128> : cache_attention_kernel<256>;
    return record_cuda(cudaLaunchKernelEx(&cfg, kern, io, static_cast<const uint8_t*>(cache), Hq, H, Tq, Ncap, cache_len, scale,
                                          causal ? 1 : 0, lse, static_cast<int*>(workspace)));
}

}  // namespace vitcop
